"""RotaryTable and PagedCache on the GPU: what their host side decides."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_two_streams_attend_beside_each_other():
    from paper_2609_29812_b200 import binding as B, pipeline as P
    with B.Context(0) as ctx:
        c = P.PagedCache(ctx, 2, 4, 128, 5000)
        g = torch.Generator(device="cuda").manual_seed(0)
        rows = lambda n, h: torch.randn(n, h, 128, generator=g, device="cuda").to(torch.bfloat16)
        x = rows(5000, 4)
        c.append(x, x.flip(0), [4999, 1])
        q = [rows(2, 4) for _ in range(2)]
        one = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
        want = [c.attend(v, [1, 1], 0.1, one) for v in q]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = [[], []]
        for _ in range(20):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    got[i].append(c.attend(q[i], [1, 1], 0.1, one))
        torch.cuda.synchronize()
        for i in range(2):
            for o, lse in got[i]:
                assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])
        c.check_status()


def test_positions_outside_a_table_are_reported():
    from paper_2609_29812_b200 import binding as B, pipeline as P
    with B.Context(0) as ctx:
        t = P.RotaryTable(ctx, 10, 64)
        x = torch.randn(3, 1, 64, device="cuda")
        t.rotate(x, torch.tensor([0, 9, 5], dtype=torch.int32, device="cuda"))
        t.check_status()
        t.rotate(x, torch.tensor([0, 10, 5], dtype=torch.int32, device="cuda"))
        with pytest.raises(B.FlashLoopError) as e:
            t.check_status()
        assert e.value.status == B.FL_ERR_INVALID_ARG
