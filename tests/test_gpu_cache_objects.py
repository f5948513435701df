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


def test_the_example_s_second_loop_starts_from_the_cache():
    """Loop 2 of the decode steps against the oracle, which takes the prompt's rows as the cache holds them for loop 1, the residuals' codec
    for loop 2, and loop 1's outputs and log-normalisers as the attention over the cache gave them."""
    import numpy as np

    from helpers import assert_attn_close, to_np
    from oracle import flashloop_oracle as fo
    from test_gpu_cache_path import example
    prompt, columns, steps = 500, 64, 2                      # (the prompt's last block stays open over both steps)
    r = example().run(prompt=prompt, steps=steps, chunk=192, columns=columns, page=64)
    base = [to_np(r[s][:prompt]) for s in ("k", "v")]
    hat = [fo.residual_update(to_np(r[s + "2"]), b, np.arange(prompt), 4, 128)[0] for s, b in zip("kv", base)]
    for i, d in enumerate(r["decode"]):
        q, q2, cols, lse1 = to_np(d["q"]), to_np(d["q2"]), d["cols"].cpu().numpy(), d["lse1"].double().cpu().numpy()
        heads = q.shape[1]
        sets = {(0, h): cols[0, h] for h in range(heads)}
        p_old = {(0, h): np.exp(base[0][cols[0, h], h].astype("f8") @ q[0, h].astype("f8") * r["sm_scale"] - lse1[0, h]) for h in range(heads)}
        want = fo.decode_sparse_attention(q2, hat[0], hat[1], base[1], to_np(d["o1"]).astype("f8"), sets, p_old, r["sm_scale"], kv_round=fo.round_bf16)
        assert_attn_close(to_np(d["o2"]), want["O"], f"example, token {i}")
        np.testing.assert_allclose(to_np(d["lse2"]), want["lse"], rtol=0, atol=5e-3)
        assert np.linalg.norm(want["O"] - to_np(d["o1"])) > 5 * 1e-2 * np.linalg.norm(want["O"])    # (what loop 2 does is well above the bound)


def test_a_captured_attend_has_a_workspace_of_its_own():
    from paper_2609_29812_b200 import binding as B, pipeline as P
    with B.Context(0) as ctx:
        c = P.PagedCache(ctx, 1, 2, 64, 3000)
        g = torch.Generator(device="cuda").manual_seed(1)
        x = torch.randn(3000, 2, 64, generator=g, device="cuda").to(torch.bfloat16)
        c.append(x[:2999], x[:2999], [2999])
        q = x[:1].clone()
        one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        want = c.attend(q, [1], 0.125, one)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, lse = c.attend(q, [1], 0.125, one)
        again = c.attend(q, [1], 0.125, one)                    # what the capture allocated is not in the way of later calls
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
        for _ in range(3):
            o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        q.copy_(x[7:8])
        graph.replay()
        other = c.attend(q, [1], 0.125, one)
        assert torch.equal(o, other[0]) and not torch.equal(o, want[0])
        c.check_status()
        c.append(x[2999:], x[2999:], [1])                       # (lets go of the lengths that the graph reads)
        torch.cuda.synchronize()
        del graph
