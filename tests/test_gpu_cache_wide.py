"""Launches that are large enough for several heads per CTA (append) or per thread (rotation), bit by bit like the small ones.  Each test
first looks whether its sizes are: the rules are those of csrc/kv_cache.cu and csrc/rope.cu, by the device's number of SMs."""
import pytest

import cache_reference as ref
from test_gpu_cache import Cache, env, fl, ints, rows, same_bits  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


def heads_per_cta(n_tokens, n_seqs, page, n_kv):
    by_block = n_tokens // page + 2 * n_seqs
    units, enough = min(n_tokens, by_block), 2 * torch.cuda.get_device_properties(0).multi_processor_count
    return 8 if units * -(-n_kv // 8) >= enough else 4 if units * -(-n_kv // 4) >= enough else 1


WIDE = [dict(n_kv=11, page=16, per=8, n=1300), dict(n_kv=7, page=16, per=4, n=1200, layout="pairs", code="e4m3"), dict(n_kv=3, page=16, per=8, n=2500, rot=20),
        dict(n_kv=9, page=32, per=8, n=2400, dim=64, rot=32, slab=True), dict(n_kv=12, page=64, per=8, n=4700, rot=0), dict(n_kv=5, page=16, per=4, n=1210, odd=True, dim=64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", WIDE, ids=str)
def test_append_with_several_heads_per_cta(env, case, dtype):
    B, ctx = env
    page, dim, n_kv, code, layout = case["page"], case.get("dim", 128), case["n_kv"], case.get("code", "int8"), case.get("layout", "half")
    rot = case.get("rot", dim)
    table = ref.make_table(rot, 6000) if rot else None
    td = table.to(DEV) if rot else None
    rope = B.make_rope(td, 6000, rot, fl(B, layout)) if rot else None
    c = Cache(B, 2, case["n"] + 200, page=page, code=code, dtype=dtype, n_kv=n_kv, dim=dim)
    g = torch.Generator().manual_seed(41)
    new = [case["n"], case["n"] - 3]
    assert heads_per_cta(sum(new), 2, page, n_kv) == case["per"]
    for cut in ([5, page - 1], new, [page, 1]):              # the large one begins and ends inside blocks
        n = sum(cut)
        c.append(ctx, cut, rows(g, n, n_kv, dim, c.dt), rows(g, n, n_kv, dim, c.dt, 3.0), rope, table, rot, layout, slab=case.get("slab", False),
                 odd=case.get("odd", False), check=False)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_a_step_that_fills_the_largest_blocks(env, dtype):
    """One token each for more sequences than half the CTAs' number: every block of 128 tokens is coded by 512 threads, two heads in turn."""
    B, ctx = env
    n_seqs = 2 * torch.cuda.get_device_properties(0).multi_processor_count + 4
    table = ref.make_table(128, 200)
    td = table.to(DEV)
    rope = B.make_rope(td, 200, 128, B.FL_ROPE_HALF)
    c = Cache(B, n_seqs, 128, page=128, dtype=dtype, n_kv=2)
    g = torch.Generator().manual_seed(42)
    for per in (127, 1):
        n = per * n_seqs
        assert heads_per_cta(n, n_seqs, 128, 2) == 8
        c.append(ctx, [per] * n_seqs, rows(g, n, 2, 128, c.dt), rows(g, n, 2, 128, c.dt), rope, table, 128, "half", check=False)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim,rot,layout,slab", [(5, 128, 128, "half", False), (7, 64, 32, "pairs", True), (6, 128, 96, "half", True)])
def test_rotation_of_four_heads_a_thread_where_their_number_is_odd(env, heads, dim, rot, layout, slab, dtype):
    B, ctx = env
    groups = -(-heads // 4)
    n = -(-torch.cuda.get_device_properties(0).multi_processor_count * 1024 // (groups * (dim // 16))) + 3
    g = torch.Generator().manual_seed(43)
    pos = torch.randint(0, 5000, (n,), generator=g, dtype=torch.int32)
    x = torch.randn(n, heads, dim, generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    table = ref.make_table(rot, 5000)
    td = table.to(DEV)
    rope = B.make_rope(td, 5000, rot, fl(B, layout))
    xd = x.to(DEV)
    if slab:
        big = torch.zeros(n, 3, heads, dim, dtype=x.dtype, device=DEV)
        big[:, 1] = xd
        xd = big[:, 1]
    for inverse in (False, True):
        y = torch.full((n + 1, heads, dim), 7.0, dtype=x.dtype, device=DEV)
        B.fl_rotate_rows(ctx, xd, xd.stride(0), pos.to(DEV), n, heads, dim, fl(B, dtype), rope, inverse, y, heads * dim)
        assert same_bits(y[:n], ref.rotate(x, pos, table, rot, layout, inverse).to(x.dtype)) and bool((y[n] == 7.0).all())
