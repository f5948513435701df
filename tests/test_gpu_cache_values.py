"""Attention over a paged 8-bit cache that holds values at the ends of their range, against the 64-bit form: the kernel of few rows, the
one of chunks (more than 128 rows of a sequence) and the one of binary32 storage have to agree with the definition and so with each other."""
import math

import pytest

import cache_reference as ref
from test_gpu_cache import Cache, env, rows  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"

KERNELS = [("bf16", 3), ("bf16", 16), ("bf16", 290), ("f32", 16), ("f32", 290)]


# ------------------------------------------------------------------------------------------------
# keys and values that are zeros
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,new", KERNELS)
@pytest.mark.parametrize("page,code,dim", [(16, "int8", 128), (64, "e4m3", 128), (64, "int8", 64), (16, "e4m3", 64), (128, "int8", 128)])
def test_blocks_of_zero_keys(env, dtype, new, page, code, dim):
    """Padding tokens: whole blocks of zero keys before a row, around it and after it."""
    B, ctx = env
    c = Cache(B, 3, 700, page=page, code=code, dtype=dtype, n_kv=2, dim=dim)
    g = torch.Generator().manual_seed(31)
    lens = [650, 310, new]
    n = sum(lens)
    k = rows(g, n, 2, dim, c.dt)
    for first, end in ((64, 128), (256, 384), (500, 640), (650 + 128, 650 + 256), (650 + 310, 650 + 310 + min(new, 128))):
        k[first:end, 0] = 0.0
    k[128:256, 1] = 1e-33                                      # below 2^-100: the same
    c.append(ctx, lens, k, rows(g, n, 2, dim, c.dt), check=False)
    c.check_attention(ctx, rows(g, 3 * new, 4, dim, c.dt), [new] * 3, f"{dtype} {new}")


@pytest.mark.parametrize("dtype,new", KERNELS)
@pytest.mark.parametrize("page,dim", [(16, 128), (64, 64)])
def test_zero_queries_beside_zero_keys(env, dtype, new, page, dim):
    """Rows of zeros, as queries and as the open block's keys: every logit is zero, a row's output the mean of the values that it sees."""
    B, ctx = env
    c = Cache(B, 2, 400, page=page, dtype=dtype, n_kv=1, dim=dim)
    g = torch.Generator().manual_seed(32)
    lens = [page * (300 // page) + 9, page * (256 // page) + page - 1]
    k = rows(g, sum(lens), 1, dim, c.dt)
    k[lens[0] - 9:lens[0]] = 0.0
    k[lens[0] + 100:] = 0.0
    c.append(ctx, lens, k, rows(g, sum(lens), 1, dim, c.dt), check=False)
    q = rows(g, 2 * new, 2, dim, c.dt)
    q[::2, 0] = 0.0
    q[1::2, 1] = 1e-36
    c.check_attention(ctx, q, [new] * 2, f"{dtype} {new}")


@pytest.mark.parametrize("dtype,new", KERNELS)
def test_rows_that_see_nothing_beside_zero_keys(env, dtype, new):
    B, ctx = env
    c = Cache(B, 2, 400, page=16, dtype=dtype, n_kv=1, dim=64)
    g = torch.Generator().manual_seed(33)
    lens = [max(1, new - 5), max(1, new // 2)]
    k = rows(g, sum(lens), 1, 64, c.dt)
    k[:lens[0] // 16 * 16] = 0.0
    c.append(ctx, lens, k, rows(g, sum(lens), 1, 64, c.dt), check=False)
    o, lse = c.check_attention(ctx, rows(g, 2 * new, 1, 64, c.dt), [new] * 2, f"{dtype} {new}")
    unseen = new - lens[0]
    assert not o[:max(0, unseen)].any() and torch.isneginf(lse[:max(0, unseen)]).all()


# ------------------------------------------------------------------------------------------------
# values far apart
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,new", KERNELS)
@pytest.mark.parametrize("page,code", [(16, "int8"), (64, "e4m3"), (128, "int8")])
def test_values_of_very_different_size(env, dtype, new, page, code):
    """Blocks of values around 1e30, 1, 1e-20 and 0 in every order: log-normalisers do not know values, outputs are those of the formula."""
    B, ctx = env
    c = Cache(B, 4, 900, page=page, code=code, dtype=dtype, n_kv=2, dim=64)
    g = torch.Generator().manual_seed(34)
    lens = [807, 640, 300 + new, 513]
    k, v = rows(g, sum(lens), 2, 64, c.dt), rows(g, sum(lens), 2, 64, torch.float32)
    sizes = [[1e30, 1e-20, 0.0, 1.0, 1e-12, 1e30, 1e-30], [1e-20, 1e30, 1.0, 0.0, 1e-12], [0.0, 1e-30, 1e-12, 1e30, 1.0], [1.0, 1e30, 1e-20, 1e-35, 0.0]]
    at = 0
    for n, order in zip(lens, sizes):
        for j in range(0, n, 128):
            v[at + j:at + min(j + 128, n), 0] *= order[j // 128 % len(order)]
        at += n
    c.append(ctx, lens, k, v.to(c.dt), check=False)
    c.check_attention(ctx, rows(g, 4 * new, 4, 64, c.dt), [new] * 4, f"{dtype} {new}")


# ------------------------------------------------------------------------------------------------
# scales that another program wrote
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,new", KERNELS)
@pytest.mark.parametrize("page,code", [(16, "e4m3"), (64, "int8")])
def test_scale_zero_beside_codes_that_are_not(env, dtype, new, page, code):
    """A value is code * scale, whoever wrote the two: keys and values of a block of scale zero are zeros whatever its codes."""
    B, ctx = env
    c = Cache(B, 2, 700, page=page, code=code, dtype=dtype, n_kv=1, dim=128)
    g = torch.Generator().manual_seed(35)
    lens = [600, 290 + page]
    c.append(ctx, lens, rows(g, sum(lens), 1, 128, c.dt), rows(g, sum(lens), 1, 128, c.dt), check=False)
    for b in range(2):
        for side, step in ((0, 3), (1, 2)):
            for j in range(1, lens[b] // page, step):
                c.scale[side][int(c.table_host[b, j])] = 0.0
                c.rows[side][b][j * page:(j + 1) * page] = 0.0
    c.check_attention(ctx, rows(g, 2 * new, 2, 128, c.dt), [new] * 2, f"{dtype} {new}")


# ------------------------------------------------------------------------------------------------
# blocks with infinities and NaN
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,new", KERNELS)
@pytest.mark.parametrize("page,code", [(16, "int8"), (64, "e4m3")])
@pytest.mark.parametrize("side", [0, 1])
def test_every_row_that_sees_a_block_without_a_scale_is_none(env, dtype, new, page, code, side):
    """Output and log-normaliser of rows that see a token of the block, also where its tokens' probabilities are zeros beside a dominant
    key; rows before the block are as without it."""
    B, ctx = env
    g = torch.Generator().manual_seed(36)
    n_seqs, dim = 3, 128
    lens = [page * (700 // page), page * (420 // page) + 3, page * (330 // page)]
    c = Cache(B, n_seqs, 720, page=page, code=code, dtype=dtype, n_kv=1, dim=dim)
    k, v = rows(g, sum(lens), 1, dim, torch.float32, 0.1), rows(g, sum(lens), 1, dim, c.dt)
    first = []                                                 # tokens before the bad block
    at = 0
    for b, (n, dominant, bad) in enumerate(zip(lens, (650, 7, 9), (100, lens[1] - 10, lens[2] - 1))):
        k[at + dominant] = 4.0                                 # logits 180 above the others: 2^-126 and less is left of those
        (k if side == 0 else v)[at + bad, 0, 5] = math.inf if b else math.nan
        first.append(bad // page * page)
        at += n
    c.append(ctx, lens, k.to(c.dt), v, check=False)
    q = (rows(g, n_seqs * new, 2, dim, torch.float32, 0.1) + 4.0).to(c.dt)
    o, lse = c.attend(ctx, q, [new] * n_seqs)
    for b in range(n_seqs):
        s = slice(b * new, (b + 1) * new)
        blind = max(0, min(new, first[b] - (lens[b] - new)))   # rows that see no token of the block
        assert torch.isnan(o[s][blind:]).all() and torch.isnan(lse[s][blind:]).all(), b
        if blind:
            want = ref.attention(q[s][:blind].double(), c.held(0, b)[:lens[b] - new + blind], c.held(1, b)[:lens[b] - new + blind], 2, dim ** -0.5)
            ref.assert_attention(o[s][:blind], lse[s][:blind], want, dim, dtype == "bf16", f"sequence {b}")


# ------------------------------------------------------------------------------------------------
# the range that rows beyond a row's own tokens leave it
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,new", KERNELS)
@pytest.mark.parametrize("page,length", [(64, 640 + 20), (16, 640 + 9), (64, 640), (128, 700)])
def test_much_larger_rows_that_come_later(env, dtype, new, page, length):
    """Keys and values 2^20 times larger in the last tokens: rows before them keep the bits that the header promises (an open key 2^-39 of
    its block's largest, which the bound on the logits holds up to 2^24; p v 2^-31 of the sequence's largest value)."""
    B, ctx = env
    c = Cache(B, 1, 720, page=page, dtype=dtype, n_kv=2, dim=128)
    g = torch.Generator().manual_seed(37)
    k, v = rows(g, length, 2, 128, c.dt), rows(g, length, 2, 128, c.dt)
    k[length - 2:] *= 2.0 ** 20
    v[length - 2:] *= 2.0 ** 20
    c.append(ctx, [length], k, v, check=False)
    c.check_attention(ctx, rows(g, new, 4, 128, c.dt), [new], f"{dtype} {new}")
