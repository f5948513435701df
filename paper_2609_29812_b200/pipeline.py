"""Call-order harness for one layer: allocates device buffers with PyTorch and calls the C-ABI
entry points in the order of the hot path.  No arithmetic of the method lives here; every step
runs inside libflashloop's kernels.

Per-layer state carried across loops (all caller-owned device tensors):
  k_base, v_base [L,H,dh]      loop-1 K/V (storage type)
  streams[r-2]                 residual payloads of loop r: codes, scale, zero (K and V)
  q_store, o_store [L,H,dh]    latest Q and attention output of every position
  lse [H,L]                    latest log-normaliser of every (head, position), updated in place
  col_idx [H,nb,c], col_cnt    selected columns per (head, query block)
"""
from __future__ import annotations

import itertools
from dataclasses import dataclass
from typing import List, Optional

import torch

from . import binding as B
from .workloads import Workload


def torch_dtype(w: Workload):
    return torch.float32 if w.dtype == "f32" else torch.bfloat16


def fl_dtype(w: Workload) -> int:
    return B.FL_F32 if w.dtype == "f32" else B.FL_BF16


def shape_of(w: Workload, bits: Optional[int] = None, q_block: Optional[int] = None):
    return B.make_shape(w.L, w.n_heads, w.head_dim, fl_dtype(w), q_block or w.q_block, bits or w.bits, w.group,
                        w.eps, w.sm_scale)


@dataclass
class TokenSelection:
    active_idx: torch.Tensor     # int32 [n]
    slot_of_pos: torch.Tensor    # int32 [L]
    scores: torch.Tensor         # f32 [n_cand]
    n: int


def select_tokens(ctx, shape, loop_r, g_prev, g_cur, cand: Optional[torch.Tensor], k: int) -> TokenSelection:
    L = shape.L
    dev = g_cur.device
    n_cand = L if cand is None else int(cand.numel())
    n = min(k, n_cand)
    scores = torch.empty(n_cand, dtype=torch.float32, device=dev)
    active = torch.empty(max(n, 1), dtype=torch.int32, device=dev)
    slot = torch.empty(L, dtype=torch.int32, device=dev)
    B.fl_select_tokens(ctx, shape, loop_r, g_prev, g_cur, cand, n_cand, k, scores, active, slot)
    return TokenSelection(active if n > 0 else active[:0], slot, scores, n)


def _device(dev) -> torch.device:
    """`dev` with its index ("cuda" is the device that is current now): what the process's pools are keyed by."""
    if not isinstance(dev, torch.device):
        dev = torch.device(dev)
    return dev if dev.index is not None or dev.type != "cuda" else torch.device("cuda", torch.cuda.current_device())


_ROWS_WS: dict = {}


def rows_workspace(dev, n: int, d: int):
    """Transient bf16 buffers [n, d] for the materialized rows of one loop: ((K before, K after), (V before,
    V after)).  One set per device, grown on demand and reused by every layer and loop: a loop's rows are dead once
    its attention call has been issued on the stream."""
    dev = _device(dev)
    key = (dev, d)
    ws = _ROWS_WS.get(key)
    if ws is None or ws[0][0].shape[0] < n:
        ws = tuple(tuple(torch.empty(n, d, dtype=torch.bfloat16, device=dev) for _ in range(2)) for _ in range(2))
        _ROWS_WS[key] = ws
    return ws


_STATUS: dict = {}     # (device, stream) -> (zeroed words, counter of the words handed out)


def status_word(dev):
    """A zeroed int32 device word of its own: one of a block of 1024 that is cleared once, on the stream that will use it
    (a fill kernel per word costs more host time than the call whose errors it collects). A block lives as long as
    any word of it; words are not handed out again. Under graph capture a clear is recorded and not executed: there a word
    is an allocation of its own, which every replay clears."""
    dev = _device(dev)
    if torch.cuda.is_current_stream_capturing():
        return torch.zeros(1, dtype=torch.int32, device=dev)
    key = (dev, B._stream_of(dev.index))
    while True:
        block = _STATUS.get(key)
        i = next(block[1]) if block is not None else 1024
        if i < 1024:
            return block[0][i:i + 1]
        _STATUS[key] = (torch.zeros(1024, dtype=torch.int32, device=dev), itertools.count())


def lend_workspace(ctx, shape, dev, stale_rows: bool = True) -> int:
    """Hands the context the workspace with which the attention launch splits the problems of its last, partly empty
    wave over two CTAs each (a scheduling aid; 0 bytes when the shape cannot profit), with room behind it for the rows
    that a launch with shrunken token sets rebuilds once (up to 256 MB; stale_rows=False: without, for a program whose
    sets keep their size).  The tensor stays referenced by the Context object.  Returns the bytes of the split's part."""
    sizes = ctx.__dict__.setdefault("_workspace_sizes", {})      # two calls into the library per layer state otherwise
    key = (shape.L, shape.n_heads, shape.head_dim, shape.dtype, shape.q_block)
    if key not in sizes:
        sizes[key] = (B.fl_loop_attention_workspace_bytes(ctx, shape), B.fl_loop_attention_full_workspace_bytes(ctx, shape))
    need, full = sizes[key]
    want = full if stale_rows else need
    if want > 0:
        ws = getattr(ctx, "_workspace", None)
        if ws is None or ws.numel() < want:
            if stale_rows and not getattr(ctx, "_row_room", False):
                ctx._workspace_before = ws      # the split's part alone (< 20 MB): a captured graph may still use it
            ws = torch.empty(want, dtype=torch.uint8, device=dev)
        # a context that holds this workspace already keeps it: every launch leaves its counters cleared
        if getattr(ctx, "_lent", None) != (ws.data_ptr(), ws.numel()):
            B.fl_set_workspace(ctx, ws, ws.numel())
            if torch.cuda.is_current_stream_capturing():
                ctx._lent = None     # the counters' clear is recorded and not executed: the next state sets it again
        ctx._workspace = ws
        ctx._row_room = stale_rows or getattr(ctx, "_row_room", False)
    return need


class LayerState:
    """Buffers of one layer and the calls that advance it by one loop."""

    def __init__(self, ctx, w: Workload, device="cuda:0", bits: Optional[int] = None, q_block: Optional[int] = None,
                 c: Optional[int] = None, split: bool = True):
        self.ctx, self.w, self.dev = ctx, w, torch.device(device)
        self.shape = shape_of(w, bits, q_block)
        self.bits = self.shape.bits
        self.c = c or w.col_budget
        self.nb = (w.L + self.shape.q_block - 1) // self.shape.q_block
        self.dt = torch_dtype(w)
        self._max_rows = 0              # of the streams so far
        self._lends = split and self.dt == torch.bfloat16
        if self.dt == torch.bfloat16:
            if split:                   # the room for rebuilt rows follows with the first set that shrinks
                lend_workspace(ctx, self.shape, self.dev, stale_rows=False)
            else:   # the context's attention launches go back to one CTA per problem
                B.fl_set_workspace(ctx, None, 0)
                ctx._workspace = None
        self.k_streams: List[dict] = []
        self.v_streams: List[dict] = []
        self.col_idx = None
        self.col_cnt = None
        self.col_scores = None
        self.lse = None
        self.store = None
        self.status = status_word(self.dev)   # asynchronous device-side errors

    # ---- loop 1 -------------------------------------------------------------------------------
    def dense_loop(self, q, k, v, want_col_scores=True):
        w = self.w
        self.k_base, self.v_base = k, v
        self.q_store = q.clone()
        self.o_store = torch.empty_like(q)
        self.lse = torch.empty(w.n_heads, w.L, dtype=torch.float32, device=self.dev)
        if want_col_scores:
            self.col_scores = torch.empty(w.n_heads, self.nb, w.L, dtype=torch.float32, device=self.dev)
        B.fl_dense_loop_attention(self.ctx, self.shape, q, k, v, self.o_store, self.lse, self.col_scores)
        self._rebuild_store()

    def select_columns_dense(self, c: Optional[int] = None, col_scores=None):
        w = self.w
        c = c or self.c
        self.c = c
        self.col_idx = torch.empty(w.n_heads, self.nb, c, dtype=torch.int32, device=self.dev)
        self.col_cnt = torch.empty(w.n_heads, self.nb, dtype=torch.int32, device=self.dev)
        B.fl_select_columns(self.ctx, self.shape, self.col_scores if col_scores is None else col_scores, None, None,
                            w.L, c, self.col_idx, self.col_cnt)

    def prune_columns(self, col_scores_next, c_next: int):
        """Sparse source loop: keep the c_next best of the current set (Eq. 6, nested selection)."""
        w = self.w
        new_idx = torch.empty(w.n_heads, self.nb, c_next, dtype=torch.int32, device=self.dev)
        new_cnt = torch.empty(w.n_heads, self.nb, dtype=torch.int32, device=self.dev)
        B.fl_select_columns(self.ctx, self.shape, col_scores_next, self.col_idx, self.col_cnt, self.c, c_next,
                            new_idx, new_cnt)
        self.col_idx, self.col_cnt, self.c = new_idx, new_cnt, c_next

    # ---- packed loop-1 base (Appendix E) ------------------------------------------------------
    def pack_base(self, k, v, group: int = 64, tail: int = 64):
        """Packs the loop-1 K and V of the layer (keys per channel over `group` positions, values per token over
        `group` channels, the last `tail` positions unquantized) and keeps only the packed form; returns its bytes."""
        w, L, d = self.w, self.w.L, self.w.d
        Lq = max(0, L - tail)
        n_tg = (Lq + group - 1) // group
        u8 = lambda *s_: torch.empty(s_, dtype=torch.uint8, device=self.dev)
        f16 = lambda *s_: torch.empty(s_, dtype=torch.float16, device=self.dev)
        self.base_tensors = [u8(max(Lq, 1), d * self.bits // 8), f16(max(n_tg, 1), d), f16(max(n_tg, 1), d),
                             u8(max(Lq, 1), d * self.bits // 8), f16(max(Lq, 1), d // group), f16(max(Lq, 1), d // group),
                             torch.empty(max(L - Lq, 1), d, dtype=self.dt, device=self.dev),
                             torch.empty(max(L - Lq, 1), d, dtype=self.dt, device=self.dev)]
        self.base_q = B.make_base_q(*self.base_tensors, group, tail)
        B.fl_quant_kv_base(self.ctx, self.shape, k, v, self.base_q)
        return B.fl_kv_base_q_bytes(self.shape, group, tail)

    def rebuild_base(self, k_out, v_out, sel: Optional["TokenSelection"] = None):
        """Rebuilds the packed base into k_out, v_out ([L, H, dh], e.g. a buffer shared by all layers) and makes them
        the layer's base.  With a token selection (and the layer's column lists) only the rows the sparse loops read."""
        mask = None
        if sel is not None and self.col_idx is not None:
            words = (self.w.L + 31) // 32
            if getattr(self, "row_mask", None) is None:
                self.row_mask = torch.empty(self.w.n_heads, words, dtype=torch.int32, device=self.dev)
            B.fl_mark_base_rows(self.ctx, self.shape, self.col_idx, self.col_cnt, self.c, sel.active_idx, sel.n,
                                self.row_mask)
            mask = self.row_mask
        B.fl_dequant_kv_base(self.ctx, self.shape, self.base_q, k_out, v_out, row_mask=mask)
        self.k_base, self.v_base = k_out, v_out
        self._rebuild_store()

    # ---- loop r >= 2 --------------------------------------------------------------------------
    def _rebuild_store(self):
        self.store = B.make_store(self.k_base, self.v_base, self.k_streams, self.v_streams)

    def alloc_stream(self, sel: TokenSelection, rows: bool = True):
        """Adds the residual stream of the next loop.  rows: also lend it the transient workspace for the loop's
        materialized rows (bf16 storage only), which the quantization kernel fills and the attention kernel of the
        same loop gathers from; the workspace is shared by every LayerState of the device.  rows="cur": only the
        rows after the loop's residual (all a call that reuses the carried old term reads)."""
        w, n = self.w, sel.n
        d = w.d
        # a set that shrinks leaves tokens whose rows an attention call rebuilds: room for them (256 MB at 32K, so not before;
        # not under capture, where the memory would be the graph's: the kernels then rebuild them on the fly)
        if n < self._max_rows and self._lends and not torch.cuda.is_current_stream_capturing():
            if getattr(self.ctx, "_workspace", self) is not None:      # None: detached by a state without the split
                lend_workspace(self.ctx, self.shape, self.dev)
            self._lends = False
        self._max_rows = max(self._max_rows, n)
        ws = rows_workspace(self.dev, n, d) if rows and self.dt == torch.bfloat16 and n > 0 else None

        # K and V in one allocation each for the codes and for scales and offsets (an allocation costs the host about as
        # much as a view of all of them), where the pieces keep the 16-byte alignment of allocations of their own
        m, codes, meta = max(n, 1), None, None
        if self.bits != 16 and (m * d * self.bits // 8) % 16 == 0 and (m * (d // w.group) * 2) % 16 == 0:
            codes = torch.empty(2, m, d * self.bits // 8, dtype=torch.uint8, device=self.dev).unbind(0)
            meta = torch.empty(4, m, d // w.group, dtype=torch.float16, device=self.dev).unbind(0)

        def one(side):
            st = {"slot_of_pos": sel.slot_of_pos, "n_rows": n}
            if ws is not None:
                prev, cur = ws[side]
                whole = cur.shape[0] == n
                st["rows_cur"] = cur if whole else cur[:n]
                if rows != "cur":    # rows="cur": a loop that reuses the carried old term reads nothing else
                    st["rows_prev"] = prev if whole else prev[:n]
            if codes is not None:
                st["codes"], st["scale"], st["zero"] = codes[side], meta[2 * side], meta[2 * side + 1]
            elif self.bits == 16:
                st.update(codes=torch.empty(max(n, 1), d, dtype=self.dt, device=self.dev), scale=None, zero=None)
            else:
                st.update(codes=torch.empty(max(n, 1), d * self.bits // 8, dtype=torch.uint8, device=self.dev),
                          scale=torch.empty(max(n, 1), d // w.group, dtype=torch.float16, device=self.dev),
                          zero=torch.empty(max(n, 1), d // w.group, dtype=torch.float16, device=self.dev))
            return st
        # every stream of the device points at the same workspace: its content belongs to whichever loop was
        # quantized last, and only that loop's attention call reads it
        self.k_streams.append(one(0))
        self.v_streams.append(one(1))
        self.store = B.extend_store(self.store, self.k_streams[-1], self.v_streams[-1]) \
            if self.store is not None and self.store.n_streams + 1 == len(self.k_streams) else None
        if self.store is None:
            self._rebuild_store()

    def quantize(self, loop_r, k_new, v_new, sel: TokenSelection):
        B.fl_quant_kv_residual(self.ctx, self.shape, loop_r, k_new, v_new, sel.active_idx, sel.n, self.store)

    def gather(self, full, sel: TokenSelection, out=None):
        row_bytes = full.shape[1] * full.shape[2] * full.element_size() if full.dim() == 3 else \
            full.shape[1] * full.element_size()
        if out is None:
            out = torch.empty((max(sel.n, 1),) + tuple(full.shape[1:]), dtype=full.dtype, device=self.dev)
        B.fl_gather_rows(self.ctx, full, sel.active_idx, sel.n, row_bytes, out)
        return out

    def scatter(self, rows, sel: TokenSelection, full):
        row_bytes = full.shape[1] * full.shape[2] * full.element_size() if full.dim() == 3 else \
            full.shape[1] * full.element_size()
        B.fl_scatter_update(self.ctx, rows, sel.active_idx, sel.n, row_bytes, full)

    def attention(self, loop_r, q_new, q_old, o_prev, o_out, sel: TokenSelection, col_scores_next=None):
        B.fl_loop_attention(self.ctx, self.shape, loop_r, q_new, q_old, sel.active_idx, sel.n, self.store,
                            self.col_idx, self.col_cnt, self.c, self.lse, self.lse, o_prev, o_out,
                            col_scores_next, status=self.status)   # lse updated in place (active rows only)

    def carry_buffers(self):
        """Buffers of the old-term economy, allocated on first use: background rows [L, H, dh] and mass [H, L]."""
        if getattr(self, "bg_store", None) is None:
            # rows of positions that were never active are neither written nor read
            self.bg_store = torch.empty_like(self.o_store)
            self.mass = torch.empty(self.w.n_heads, self.w.L, dtype=torch.float32, device=self.dev)
        return self.bg_store, self.mass

    def attention_indexed(self, loop_r, q_new, sel: TokenSelection, col_scores_next=None, check=True,
                          carry: Optional[str] = None) -> int:
        """Same step on the position-indexed Q / O stores, updated in place (no gathers or scatters around it);
        returns the status code, FL_ERR_UNSUPPORTED when the shape is outside the tensor path.
        carry: None (plain call), "write" (recompute the old term and leave background rows and masses for later
        loops) or "reuse" (take the old term from them: valid while the column sets are unchanged and the token sets
        nested)."""
        if carry is None:
            return B.fl_loop_attention_indexed(self.ctx, self.shape, loop_r, q_new, self.q_store, self.q_store,
                                               sel.active_idx, sel.n, self.store, self.col_idx, self.col_cnt, self.c,
                                               self.lse, self.lse, self.o_store, self.o_store, col_scores_next,
                                               status=self.status, check=check)
        bg, mass = self.carry_buffers()
        cs = B.make_carry(bg, mass, carry == "reuse")
        return B.fl_loop_attention_indexed_carry(self.ctx, self.shape, loop_r, q_new, self.q_store, self.q_store,
                                                 sel.active_idx, sel.n, self.store, self.col_idx, self.col_cnt,
                                                 self.c, self.lse, self.lse, self.o_store, self.o_store, cs,
                                                 col_scores_next, status=self.status, check=check)

    def check_status(self):
        """Synchronises and raises if a kernel reported an asynchronous error (e.g. a bounded wait ran out)."""
        code = int(self.status.item())
        if code != 0:
            raise B.FlashLoopError("device status", code)

    def sparse_loop(self, loop_r, q_new, k_new, v_new, sel: TokenSelection, want_col_scores_next=False,
                    indexed=False, carry: Optional[str] = None, rows: bool = True):
        """One loop r >= 2 for this layer: store residuals, gather the carried rows, attend, scatter back
        (indexed=True: one call on the stores instead).  q_new, k_new, v_new: [n, H, dh] rows of the active tokens.
        Returns (o_rows, col_scores_next)."""
        self.alloc_stream(sel, rows=rows)
        self.quantize(loop_r, k_new, v_new, sel)
        if indexed:
            csn = None
            if want_col_scores_next:
                csn = torch.zeros(self.w.n_heads, self.nb, self.c, dtype=torch.float32, device=self.dev)
            self.attention_indexed(loop_r, q_new, sel, csn, carry=carry)
            return self.gather(self.o_store, sel), csn
        q_old = self.gather(self.q_store, sel)
        o_prev = self.gather(self.o_store, sel)
        o_out = torch.empty_like(o_prev)
        csn = None
        if want_col_scores_next:
            csn = torch.zeros(self.w.n_heads, self.nb, self.c, dtype=torch.float32, device=self.dev)
        self.attention(loop_r, q_new, q_old, o_prev, o_out, sel, csn)
        self.scatter(o_out, sel, self.o_store)
        self.scatter(q_new, sel, self.q_store)
        return o_out, csn


# The library takes addresses. What these objects hand it is looked at here: a tensor of another type, shape or place would be read, or
# written, past its end.
def _refuse(call: str, why: str):
    raise B.FlashLoopError(f"{call} ({why})", B.FL_ERR_INVALID_ARG)


def _row_stride(call: str, name: str, x, like, n: int = 0, heads: Optional[int] = None, dim: Optional[int] = None) -> int:
    """Elements from one row of x [n or more, heads, dim] to the next; its type is one of `like`'s (types, device). A row's heads stand side
    by side, the rows any distance apart that keeps them so."""
    types, device = like
    if x.dim() != 3 or x.shape[0] < n or x.shape[1] != (heads or x.shape[1]) or x.shape[2] != (dim or x.shape[2]):
        _refuse(call, f"{name} is {list(x.shape)}, not [{n}, {heads or 'heads'}, {dim or 'head_dim'}]")
    if x.dtype not in types or x.device != device:
        _refuse(call, f"{name} is {x.dtype} on {x.device}, not {' or '.join(map(str, types))} on {device}")
    row = x.shape[1] * x.shape[2]
    if x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != x.shape[2]):
        _refuse(call, f"the heads of a row of {name} do not follow one another")
    if x.shape[0] <= 1:
        return row
    if x.stride(0) < row:
        _refuse(call, f"the rows of {name} overlap")
    return x.stride(0)


def _indices(call: str, name: str, x, n: int, device):
    if x is not None and (x.dim() != 1 or x.numel() < n or x.dtype != torch.int32 or x.device != device or not x.is_contiguous()):
        _refuse(call, f"{name} is {x.dtype} {list(x.shape)} on {x.device}, not {n} contiguous int32 on {device}")


_STORAGE = {torch.bfloat16: B.FL_BF16, torch.float32: B.FL_F32}


class RotaryTable:
    """Cosines and sines of positions 0 .. n_pos - 1, and the two descriptors that a rotation needs."""

    def __init__(self, ctx, n_pos: int, rot_dim: int, layout=B.FL_ROPE_HALF, kind=B.FL_ROPE_PLAIN, device="cuda:0", **spec):
        self.ctx, self.n_pos = ctx, n_pos
        self.table = torch.empty(n_pos, rot_dim // 2, 2, dtype=torch.float32, device=_device(device))
        self.status = status_word(self.table.device)
        B.fl_rope_table(ctx, B.make_rope_spec(kind, rot_dim, **spec), self.table, n_pos)
        self.rope = B.make_rope(self.table, n_pos, rot_dim, layout)

    def rotate(self, x, pos, inverse: bool = False, out=None, pos0: int = 0):
        """x: [n, heads, head_dim], rows any distance apart (a part of a stacked projection); pos: int32 [n], or None for pos0, pos0 + 1, ...
        Positions that the table does not hold are reported by check_status()."""
        like = (tuple(_STORAGE), self.table.device)
        stride = _row_stride("RotaryTable.rotate", "x", x, like)
        n, heads, dim = x.shape
        _indices("RotaryTable.rotate", "pos", pos, n, self.table.device)
        if out is None:
            out = torch.empty(n, heads, dim, dtype=x.dtype, device=x.device)
        out_stride = _row_stride("RotaryTable.rotate", "out", out, ((x.dtype,), x.device), n, heads, dim)
        B.fl_rotate_rows(self.ctx, x, stride, pos, n, heads, dim, _STORAGE[x.dtype], self.rope, inverse, out, out_stride, pos0=pos0,
                         status=self.status)
        return out

    def check_status(self):
        """Synchronises and raises if a position was outside the table."""
        code = int(self.status.item())
        if code != 0:
            raise B.FlashLoopError("device status", code)


class PagedCache:
    """A paged 8-bit K/V cache of one layer and the calls on it: pages are handed out on the host as sequences grow, everything else stays
    on the device.  `code`: B.FL_INT8 or B.FL_E4M3.  On more than one stream calls are ordered by the program, as with any tensors: append
    and release write what attend and read look at.  Those two may run beside one another; each stream has a workspace of its own.
    In a captured graph they go by the lengths that were there at the capture, until the next append lets go of them."""

    def __init__(self, ctx, n_seqs: int, n_kv_heads: int, head_dim: int, max_tokens: int, n_pages: Optional[int] = None, page: int = 64,
                 dtype=torch.bfloat16, code=B.FL_INT8, device="cuda:0"):
        if dtype not in _STORAGE or code not in (B.FL_INT8, B.FL_E4M3):
            _refuse("PagedCache", f"storage {dtype}, code {code}")
        self.ctx, self.dev = ctx, _device(device)
        self.n_seqs, self.page, self.dtype, self.n_kv_heads, self.head_dim = n_seqs, page, dtype, n_kv_heads, head_dim
        self.max_pages = max(1, -(-max_tokens // page))
        n_pages = n_seqs * self.max_pages if n_pages is None else n_pages
        ct = torch.int8 if code == B.FL_INT8 else torch.float8_e4m3fn
        pool = lambda: torch.zeros(n_pages, n_kv_heads, page, head_dim, dtype=ct, device=self.dev)
        self.k_codes, self.v_codes = pool(), pool()
        self.k_scale, self.v_scale = (torch.zeros(n_pages, n_kv_heads, device=self.dev) for _ in range(2))
        self.k_open, self.v_open = (torch.zeros(n_seqs, n_kv_heads, page, head_dim, dtype=dtype, device=self.dev) for _ in range(2))
        self.page_table = torch.zeros(n_seqs, self.max_pages, dtype=torch.int32, device=self.dev)
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages = [[] for _ in range(n_seqs)]
        self.lens = [0] * n_seqs                                   # on the host, as the program knows them
        self.len_dev = torch.zeros(n_seqs, dtype=torch.int32, device=self.dev)
        self.status = status_word(self.dev)
        self.handle = B.make_paged_kv(self.k_codes, self.v_codes, self.k_scale, self.v_scale, self.k_open, self.v_open, self.page_table,
                                      page=page, dtype=_STORAGE[dtype], code=code)
        self._workspaces = {}                                      # by stream: calls that may overlap must not share one
        self._len_stream = self._stream()                          # where len_dev was allocated

    def _stream(self):
        return B._stream_of(self.dev.index)

    def _lens_read_here(self):
        """The next append drops len_dev: on another stream than its own the allocator has to hear of this use."""
        if self._stream() != self._len_stream:
            self.len_dev.record_stream(torch.cuda.current_stream(self.dev))

    def _workspace(self, need: int):
        """Cleared once, on the stream that uses it; a call leaves it cleared.  Under graph capture a clear is recorded and not executed:
        there a workspace is an allocation of its own, which every replay clears."""
        if torch.cuda.is_current_stream_capturing():
            return torch.zeros(need, dtype=torch.uint8, device=self.dev)
        ws = self._workspaces.get(self._stream())
        if ws is None or ws.numel() < need:
            ws = self._workspaces[self._stream()] = torch.zeros(need, dtype=torch.uint8, device=self.dev)
        return ws

    def _ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device=self.dev)

    def _counts(self, call: str, new: List[int]) -> int:
        if len(new) != self.n_seqs or any(n < 0 for n in new):
            _refuse(call, f"new is {list(new)}, not a number of tokens for each of {self.n_seqs} sequences")
        return sum(new)

    def reserve(self, new: List[int]):
        """Pages for the blocks that `new` more tokens per sequence complete: all of them, or RuntimeError and none."""
        self._counts("PagedCache.reserve", new)
        free = len(self.free)
        for b, n in enumerate(new):
            blocks = (self.lens[b] + n) // self.page
            free -= max(0, blocks - len(self.pages[b]))
            if free < 0 or blocks > self.max_pages:
                raise RuntimeError(f"no page for sequence {b}")
        for b, n in enumerate(new):
            while len(self.pages[b]) < (self.lens[b] + n) // self.page:
                p = self.free.pop()
                self.page_table[b, len(self.pages[b])] = p
                self.pages[b].append(p)

    def release(self, b: int):
        """Forgets a sequence and gives its pages back."""
        self.free.extend(reversed(self.pages[b]))
        self.pages[b], self.lens[b] = [], 0
        self.len_dev[b] = 0

    def append(self, k, v, new: List[int], rotary: Optional[RotaryTable] = None, pos=None):
        """k, v: [sum(new), n_kv_heads, head_dim], new[b] rows for sequence b; keys are rotated on the way where `rotary` is given."""
        call, like = "PagedCache.append", ((self.dtype,), self.dev)
        n = self._counts(call, new)
        strides = [_row_stride(call, name, x, like, n, self.n_kv_heads, self.head_dim) for name, x in (("k", k), ("v", v))]
        _indices(call, "pos", pos, n, self.dev)
        if rotary is not None and rotary.table.device != self.dev:
            _refuse(call, f"the rotation's table is on {rotary.table.device}, not on {self.dev}")
        self.reserve(new)
        starts = self._ints(list(itertools.accumulate(new, initial=0)))
        after = torch.empty_like(self.len_dev)
        B.fl_cache_append(self.ctx, self.handle, rotary.rope if rotary is not None else None, k, strides[0], v, strides[1], starts, n,
                          self.len_dev, after, pos=pos, status=self.status)
        self._lens_read_here()
        self.len_dev, self._len_stream = after, self._stream()
        self.lens = [a + n for a, n in zip(self.lens, new)]
        return starts

    def attend(self, q, new: List[int], sm_scale: float, starts=None):
        """Attention of the last new[b] tokens of each sequence (their rows are in the cache): outputs [n, heads, head_dim] and
        log-normalisers [n, heads], which are what fl_decode_attention takes as o_prev and lse_prev.  Sequence b has rows starts[b] ..
        starts[b + 1] - 1 of q (int32 on the device, as append returns them; None: one sequence after the other)."""
        call, total = "PagedCache.attend", self._counts("PagedCache.attend", new)
        stride = _row_stride(call, "q", q, ((self.dtype,), self.dev), total, None, self.head_dim)
        n, heads, dim = q.shape
        if starts is None:
            if n != total:
                _refuse(call, f"q has {n} rows, not {total}")
            starts = self._ints(list(itertools.accumulate(new, initial=0)))
        _indices(call, "starts", starts, self.n_seqs + 1, self.dev)
        max_q = max(max(new), 1)
        need = B.fl_cache_attention_workspace_bytes(self.ctx, self.handle, heads, n, max_q)
        ws = self._workspace(need)
        o = torch.empty(n, heads, dim, dtype=self.dtype, device=self.dev)
        lse = torch.empty(n, heads, dtype=torch.float32, device=self.dev)
        B.fl_cache_attention(self.ctx, self.handle, q, stride, heads, starts, n, max_q, self.len_dev, sm_scale, o, lse, ws, ws.numel(),
                             status=self.status)
        self._lens_read_here()
        return o, lse

    def read(self, b: int, first: int = 0, n: Optional[int] = None):
        """Rows first .. first + n - 1 of a sequence as the cache holds them, in the storage type: a base for the sparse loops."""
        if not 0 <= b < self.n_seqs or first < 0 or (n is not None and n < 0) or (n is None and first > self.lens[b]):
            _refuse("PagedCache.read", f"rows {first} on, {n} of them, of sequence {b}")
        n = self.lens[b] - first if n is None else n
        k = torch.empty(n, *self.k_open.shape[1:2], self.k_open.shape[3], dtype=self.dtype, device=self.dev)
        v = torch.empty_like(k)
        starts = self._ints([0] * (b + 1) + [n] * (self.n_seqs - b))
        firsts = self._ints([first if i == b else 0 for i in range(self.n_seqs)])
        B.fl_cache_read(self.ctx, self.handle, starts, firsts, n, self.len_dev, k, v, status=self.status)
        self._lens_read_here()
        return k, v

    def check_status(self):
        """Synchronises and raises if a kernel reported an asynchronous error."""
        code = int(self.status.item())
        if code != 0:
            raise B.FlashLoopError("device status", code)
