// Appending to the paged 8-bit K/V cache, with the keys' rotation on the way, and rows read back from it.
#include "cache.cuh"
#include "rope.cuh"

namespace {

struct AppendArgs {
  CacheArgs c;
  RopeArgs rope;
  const void* x[2];            // k, v
  int64_t stride[2];
  const int32_t* seq_start;
  const int32_t* len_before;
  const int32_t* pos;
  int32_t* len_after;
  int n_tokens;
  int by_token;                // a unit is a token that is the first of its block, else a block counted from an upper bound
  int heads;                   // kv heads per CTA
  int32_t* status;
};

// The block a CTA is about: sequence b, its block `blk`; rows [lo, hi) of it are new, the first of them token t0 of the call.
struct Block {
  int b, blk, lo, hi, t0;
  int tail_blk, tail_rows, tail_lo, tail_t0;   // the block that stays open: its number, its rows, the first new one
};

// (rows [lo, hi) from token t0) of block `blk` of a sequence with `before` tokens held, n new ones from token s.
__device__ __forceinline__ void new_rows(int before, int n, int s, int blk, int page, int* lo, int* hi, int* t0) {
  const int at = blk * page;
  *lo = max(0, before - at);
  *hi = min(page, before + n - at);
  *t0 = s + at + *lo - before;
}

// Largest magnitude of a piece against m, as integers: an infinity and a NaN are the largest ones. bf16: two halves side by side.
__device__ __forceinline__ uint32_t top_of(const Piece<__nv_bfloat16>& x, uint32_t m) {
  return __vmaxu2(__vmaxu2(__vmaxu2(m, x.r[0].x & 0x7fff7fffu), __vmaxu2(x.r[0].y & 0x7fff7fffu, x.r[0].z & 0x7fff7fffu)), x.r[0].w & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t top_of(const Piece<float>& x, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    m = max(max(max(m, x.r[i].x & 0x7fffffffu), max(x.r[i].y & 0x7fffffffu, x.r[i].z & 0x7fffffffu)), x.r[i].w & 0x7fffffffu);
  return m;
}
template <typename T> __device__ __forceinline__ uint32_t top_bits(uint32_t m) { return sizeof(T) == 2 ? max(m << 16, m & 0xffff0000u) : m; }

// One (block, group of kv heads, side) per CTA; side 0 is K. A thread keeps two items of 16 elements of the block in
// registers, as they are stored: loaded while the head before is coded (rows already held from the open block, the new ones from
// the input, rotated with cosines and sines that serve all of the CTA's heads), their largest magnitude taken over the CTA, coded
// and written: one pass over the data. The block that stays open is written by the sequence's first CTA, after it has read the rows that
// the open block held, so no two CTAs touch an open block.
// 2 (4) bytes an element in and 1 out: 32768 tokens of 16 heads 86 us = 4.9 TB/s with the rotation, 76 without. Between HBM (54% of its
// nominal rate) and instructions (one leaves in 68% of the cycles; ALU 54%, conversions 37% of their rates). It lives on loads on their way: with
// numbers in place of the stored pieces and room for four items in every instance one CTA fitted an SM (164 registers). binary32: 177 us
// (floor 105), one CTA of eight warps an SM; 137 with pages of 128, whose CTAs have sixteen. Rotations that are no multiple of 16 elements, and rows
// off 16-byte boundaries, go element by element and head by head: 195 us, binary32 446.
template <typename T, int CODE, int MODE>
__device__ __forceinline__ void append_block(const AppendArgs& a, const Block& k, int side, int head0, int page, int head_dim, int page_id, int slot) {
  constexpr int ITEMS = 2;
  constexpr bool kTurns = MODE == kRopeHalf || MODE == kRopePairs;
  const int rot = side == 0 ? a.rope.rot_dim : 0;    // (values are not rotated)
  __shared__ uint32_t top_s[2][16];
  const int tid = threadIdx.x, shift = head_dim == 128 ? 3 : 2;
  const T* x = static_cast<const T*>(a.x[side]);
  const T* open = static_cast<const T*>(a.c.open[side]) + (int64_t)max(slot, 0) * a.c.n_kv * page * head_dim;
  auto table_row = [&](int t) -> const float* {
    int p = a.pos != nullptr ? __ldg(a.pos + t) : k.blk * page + k.lo + (t - k.t0);
    if ((unsigned)p >= (unsigned)a.rope.n_pos) {
      cache_report(a.status);
      p = 0;
    }
    return a.rope.table + (int64_t)p * rot;
  };
  // a thread's cosines and sines stand in places of its own in shared memory, read again for every head: in registers (32 of them) they
  // cost a CTA per SM
  extern __shared__ float4 turn_s[];
  bool turns[ITEMS];
#pragma unroll
  for (int m = 0; m < ITEMS; ++m) {
    const int id = m * blockDim.x + tid, r = id >> shift, j = id & ((1 << shift) - 1);
    turns[m] = kTurns && r >= k.lo && rope_item<MODE>(j, rot).turns;
    if (kTurns && turns[m]) {
      const float4* p = reinterpret_cast<const float4*>(table_row(k.t0 + r - k.lo) + 16 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) turn_s[(4 * m + i) * blockDim.x + tid] = __ldg(p + i);
    }
  }
  Piece<T> u[ITEMS], v[ITEMS];
  auto fetch = [&](int h) {
#pragma unroll
    for (int m = 0; m < ITEMS; ++m) {
      const int id = m * blockDim.x + tid, r = id >> shift;
      const RopeItem it = rope_item<MODE>(id & ((1 << shift) - 1), rot);
      if (r < k.lo) {                                // held open, as it is to be coded
        const T* p = open + ((int64_t)h * page + r) * head_dim;
        get_piece(u[m], p + it.a);
        get_piece(v[m], p + it.b);
      } else {
        const int t = k.t0 + r - k.lo;
        const T* p = x + (int64_t)t * a.stride[side] + (int64_t)h * head_dim;
        if (MODE == kRopeAny) {                      // any alignment: element by element (rot 0: nothing turns)
          const float* row = rot > 0 ? table_row(t) : nullptr;
          float f[8], g[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            f[i] = rope_any(p, it.a + i, row, rot, a.rope.layout);
            g[i] = rope_any(p, it.b + i, row, rot, a.rope.layout);
          }
          close_piece(u[m], f);
          close_piece(v[m], g);
        } else {
          get_piece(u[m], p + it.a);
          get_piece(v[m], p + it.b);
        }
      }
    }
  };
  const int head_end = min(a.c.n_kv, head0 + a.heads);
  fetch(head0);
  for (int h = head0; h < head_end; ++h) {
    uint32_t top = 0;
    Piece<T> y[ITEMS], z[ITEMS];
#pragma unroll
    for (int m = 0; m < ITEMS; ++m) {
      y[m] = u[m];
      z[m] = v[m];
      if (kTurns && turns[m]) {
        float f[8], g[8];
        open_piece(y[m], f);
        open_piece(z[m], g);
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 q = turn_s[(4 * m + i) * blockDim.x + tid];
          c[2 * i] = q.x;
          s[2 * i] = q.y;
          c[2 * i + 1] = q.z;
          s[2 * i + 1] = q.w;
        }
        rope_apply<MODE>(f, g, c, s);
        close_piece(y[m], f);
        close_piece(z[m], g);
      }
      top = top_of(z[m], top_of(y[m], top));
    }
    if (h + 1 < head_end) fetch(h + 1);
    top = __reduce_max_sync(0xffffffffu, top_bits<T>(top));
    uint32_t* ts = top_s[h & 1];                     // the head before last has been read by all that passed the last barrier
    if ((tid & 31) == 0) ts[tid >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w)
      if (w < (int)blockDim.x >> 5) top = max(top, ts[w]);
    const float amax = __uint_as_float(top), most = CODE == FL_INT8 ? 127.f : 448.f;
    const bool none = top < 0x0d800000u;             // 2^-100
    const bool bad = top >= 0x7f800000u;
    const float inv = none || bad ? 0.f : __fdiv_rn(most, amax);
    uint8_t* codes = a.c.codes[side] + ((int64_t)page_id * a.c.n_kv + h) * page * head_dim;
#pragma unroll
    for (int m = 0; m < ITEMS; ++m) {
      const int id = m * blockDim.x + tid, r = id >> shift;
      const RopeItem it = rope_item<MODE>(id & ((1 << shift) - 1), rot);
      auto put = [&](const Piece<T>& w, int at) {
        float f[8];
        open_piece(w, f);
        uint2 q = make_uint2(encode4<CODE>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), encode4<CODE>(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
        if (none || bad) q = make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(codes + r * head_dim + at) = q;
      };
      put(y[m], it.a);
      put(z[m], it.b);
    }
    if (tid == 0) a.c.scale[side][(int64_t)page_id * a.c.n_kv + h] = bad ? __int_as_float(0x7fc00000) : none ? 0.f : __fdiv_rn(amax, most);
  }
}

// New rows of the block that stays open, for the CTA's heads.
template <typename T, int MODE>
__device__ __forceinline__ void append_open(const AppendArgs& a, const Block& k, int side, int head0, int page, int head_dim, int slot) {
  const int rot = side == 0 ? a.rope.rot_dim : 0;
  const int shift = head_dim == 128 ? 3 : 2, rows = k.tail_rows - k.tail_lo;
  const int heads = min(a.c.n_kv - head0, a.heads);
  const T* x = static_cast<const T*>(a.x[side]);
  T* open = static_cast<T*>(a.c.open[side]) + (int64_t)slot * a.c.n_kv * page * head_dim;
  for (int id = threadIdx.x; id < (rows * heads) << shift; id += blockDim.x) {
    const int j = id & ((1 << shift) - 1), hr = id >> shift, r = hr / heads, h = head0 + hr - r * heads;
    const RopeItem it = rope_item<MODE>(j, rot);
    const int t = k.tail_t0 + r;
    const T* p = x + (int64_t)t * a.stride[side] + (int64_t)h * head_dim;
    T* o = open + ((int64_t)h * page + k.tail_lo + r) * head_dim;
    const float* row = nullptr;
    if (MODE != kRopeNone && rot > 0) {
      int ps = a.pos != nullptr ? __ldg(a.pos + t) : k.tail_blk * page + k.tail_lo + r;
      if ((unsigned)ps >= (unsigned)a.rope.n_pos) {
        cache_report(a.status);
        ps = 0;
      }
      row = a.rope.table + (int64_t)ps * rot;
    }
    if (MODE == kRopeAny) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e0 = it.a + i, e1 = it.b + i;
        if (e0 < rot) store1(o + e0, rope_any(p, e0, row, rot, a.rope.layout));
        else o[e0] = p[e0];
        if (e1 < rot) store1(o + e1, rope_any(p, e1, row, rot, a.rope.layout));
        else o[e1] = p[e1];
      }
    } else if (MODE != kRopeNone && it.turns) {
      float u[8], v[8], c[8], s[8];
      load8(p + it.a, u);
      load8(p + it.b, v);
      rope_load(row, j, 1.f, c, s);
      rope_apply<MODE>(u, v, c, s);
      store8(o + it.a, u);
      store8(o + it.b, v);
    } else {                                                  // as they come
      Piece<T> u, v;
      get_piece(u, p + it.a);
      get_piece(v, p + it.b);
      put_piece(o + it.a, u);
      put_piece(o + it.b, v);
    }
  }
}

template <typename T, int CODE, int KMODE, int VMODE, int THREADS>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 4 ? 1 : THREADS == 256 ? 3 : 2) cache_append_kernel(const __grid_constant__ AppendArgs a, int page, int head_dim) {
  fl_grid_wait();
  fl_grid_release();
  const int u = blockIdx.x, head0 = blockIdx.y * a.heads, side = blockIdx.z;
  if (a.len_after != nullptr && u == 0 && blockIdx.y == 0 && side == 0)
    for (int b = threadIdx.x; b < a.c.n_seqs; b += blockDim.x)
      a.len_after[b] = __ldg(a.len_before + b) + __ldg(a.seq_start + b + 1) - __ldg(a.seq_start + b);
  // the unit's sequence: units ascend with the tokens, two more per sequence than its whole blocks where they are counted by blocks
  const int shift = 31 - __clz(page);
  const int64_t target = u;
  auto first = [&](int b) -> int64_t {
    const int s = __ldg(a.seq_start + b);
    return a.by_token ? (int64_t)s : (int64_t)(s >> shift) + 2 * b;
  };
  const int b = cta_count_not_after(a.c.n_seqs, target, first) - 1;
  if (b < 0) return;
  const int s = __ldg(a.seq_start + b), e = min(__ldg(a.seq_start + b + 1), a.n_tokens), before = __ldg(a.len_before + b);
  if (s < 0 || before < 0) {
    if (threadIdx.x == 0) cache_report(a.status);
    return;
  }
  const int n = e - s;
  if (n <= 0) return;
  const int held = before & (page - 1), blk0 = before >> shift, last = (before + n - 1) >> shift;
  int blk;
  if (a.by_token) {
    const int i = u - s;
    if (i >= n || (i > 0 && ((before + i) & (page - 1)) != 0)) return;
    blk = (before + i) >> shift;
  } else {
    blk = blk0 + (int)(target - first(b));
    if (blk > last) return;
  }
  Block k;
  k.b = b;
  k.blk = blk;
  new_rows(before, n, s, blk, page, &k.lo, &k.hi, &k.t0);
  // who writes the open block: its own unit, unless the sequence's first unit has to read the rows that it held before
  k.tail_rows = (before + n) & (page - 1);
  k.tail_blk = last;
  const bool moved = held > 0 && last > blk0;                 // the open block's rows belong to an earlier block now
  const bool tail = k.tail_rows > 0 && (moved ? blk == blk0 : blk == last);
  const int slot = tail || k.lo > 0 ? cache_slot(a.c, b, a.status) : 0;
  const bool closes = k.hi == page;
  const int page_id = closes ? cache_page(a.c, b, blk, a.status) : -1;
  if (slot < 0) return;
  if (closes && page_id >= 0) {
    if (side == 0) append_block<T, CODE, KMODE>(a, k, side, head0, page, head_dim, page_id, slot);
    else append_block<T, CODE, VMODE>(a, k, side, head0, page, head_dim, page_id, slot);
  }
  if (tail) {
    int hi;
    new_rows(before, n, s, last, page, &k.tail_lo, &hi, &k.tail_t0);
    __syncthreads();                                          // the rows held open are in registers, and their codes out
    if (side == 0) append_open<T, KMODE>(a, k, side, head0, page, head_dim, slot);
    else append_open<T, VMODE>(a, k, side, head0, page, head_dim, slot);
  }
}

template <typename T, int CODE, int KMODE, int VMODE>
int launch_append(fl_ctx* ctx, AppendArgs& a, const fl_paged_kv* c, cudaStream_t st) {
  const int64_t by_block = (int64_t)a.n_tokens / c->page + 2 * (int64_t)c->n_seqs;
  a.by_token = a.n_tokens < by_block;
  const int64_t units = a.by_token ? (a.n_tokens > 0 ? a.n_tokens : 1) : by_block;   // (no tokens: len_after alone)
  // Eight heads per CTA share its cosines and sines (a 32768-token prompt of 16 heads: 94 us with four), four or one where fewer CTAs than
  // four per SM would be left.
  const int64_t enough = 2 * (int64_t)ctx->sm_count;
  a.heads = units * ((c->n_kv_heads + 7) / 8) >= enough ? 8 : units * ((c->n_kv_heads + 3) / 4) >= enough ? 4 : 1;
  const bool large = c->page * c->head_dim > 8192;
  const int threads = c->page * c->head_dim / 32;
  if (large) FL_FUNC_ATTR_ONCE(ctx, (cache_append_kernel<T, CODE, KMODE, VMODE, 512>), 512 * 128, false);
  FL_CHECK_CUDA(fl_launch(ctx, large ? cache_append_kernel<T, CODE, KMODE, VMODE, 512> : cache_append_kernel<T, CODE, KMODE, VMODE, 256>,
                          dim3((unsigned)units, (unsigned)((c->n_kv_heads + a.heads - 1) / a.heads), 2),
                          dim3(threads), KMODE == kRopeHalf || KMODE == kRopePairs ? threads * 128 : 0, st, a, (int)c->page, (int)c->head_dim));
  return fl_launch_status();
}

template <typename T, int CODE>
int append(fl_ctx* ctx, AppendArgs& a, const fl_paged_kv* c, int mode, bool vec, cudaStream_t st) {
  if (!vec) return launch_append<T, CODE, kRopeAny, kRopeAny>(ctx, a, c, st);
  if (mode == kRopeAny) return launch_append<T, CODE, kRopeAny, kRopeNone>(ctx, a, c, st);
  if (mode == kRopeHalf) return launch_append<T, CODE, kRopeHalf, kRopeNone>(ctx, a, c, st);
  if (mode == kRopePairs) return launch_append<T, CODE, kRopePairs, kRopeNone>(ctx, a, c, st);
  return launch_append<T, CODE, kRopeNone, kRopeNone>(ctx, a, c, st);
}

// ------------------------------------------------------------------------------------------------------------
// Rows read back. A CTA has 16 consecutive rows; a thread 16 elements of one (row, head): 8 threads (4 with heads of 64) per
// 128-byte row of codes, four consecutive tokens per warp, so that a warp reads 512 bytes of a page in one go and writes four
// whole rows of a head. Bound by HBM, 1 byte in, 2 (4) out: 32768 tokens of 16 heads 68 us = 5.9 TB/s (a warp waits 12 cycles of 23 for its loads).
// ------------------------------------------------------------------------------------------------------------
constexpr int kReadRows = 16;

struct ReadArgs {
  CacheArgs c;
  const int32_t* row_start;
  const int32_t* first;
  const int32_t* kv_len;
  void* out[2];
  int n_rows, heads;
  int32_t* status;
};

template <typename T, int CODE>
__global__ void __launch_bounds__(256) cache_read_kernel(const __grid_constant__ ReadArgs a, int page, int head_dim) {
  fl_grid_wait();
  fl_grid_release();
  __shared__ int page_s[kReadRows], at_s[kReadRows];          // page (or ~slot of an open block, INT_MIN: nothing there), row inside it
  const int r0 = blockIdx.x * kReadRows, side = blockIdx.z;
  const int b0 = cta_count_not_after(a.c.n_seqs, r0, [&](int b) -> int64_t { return __ldg(a.row_start + b); }) - 1;
  const int tid = threadIdx.x, page_shift = 31 - __clz(page);
  if (tid < kReadRows) {
    const int r = r0 + tid;
    int pg = INT_MIN, at = 0;
    if (r < a.n_rows && b0 >= 0) {
      int b = b0;
      while (b + 1 < a.c.n_seqs && __ldg(a.row_start + b + 1) <= r) ++b;
      const int64_t t = (int64_t)(a.first != nullptr ? __ldg(a.first + b) : 0) + r - __ldg(a.row_start + b);
      const int len = __ldg(a.kv_len + b);
      if (t < 0 || t >= len) {
        cache_report(a.status);
      } else {
        at = (int)t & (page - 1);
        if (t >= (len >> page_shift) << page_shift) {
          const int s = cache_slot(a.c, b, a.status);
          if (s >= 0) pg = ~s;
        } else {
          const int p = cache_page(a.c, b, (int)t >> page_shift, a.status);
          if (p >= 0) pg = p;
        }
      }
    }
    page_s[tid] = pg;
    at_s[tid] = at;
  }
  __syncthreads();
  if (a.out[side] == nullptr) return;
  const int shift = head_dim == 128 ? 3 : 2;
  const int h0 = blockIdx.y * a.heads, heads = min(a.heads, a.c.n_kv - h0), n = (kReadRows * heads) << shift;
  T* out = static_cast<T*>(a.out[side]);
  for (int id = tid; id < n; id += blockDim.x) {
    const int j = id & ((1 << shift) - 1), rr = (id >> shift) & (kReadRows - 1), h = h0 + (id >> (shift + 4)), r = r0 + rr;
    if (r >= a.n_rows) continue;
    const int pg = page_s[rr], at = at_s[rr];
    float x[2][8];
    if (pg >= 0) {
      const int64_t head = (int64_t)pg * a.c.n_kv + h;
      const uint4 w = __ldg(reinterpret_cast<const uint4*>(a.c.codes[side] + (head * page + at) * head_dim + 16 * j));
      const float sc = __ldg(a.c.scale[side] + head);
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[4];
        decode4<CODE>(ws[i], f);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i >> 1][(i & 1) * 4 + e] = f[e] * sc;
      }
    } else if (pg != INT_MIN) {
      const T* p = static_cast<const T*>(a.c.open[side]) + (((int64_t)~pg * a.c.n_kv + h) * page + at) * head_dim + 16 * j;
      load8(p, x[0]);
      load8(p + 8, x[1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[0][e] = x[1][e] = 0.f;
    }
    T* o = out + ((int64_t)r * a.c.n_kv + h) * head_dim + 16 * j;
    store8(o, x[0]);
    store8(o + 8, x[1]);
  }
}

template <typename T>
int read_rows(fl_ctx* ctx, const ReadArgs& a, const fl_paged_kv* c, cudaStream_t st) {
  const dim3 grid((unsigned)((a.n_rows + kReadRows - 1) / kReadRows), (unsigned)((c->n_kv_heads + a.heads - 1) / a.heads), 2);
  FL_CHECK_CUDA(fl_launch(ctx, c->code == FL_INT8 ? cache_read_kernel<T, FL_INT8> : cache_read_kernel<T, FL_E4M3>, grid, dim3(256), 0, st, a,
                          (int)c->page, (int)c->head_dim));
  return fl_launch_status();
}

}  // namespace

extern "C" int fl_cache_append(fl_ctx* ctx, const fl_paged_kv* cache, const fl_rope* rope, const void* k, int64_t k_stride, const void* v,
                               int64_t v_stride, const int32_t* seq_start, int32_t n_tokens, const int32_t* len_before, const int32_t* pos,
                               int32_t* len_after, int32_t* status, void* stream) {
  FL_REQUIRE(ctx != nullptr);
  int rc = fl_check_cache(cache);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(n_tokens >= 0 && seq_start != nullptr && len_before != nullptr && len_after != len_before);
  if (rope != nullptr) {
    rc = fl_check_rope(rope, cache->head_dim);
    if (rc != FL_OK) return rc;
  }
  const int64_t d = (int64_t)cache->n_kv_heads * cache->head_dim;
  FL_REQUIRE(k_stride >= d && v_stride >= d);
  if (n_tokens == 0 && len_after == nullptr) return FL_OK;
  const uintptr_t es = cache->dtype == FL_BF16 ? 2 : 4;
  if (n_tokens > 0) {
    FL_REQUIRE(k != nullptr && v != nullptr);
    FL_REQUIRE(reinterpret_cast<uintptr_t>(k) % es == 0 && reinterpret_cast<uintptr_t>(v) % es == 0);
  }
  AppendArgs a = {};
  a.c = fl_cache_args(cache);
  if (rope != nullptr) a.rope = {rope->table, rope->n_pos, rope->rot_dim, rope->layout};
  a.x[0] = k;
  a.x[1] = v;
  a.stride[0] = k_stride;
  a.stride[1] = v_stride;
  a.seq_start = seq_start;
  a.len_before = len_before;
  a.pos = pos;
  a.len_after = len_after;
  a.n_tokens = n_tokens;
  a.status = status;
  const int64_t piece = 16 / (int64_t)es;
  const bool vec = fl_aligned16(k) && fl_aligned16(v) && k_stride % piece == 0 && v_stride % piece == 0;
  const int mode = fl_rope_mode(rope);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cache->dtype == FL_BF16)
    return cache->code == FL_INT8 ? append<__nv_bfloat16, FL_INT8>(ctx, a, cache, mode, vec, st)
                                  : append<__nv_bfloat16, FL_E4M3>(ctx, a, cache, mode, vec, st);
  return cache->code == FL_INT8 ? append<float, FL_INT8>(ctx, a, cache, mode, vec, st) : append<float, FL_E4M3>(ctx, a, cache, mode, vec, st);
}

extern "C" int fl_cache_read(fl_ctx* ctx, const fl_paged_kv* cache, const int32_t* row_start, const int32_t* first, int32_t n_rows,
                             const int32_t* kv_len, void* k_rows, void* v_rows, int32_t* status, void* stream) {
  FL_REQUIRE(ctx != nullptr);
  const int rc = fl_check_cache(cache);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(n_rows >= 0);
  if (n_rows == 0) return FL_OK;
  FL_REQUIRE(row_start != nullptr && kv_len != nullptr && (k_rows != nullptr || v_rows != nullptr));
  FL_REQUIRE(fl_aligned16(k_rows) && fl_aligned16(v_rows));
  ReadArgs a = {};
  a.c = fl_cache_args(cache);
  a.row_start = row_start;
  a.first = first;
  a.kv_len = kv_len;
  a.out[0] = k_rows;
  a.out[1] = v_rows;
  a.n_rows = n_rows;
  a.heads = cache->n_kv_heads < 4 ? cache->n_kv_heads : 4;
  a.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cache->dtype == FL_BF16 ? read_rows<__nv_bfloat16>(ctx, a, cache, st) : read_rows<float>(ctx, a, cache, st);
}
