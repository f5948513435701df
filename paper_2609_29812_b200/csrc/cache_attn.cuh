// What the kernels of the attention over the paged 8-bit cache share: their arguments, how the work is cut, how partial results meet.
#pragma once
#include "cache.cuh"
#include "tc_attn_common.cuh"

namespace fl_ca {

// Which kernel takes a sequence (each looks for itself; lengths stand on the device): the one for few rows up to 16 rows (new tokens x
// group), and up to 128 where all there is to do is little, for it starts sooner; over long caches the other one multiplies faster.
// One sequence, 16 kv heads, few / many, us:
//   tokens            512        1024        2048        4096        8192       16384
//    32 rows      26 / 32     27 / 32     28 / 37     32 / 41     39 / 54     52 / 76
//    64 rows      27 / 32     28 / 33     31 / 37     38 / 41     50 / 55     78 / 77
//   128 rows      28 / 33     33 / 33     39 / 37     52 / 41     78 / 52    128 / 73
// The border lies at 64 rows x 4096 tokens, 128 x 2048: where 128 rows cross; fewer rows would cross later, for the tiles of 16 that read the
// same codes again are what costs the first kernel. All sequences count, those without new tokens too: the number of them is all that
// the host knows.
constexpr int kFewRows = 16;
constexpr int64_t kLittle = 1 << 22;   // rows x tokens x kv heads x sequences
enum { kEvery = 0, kFew = 1, kMany = 2 };

struct alignas(64) AttnArgs {
  CUtensorMap map[2];        // K and V codes as rows of head_dim bytes, 16 to a box (not with binary32 storage)
  CacheArgs c;
  const void* q;
  int64_t q_stride;
  const int32_t* seq_start;
  const int32_t* kv_len;
  void* o;
  float* lse;
  int32_t* counters;         // arrivals at split problems (few rows), zero between calls
  float* part;               // partial results: per CTA two slots of ROWS x (head_dim + 2)
  int32_t* status;
  int n_tokens, n_heads, group, max_q, page, page_shift;
  int which;                 // sequences that this kernel takes: kEvery, kFew, kMany
  int64_t little;            // rows x tokens of a sequence up to which more rows than kFewRows count as few
  int max_parts;             // most CTAs for a problem
  int min_units;             // fewest units worth a CTA of their own
  int head_units;            // units that a problem's first load and last store are worth: counted before its tokens
  float scale_log2;          // sm_scale log2 e
};

// A sequence's share of the work, in units of (problem, TOKENS consecutive tokens). A problem is a tile of ROWS rows (query token x
// query head, heads fastest) that share a kv head.
struct SeqWork {
  int s, n, len, tiles;
  int64_t head;              // units of a kv head's problems
  int64_t units;
  // units of tokens that tile t's last row sees (one at least: a row that sees nothing is written, too)
  template <int ROWS, int TOKENS>
  __device__ int blocks(const AttnArgs& a, int t) const {
    const int last = (int)min((int64_t)n * a.group, (int64_t)(t + 1) * ROWS) - 1;
    return max(1, (min(len, len - n + last / a.group + 1) + TOKENS - 1) / TOKENS);
  }
};
template <int ROWS, int TOKENS>
__device__ __forceinline__ SeqWork seq_work(const AttnArgs& a, int b) {
  SeqWork w;
  w.s = __ldg(a.seq_start + b);
  const int e = min(__ldg(a.seq_start + b + 1), a.n_tokens);
  w.len = __ldg(a.kv_len + b);
  w.n = w.s >= 0 ? max(0, e - w.s) : 0;
  if (w.n > a.max_q || w.len < 0 || (w.len >> a.page_shift) > a.c.max_pages) {
    cache_report(a.status);
    w.n = 0;
  }
  const int64_t rows = (int64_t)w.n * a.group;
  if (a.which != kEvery) {
    const bool few = rows <= kFewRows || (rows <= 128 && rows * w.len <= a.little);
    if (few != (a.which == kFew)) w.n = 0;
  }
  w.tiles = (int)((w.n == 0 ? 0 : rows + ROWS - 1) / ROWS);
  w.head = (int64_t)w.tiles * a.head_units;
  for (int t = 0; t < w.tiles; ++t) w.head += w.blocks<ROWS, TOKENS>(a, t);
  w.units = w.head * a.c.n_kv;
  return w;
}

// The CTAs take equal consecutive ranges of the units of all sequences, whatever their lengths: CTA c has units
// [start(c), start(c + 1)). A problem that a border cuts leaves partial results.
struct Range {
  int64_t total, u0, u1;
  int n_ctas;
  int b;                     // sequence of unit u0
  int64_t off;               // units of that sequence before u0
};
__device__ __forceinline__ int64_t range_start(int64_t total, int n, int c) { return total * c / n; }
__device__ __forceinline__ int range_owner(int64_t total, int n, int64_t u) { return (int)(((u + 1) * n - 1) / total); }

// By one warp, all its lanes.
template <int ROWS, int TOKENS>
__device__ __forceinline__ Range find_range(const AttnArgs& a, int lane) {
  Range r;
  int64_t sum = 0, mine = 0, problems = 0;
  for (int b0 = 0; b0 < a.c.n_seqs; b0 += 32) {
    mine = 0;
    if (b0 + lane < a.c.n_seqs) {
      const SeqWork w = seq_work<ROWS, TOKENS>(a, b0 + lane);
      mine = w.units;
      problems += (int64_t)w.tiles * a.c.n_kv;
    }
    sum += mine;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    problems += __shfl_xor_sync(0xffffffffu, problems, o);
  }
  r.total = sum;
  // As many CTAs as the tokens' units are worth, and one for each problem; where there are more CTAs than problems, the same number for
  // each if that leaves few idle, so that problems of one length are cut alike and none begins inside a CTA's range.
  const int64_t want = max(problems, min(problems * a.max_parts, (sum - problems * a.head_units) / a.min_units));
  r.n_ctas = (int)(want < gridDim.x ? want : gridDim.x);
  if (problems > 0 && problems < r.n_ctas) {
    const int rest = r.n_ctas % (int)problems;
    if (16 * rest <= r.n_ctas) r.n_ctas -= rest;
  }
  r.u0 = r.u1 = r.off = 0;
  r.b = 0;
  if ((int)blockIdx.x >= r.n_ctas) return r;
  r.u0 = range_start(sum, r.n_ctas, blockIdx.x);
  r.u1 = range_start(sum, r.n_ctas, blockIdx.x + 1);
  int64_t before = 0;
  for (int b0 = 0; b0 < a.c.n_seqs; b0 += 32) {
    if (a.c.n_seqs > 32) mine = b0 + lane < a.c.n_seqs ? seq_work<ROWS, TOKENS>(a, b0 + lane).units : 0;
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, before + upto > r.u0);
    if (past != 0) {
      const int l = __ffs(past) - 1;
      r.b = b0 + l;
      r.off = r.u0 - before - (__shfl_sync(0xffffffffu, upto, l) - __shfl_sync(0xffffffffu, mine, l));
      break;
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
  return r;
}

// One CTA's part of a problem: tokens [blk0, blk1) x TOKENS of it.
struct Segment {
  int b, kvh, tile, blk0, blk1;
  int s, n, len;
  int first, last;           // CTAs that have parts of the problem
  __device__ bool whole() const { return first == last; }
};

// Rows of a tile: row r is token i = (tile ROWS + r) / group of the sequence's new ones, head (tile ROWS + r) % group of the kv head's.
__device__ __forceinline__ int rows_of(const AttnArgs& a, const Segment& g, int rows) { return min(rows, g.n * a.group - g.tile * rows); }
__device__ __forceinline__ int limit_of(const AttnArgs& a, const Segment& g, int row) { return g.len - g.n + row / a.group + 1; }   // tokens seen
__device__ __forceinline__ int64_t out_row(const AttnArgs& a, const Segment& g, int row) {
  const int i = row / a.group;
  return (int64_t)(g.s + i) * a.n_heads + g.kvh * a.group + (row - i * a.group);
}

// Calls body(segment) for every part of a problem in the CTA's range, in order. The whole CTA calls it.
template <int ROWS, int TOKENS, typename F>
__device__ __forceinline__ void for_each_segment(const AttnArgs& a, const Range& r, F body) {
  int b = r.b;
  int64_t u = r.u0, off = r.off;
  while (u < r.u1) {
    const SeqWork w = seq_work<ROWS, TOKENS>(a, b);
    if (off < w.units) {
      int kvh = (int)(off / w.head), tile = 0;
      int64_t in = off - kvh * w.head;                 // units before u of the problem
      int span = a.head_units + w.blocks<ROWS, TOKENS>(a, 0);
      while (in >= span) {
        in -= span;
        span = a.head_units + w.blocks<ROWS, TOKENS>(a, ++tile);
      }
      while (u < r.u1 && kvh < a.c.n_kv) {
        Segment g;
        const int64_t left = r.u1 - u;
        const int from = (int)in, upto = left < span - from ? from + (int)left : span;
        const int64_t p0 = u - from + a.head_units;    // the problem's first unit of tokens
        u += upto - from;
        if (upto > a.head_units) {                     // (else none of the problem's tokens)
          g.b = b;
          g.kvh = kvh;
          g.tile = tile;
          g.blk0 = max(0, from - a.head_units);
          g.blk1 = upto - a.head_units;
          g.s = w.s;
          g.n = w.n;
          g.len = w.len;
          const bool cut = g.blk0 > 0 || upto < span;
          g.first = cut ? range_owner(r.total, r.n_ctas, p0) : blockIdx.x;
          g.last = cut ? range_owner(r.total, r.n_ctas, p0 + span - a.head_units - 1) : blockIdx.x;
          body(g);
        }
        in = 0;
        if (upto == span) {
          if (++tile == w.tiles) {
            tile = 0;
            ++kvh;
          }
          span = a.head_units + w.blocks<ROWS, TOKENS>(a, tile);
        }
      }
    }
    ++b;
    off = 0;
  }
}

// Slot of CTA c's partial result of a problem that begins in CTA `first`: a CTA has at most two cut problems, the one that comes in from
// the CTA before it and the one that goes on after it.
__device__ __forceinline__ int part_slot(int c, int first) { return 2 * c + (c == first ? 1 : 0); }

constexpr float kMove = 8.f;       // log2: how far a logit may pass the reference before the reference moves

// Weight of a part whose reference is m against the largest one.
__device__ __forceinline__ float part_weight(float m, float top) { return m == -INFINITY ? 0.f : tc::ex2(m - top); }

// Two codes (bytes SEL and SEL + 1 of a word) as a pair of f16, exactly.
//   int8: the byte plus 128 in the low bits of 1024 is the number 1152 + code (the magic-number conversion: an integer set into the
//   mantissa of a number whose unit is its last place).
//   e4m3: one conversion (as fast as a byte permutation).
template <int CODE, int SEL>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  uint32_t r;
  if (CODE == FL_INT8) {
    const uint32_t p = __byte_perm(w ^ 0x80808080u, 0x64646464u, SEL == 0 ? 0x4140 : 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(p), "r"(0x64806480u));
  } else {
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)(SEL == 0 ? w : w >> 16)));
  }
  return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two bf16 times a power of two, as f16.
__device__ __forceinline__ uint32_t scaled_f16(uint32_t w, float mul) {
  return pack_f16(__uint_as_float(w << 16) * mul, __uint_as_float(w & 0xffff0000u) * mul);
}
// Largest magnitude of two bf16 that are numbers, as bits, against m.
__device__ __forceinline__ uint32_t largest(uint32_t m, uint32_t w) {
  const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
  if (lo < 0x7f80u) m = max(m, lo);
  if (hi < 0x7f80u) m = max(m, hi);
  return m;
}
// The power of two that brings a bf16 of magnitude bits m (not below 2^-100) into [2^to, 2^(to+1)), and its inverse.
__device__ __forceinline__ void to_power(uint32_t m, int to, float* mul, float* inv) {
  const int e = max((int)(m >> 7) - 127, -100);
  *mul = __int_as_float((to - e + 127) << 23);
  *inv = __int_as_float((e - to + 127) << 23);
}

}  // namespace fl_ca

// Chunks of prompts (cache_attn_tc.cu): rows (new tokens x group) above fl_ca::kFewRows, bf16 storage.
int fl_launch_cache_attn_tc(fl_ctx* ctx, const fl_ca::AttnArgs& args, int head_dim, int code, cudaStream_t st);
int64_t fl_cache_attn_tc_part_bytes(const fl_ctx* ctx, int head_dim);
