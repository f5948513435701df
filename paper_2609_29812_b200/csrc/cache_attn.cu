// Attention of a sequence's last tokens over its paged 8-bit cache: the kernels for few rows (decode steps).
//
// A problem is (sequence, kv head, tile of up to ROWS rows); its tokens are cut into units of 64 and the CTAs of one launch
// take equal runs of the units of all problems, so that one long sequence among short ones, or one sequence alone, fills the chip. The
// four warps of a CTA take a quarter of a run each, with a running reference and sum of their own per row, and meet in shared memory;
// a problem that a run's border cuts is put together by the CTA that comes last, in the order of the parts.
// Bound by HBM where the batch fills the chip, each code read once: 32 sequences of up to 16384 tokens x 16 heads 208 us = 6.1 TB/s
// call after call on the same cache, 240 us = 5.3 TB/s on one cache after another (with copies by the lanes in place of the ring of tiles
// 320, whatever their number on the way); an instruction leaves in 59% of the cycles then. By latency where it does not: one row over
// 8192 tokens 16 us (18.7 on changing caches; floor 5), of which the first pages, the join and the launch are 8. With 16 rows (254 registers, eight warps an
// SM) an instruction leaves in 27% of the cycles, and the warps wait for the next one to be fetched more than for anything else.
#include "cache_attn.cuh"

namespace {

using namespace fl_ca;
using fl_tc::kLn2;
using fl_tc::kLog2e;

constexpr int kUnit = 64;          // tokens of a unit
constexpr int kWarps = 4;
constexpr int kMostStages = 6;     // tiles of a warp's ring

// The pages of a warp's tiles, 32 at a time: lane i has page `base + i` of the sequence and its scales. A row is none if it sees a block
// without a scale, whatever its probabilities there: that goes by the logits, since a value's factor is lost where a probability is zero.
struct PageWindow {
  int base, id;
  float ks, vs;
  __device__ void fill(const AttnArgs& a, const Segment& g, int first, int end, int lane) {
    base = first;
    id = 0;
    ks = vs = 0.f;
    if (first + lane < end) {
      id = max(0, cache_page(a.c, g.b, first + lane, a.status));
      ks = __ldg(a.c.scale[0] + (int64_t)id * a.c.n_kv + g.kvh);
      vs = __ldg(a.c.scale[1] + (int64_t)id * a.c.n_kv + g.kvh);
      if (!(ks < INFINITY && vs < INFINITY)) ks = __int_as_float(0x7fc00000);   // either is none: so are the logits of the rows that see the block
    }
  }
};

__device__ __forceinline__ void movmatrix(uint32_t& x) {
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(x));
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ------------------------------------------------------------------------------------------------------------
// bf16 storage: products by warp MMAs (m16n8k16), the TOKENS as the accumulator's rows and the query rows as its columns,
//   S^T [16 tokens x 8 rows] = K Q^T,   O^T [dim x 8 rows] += V^T P^T,
// because a decode step has few rows: eight columns are the narrowest tile there is, and the 16-bit operand that the codes turn into
// is built in registers straight from 16-byte loads of the page. The order of the summed index is free: a lane's
// four dims (K) or tokens (V) of a step are those that its loads bring.
// The operands are f16: codes of either type fit it, two instructions a pair (bf16 takes four); the bf16 numbers that are no codes (Q, the open
// block's rows) are brought into its range by a power of two per row or tile, which keeps their eight bits down to 2^-30 of the
// largest; and a probability loses 2^-12 of itself where bf16 would take 2^-9. Probabilities go in as p 2^7 vs / vref, vref the largest
// scale of V so far: at most 2^15 (a logit passes the reference by 2^8 at most).
// ------------------------------------------------------------------------------------------------------------
template <int DH, int CODE, int NB>
struct MmaEngine {
  static constexpr int kRows = 8 * NB, kDim = DH;
  static constexpr int kHalves = DH / 64;          // 16-byte pieces of a K row per lane
  static constexpr int kVw = DH / 32;              // words of a V row per lane
  static constexpr int kCtas = NB * DH == 256 ? 2 : 3;   // per SM
  static constexpr int kTileBytes = 16 * DH, kStageBytes = 2 * kTileBytes;   // 16 tokens of K and V
  static constexpr int kStages = kCtas == 2 ? 6 : 4;   // what two or three CTAs' shared memory holds
  static constexpr int kWarpBytes = kStages * kStageBytes;
  static constexpr int kExtra = kWarps * kWarpBytes;
  static_assert(kWarpBytes >= kRows * DH * 4, "a warp's results take the place of its ring");
  using T = __nv_bfloat16;

  uint32_t qf[NB][DH / 8];                         // Q^T fragments: two words per step of 16 dims
  float o[DH / 16][NB][4];
  float l[NB][2];
  float sub[NB][2], over[NB][2];                   // the rows' references (0 where there is none yet), the logits that move them
  float unit[NB][2];                               // log2 of a logit per unit of the row's products
  float vref, vinv;                                // largest scale of V so far, 2^7 over it
  int lim[NB][2];
  struct Keys { uint32_t w[2][kHalves * 4]; };
  struct Values { uint32_t w[4][kVw]; };
  int lane, gq, q4;
  uint8_t* ring;
  uint64_t* bars;                                  // a barrier per stage
  volatile int* abort_flag;
  int put, get;                                    // stage of the next tile to ask for, of the next one to take
  uint32_t phase;                                  // of the latter

  __device__ void place(uint8_t* extra, uint64_t* bars_, int* abort_) {
    ring = extra + (threadIdx.x >> 5) * kWarpBytes;
    bars = bars_ + (threadIdx.x >> 5) * kMostStages;
    abort_flag = abort_;
    put = get = 0;
    phase = 0;
  }
  // Q rows are on their way when this returns; settle() makes the operand of them.
  __device__ void begin(const AttnArgs& a, const Segment& g, int rows) {
    lane = threadIdx.x & 31;
    gq = lane >> 2;
    q4 = lane & 3;
    vref = 0x1p-110f;                              // below any scale but zero
    vinv = 0x1p117f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = nb * 8 + gq, row = g.tile * kRows + r;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
        if (r < rows) {
          const int i = row / a.group;
          const uint4* p = reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (int64_t)(g.s + i) * a.q_stride +
                                                          (int64_t)(g.kvh * a.group + row - i * a.group) * DH + 16 * (kHalves * q4 + h));
          x = __ldg(p);
          y = __ldg(p + 1);
        }
        uint32_t* f = &qf[nb][h * 8];
        f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
        f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = nb * 8 + 2 * q4 + e;
        lim[nb][e] = c < rows ? limit_of(a, g, g.tile * kRows + c) : 0;
        l[nb][e] = sub[nb][e] = 0.f;
        over[nb][e] = -INFINITY;
      }
#pragma unroll
      for (int m = 0; m < DH / 16; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][nb][e] = 0.f;
    }
  }

  __device__ void settle(const AttnArgs& a) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) top = largest(top, qf[nb][i]);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      float mul, inv;
      to_power(top, 14, &mul, &inv);
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) qf[nb][i] = scaled_f16(qf[nb][i], mul);
#pragma unroll
      for (int e = 0; e < 2; ++e) unit[nb][e] = a.scale_log2 * __shfl_sync(0xffffffffu, inv, (2 * q4 + e) * 4);
    }
  }

  // Tiles come into the warp's own ring by TMA, swizzled, kStages of them; nobody else waits for them. (Copies by the lanes
  // themselves, 16 bytes each, took the same 320 us for the decode step of 32 sequences however the rest was arranged: they stand
  // in one queue with the reads of shared memory, the shuffles and the exponentials.)
  __device__ void take_k(Keys& kr, const uint8_t* stage) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const uint4 x = *reinterpret_cast<const uint4*>(stage + place_of(gq + 8 * r, kHalves * q4 + h));
        kr.w[r][4 * h] = x.x; kr.w[r][4 * h + 1] = x.y; kr.w[r][4 * h + 2] = x.z; kr.w[r][4 * h + 3] = x.w;
      }
  }
  __device__ void take_v(Values& vr, const uint8_t* stage) {
    stage += kTileBytes;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int row = 2 * q4 + (t & 1) + 8 * (t >> 1);
      if (DH == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(stage + place_of(row, gq));
        vr.w[t][0] = x.x; vr.w[t][1] = x.y; vr.w[t][2 % kVw] = x.z; vr.w[t][3 % kVw] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(stage + place_of(row, gq >> 1) + 8 * (gq & 1));
        vr.w[t][0] = x.x; vr.w[t][1] = x.y;
      }
    }
  }
  // byte of 16-byte piece c of row r of a tile, as the copy's swizzle lays it
  __device__ static int place_of(int r, int c) { return DH == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4); }

  // The products of a tile, in two chains of accumulators where a row has two halves.
  __device__ void logits(const Keys& kr, float (&s)[NB][4]) {
    float z[kHalves][NB][4];
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[h][nb][e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        const uint32_t k0 = kr.w[0][4 * h + w], k1 = kr.w[1][4 * h + w];
        const uint32_t a0 = code_pair<CODE, 0>(k0), a1 = code_pair<CODE, 0>(k1), a2 = code_pair<CODE, 2>(k0), a3 = code_pair<CODE, 2>(k1);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mma16816(z[h][nb], a0, a1, a2, a3, qf[nb][8 * h + 2 * w], qf[nb][8 * h + 2 * w + 1]);
      }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nb][e] = kHalves == 2 ? z[0][nb][e] + z[kHalves - 1][nb][e] : z[0][nb][e];
  }

  // s -> probabilities of N tiles (tokens from t0 on; rows see those below their limit and below `end`) against the rows' references,
  // summed; pb: as the second product's operand. A probability of zero stays zero whatever the scale: a block that the row does not
  // see may have none that is a number.
  template <int N>
  __device__ void softmax(float (&s)[N][NB][4], const float (&ks)[N], const float (&vs)[N], int t0, int end, int whole, uint32_t (&pb)[N][NB][2]) {
    bool move = false;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][nb][e] *= ks[n] * unit[nb][e & 1];
    if (t0 + 16 * N > whole) {                       // (uniform: a row's limit, or the warp's last tile, lies in these tiles; a row
                                                     // that pads the tile has limit 0, so with fewer rows than it holds in all of them)
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][nb][e] = t0 + 16 * n + gq + 8 * (e >> 1) < min(end, lim[nb][e & 1]) ? s[n][nb][e] : -INFINITY;
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) move |= s[n][nb][e] > over[nb][e & 1];
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = -INFINITY;
#pragma unroll
          for (int n = 0; n < N; ++n) m = fmaxf(m, fmaxf(s[n][nb][e], s[n][nb][e + 2]));
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
          const bool none = over[nb][e] == -INFINITY;
          const float from = none ? -INFINITY : sub[nb][e], to = fmaxf(from, m);
          const float f = from == to ? 1.f : tc::ex2(from - to);
          sub[nb][e] = to == -INFINITY ? 0.f : to;
          over[nb][e] = to + kMove;
          l[nb][e] *= f;
#pragma unroll
          for (int i = 0; i < DH / 16; ++i) {
            o[i][nb][e] *= f;
            o[i][nb][e + 2] *= f;
          }
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float vmul = vs[n] * vinv;
      const bool odd = !(vmul < INFINITY);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][nb][e] = tc::ex2(s[n][nb][e] - sub[nb][e & 1]);
          p[e] = s[n][nb][e] * vmul;
        }
        l[nb][0] += s[n][nb][0] + s[n][nb][2];
        l[nb][1] += s[n][nb][1] + s[n][nb][3];
        if (odd) {
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = s[n][nb][e] == 0.f ? 0.f : p[e];
        }
        pb[n][nb][0] = pack_f16(p[0], p[1]);
        pb[n][nb][1] = pack_f16(p[2], p[3]);
        movmatrix(pb[n][nb][0]);
        movmatrix(pb[n][nb][1]);
      }
    }
  }
  // the unit of the accumulator is vref 2^-7: a larger scale of V moves it
  __device__ void raise(float vs) {
    if (vs > vref) {
      const float f = vref / vs;
      vref = vs;
      vinv = 128.f / vs;
#pragma unroll
      for (int i = 0; i < DH / 16; ++i)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][nb][e] *= f;
    }
  }

  __device__ void values(const Values& vr, const uint32_t (&pb)[NB][2]) {
#pragma unroll
    for (int w = 0; w < kVw; ++w) {
      const uint32_t x0 = __byte_perm(vr.w[0][w], vr.w[1][w], 0x5140), y0 = __byte_perm(vr.w[0][w], vr.w[1][w], 0x7362);
      const uint32_t x1 = __byte_perm(vr.w[2][w], vr.w[3][w], 0x5140), y1 = __byte_perm(vr.w[2][w], vr.w[3][w], 0x7362);
      const uint32_t a0 = code_pair<CODE, 0>(x0), a1 = code_pair<CODE, 2>(x0), a2 = code_pair<CODE, 0>(x1), a3 = code_pair<CODE, 2>(x1);
      const uint32_t c0 = code_pair<CODE, 0>(y0), c1 = code_pair<CODE, 2>(y0), c2 = code_pair<CODE, 0>(y1), c3 = code_pair<CODE, 2>(y1);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        mma16816(o[2 * w][nb], a0, a1, a2, a3, pb[nb][0], pb[nb][1]);
        mma16816(o[2 * w + 1][nb], c0, c1, c2, c3, pb[nb][0], pb[nb][1]);
      }
    }
  }

  // Tiles [ta, tb) of 16 coded tokens.
  __device__ void coded(const AttnArgs& a, const Segment& g, int ta, int tb) {
    if (ta >= tb) {
      settle(a);
      return;
    }
    const int per = a.page >> 4, sh = a.page_shift - 4;       // tiles per page
    PageWindow w;
    const int end_page = ((tb - 1) >> sh) + 1;
    auto fill = [&](int first) {
      w.fill(a, g, first, end_page, lane);
      raise(__uint_as_float(__reduce_max_sync(0xffffffffu, w.vs < INFINITY ? __float_as_uint(w.vs) : 0u)));
    };
    fill(ta >> sh);
    int whole = tb * 16;                                      // tokens that every row of the tile sees (0 where some are padding)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) whole = min(whole, lim[nb][e]);
    whole = __reduce_min_sync(0xffffffffu, whole);
    float ks[kStages], vs[kStages];                           // of the tiles in the ring, the nearest first
    auto ask = [&](int t, int i) {                            // tile t is to be the ring's i-th
      if (t < tb) {
        if (t >> sh >= w.base + 32) fill(t >> sh);
        const int p = (t >> sh) - w.base;
        const int id = __shfl_sync(0xffffffffu, w.id, p);
        ks[i] = __shfl_sync(0xffffffffu, w.ks, p);
        vs[i] = __shfl_sync(0xffffffffu, w.vs, p);
        if (tc::elect_one()) {
          const int st = put, row = ((id * a.c.n_kv + g.kvh) << a.page_shift) + (t & (per - 1)) * 16;
          tc::mbar_arrive_expect_tx(bars + st, kStageBytes);
          tc::tma_tile2d(ring + st * kStageBytes, &a.map[0], bars + st, 0, row);
          tc::tma_tile2d(ring + st * kStageBytes + kTileBytes, &a.map[1], bars + st, 0, row);
        }
        put = put + 1 == kStages ? 0 : put + 1;
      }
    };
#pragma unroll
    for (int i = 0; i < kStages - 2; ++i) ask(ta + i, i);
    settle(a);
    // Two tiles at a time: their chains of products run beside each other, and one vote and one look at the references serve both.
#pragma unroll 1
    for (int t = ta; t < tb; t += 2) {
      __syncwarp();                                           // the stages asked for next have been read by all lanes
      ask(t + kStages - 2, kStages - 2);
      ask(t + kStages - 1, kStages - 1);
      const bool two = t + 1 < tb;
      float s[2][NB][4];
      uint32_t pb[2][NB][2];
      const int next = get + 1 == kStages ? 0 : get + 1;
      const uint32_t next_phase = next == 0 ? phase ^ 1u : phase;
      const uint8_t* t0 = ring + get * kStageBytes;
      const uint8_t* t1 = ring + next * kStageBytes;
      if (!fl_tc::warp_wait(bars + get, phase, abort_flag)) return;
      if (two && !fl_tc::warp_wait(bars + next, next_phase, abort_flag)) return;
      get = next;
      phase = next_phase;
      if (two) {
        get = next + 1 == kStages ? 0 : next + 1;
        phase = get == 0 ? next_phase ^ 1u : next_phase;
      }
      Keys k0, k1;
      Values x0, x1;
      take_k(k0, t0);
      take_k(k1, t1);
      take_v(x0, t0);
      logits(k0, s[0]);
      if (two) {
        logits(k1, s[1]);
      } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[1][nb][e] = 0.f;
        ks[1] = vs[1] = 0.f;
      }
      const float k2[2] = {ks[0], ks[1]}, v2[2] = {vs[0], vs[1]};
      softmax<2>(s, k2, v2, t * 16, tb * 16, whole, pb);
      take_v(x1, t1);
      values(x0, pb[0]);
      if (two) values(x1, pb[1]);
#pragma unroll
      for (int k = 0; k + 2 < kStages; ++k) {
        ks[k] = ks[k + 2];
        vs[k] = vs[k + 2];
      }
    }
  }

  // Every kWarps-th tile of the open block, whose rows are bf16. Rows from the sequence's end on are taken as zeros. A value that is no number is
  // added only to the rows that see it.
  __device__ void opened(const AttnArgs& a, const Segment& g, int ta, int tb, int full, int slot) {
    const int64_t head = ((int64_t)slot * a.c.n_kv + g.kvh) * a.page * DH;
#pragma unroll 1
    for (int t = ta; t < tb; t += kWarps) {
      const T* kp = static_cast<const T*>(a.c.open[0]) + head;
      const T* vp = static_cast<const T*>(a.c.open[1]) + head;
      const int r0 = t * 16 - full;
      float s1[1][NB][4];
      float(&s)[NB][4] = s1[0];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nb][e] = 0.f;
      uint32_t x[2][kHalves * 8], top = 0;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const bool in = t * 16 + gq + 8 * r < g.len;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          const uint4* p = reinterpret_cast<const uint4*>(kp + (int64_t)(r0 + gq + 8 * r) * DH + 16 * (kHalves * q4 + h));
          const uint4 zero = make_uint4(0u, 0u, 0u, 0u), u = in ? *p : zero, v = in ? p[1] : zero;
          uint32_t* f = &x[r][8 * h];
          f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w;
          f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
        }
#pragma unroll
        for (int i = 0; i < kHalves * 8; ++i) top = largest(top, x[r][i]);
      }
      uint32_t y[4][DH / 16];                        // four tokens, DH / 8 dims
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = 2 * q4 + (k & 1) + 8 * (k >> 1);
        const bool in = t * 16 + r < g.len;
        const uint4* p = reinterpret_cast<const uint4*>(vp + (int64_t)(r0 + r) * DH + (DH / 8) * gq);
#pragma unroll
        for (int i = 0; i < DH / 64; ++i) {
          const uint4 u = in ? p[i] : make_uint4(0u, 0u, 0u, 0u);
          y[k][4 * i] = u.x; y[k][4 * i + 1] = u.y; y[k][4 * i + 2] = u.z; y[k][4 * i + 3] = u.w;
        }
      }
      float mul, inv;
      to_power(__reduce_max_sync(0xffffffffu, top), 14, &mul, &inv);
#pragma unroll
      for (int w = 0; w < kHalves * 4; ++w) {
        const uint32_t a0 = scaled_f16(x[0][2 * w], mul), a1 = scaled_f16(x[1][2 * w], mul);
        const uint32_t a2 = scaled_f16(x[0][2 * w + 1], mul), a3 = scaled_f16(x[1][2 * w + 1], mul);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mma16816(s[nb], a0, a1, a2, a3, qf[nb][2 * w], qf[nb][2 * w + 1]);
      }
      const float ks[1] = {inv};
      bool odd = false;
      top = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) {
          odd |= (y[k][i] & 0x7f80u) == 0x7f80u || (y[k][i] & 0x7f800000u) == 0x7f800000u;
          top = largest(top, y[k][i]);
        }
      to_power(__reduce_max_sync(0xffffffffu, top), 6, &mul, &inv);
      raise(inv);
      uint32_t pb1[1][NB][2];
      const float vs[1] = {inv};
      softmax<1>(s1, ks, vs, t * 16, g.len, 0, pb1);
      uint32_t(&pb)[NB][2] = pb1[0];
      if (!__any_sync(0xffffffffu, odd)) {
#pragma unroll
        for (int m = 0; m < DH / 16; ++m) {
          const uint32_t y0 = scaled_f16(y[0][m], mul), y1 = scaled_f16(y[1][m], mul), y2 = scaled_f16(y[2][m], mul), y3 = scaled_f16(y[3][m], mul);
          const uint32_t a0 = __byte_perm(y0, y1, 0x5410), a1 = __byte_perm(y0, y1, 0x7632);
          const uint32_t a2 = __byte_perm(y2, y3, 0x5410), a3 = __byte_perm(y2, y3, 0x7632);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma16816(o[m][nb], a0, a1, a2, a3, pb[nb][0], pb[nb][1]);
        }
      } else {
#pragma unroll 1
        for (int r = 0; r < 16 && t * 16 + r < g.len; ++r) {
          const T* p = vp + (int64_t)(r0 + r) * DH + (DH / 8) * gq;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float w0 = __shfl_sync(0xffffffffu, s[nb][e], (r & 7) * 4 + q4), w1 = __shfl_sync(0xffffffffu, s[nb][e + 2], (r & 7) * 4 + q4);
              if (t * 16 + r < lim[nb][e]) {
                const float w = (r < 8 ? w0 : w1) * vinv;
#pragma unroll
                for (int m = 0; m < DH / 16; ++m) {
                  o[m][nb][e] += w * __bfloat162float(p[2 * m]);
                  o[m][nb][e + 2] += w * __bfloat162float(p[2 * m + 1]);
                }
              }
            }
        }
      }
    }
  }

  // Leaves the warp's sums and accumulators: [row][dim], and (reference, sum) of a row.
  __device__ void leave(float* so, float2* sm) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sum = l[nb][e];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        const int r = nb * 8 + 2 * q4 + e;
        if (gq == 0) sm[r] = make_float2(over[nb][e] == -INFINITY ? -INFINITY : sub[nb][e], sum);
#pragma unroll
        for (int m = 0; m < DH / 16; ++m)
          *reinterpret_cast<float2*>(so + r * DH + (DH / 8) * gq + 2 * m) = make_float2(o[m][nb][e] * (vref * 0x1p-7f), o[m][nb][e + 2] * (vref * 0x1p-7f));
      }
  }
};

// ------------------------------------------------------------------------------------------------------------
// Binary32 storage: the same work on the FMA pipe. A pair of lanes has a token of the tile for the first product, a lane four (two)
// dims for the second; Q rows and probabilities stand in shared memory. With one row per kv head the conversions cost as much as the products.
// Bound by its instructions at eight warps an SM (255 registers, 64 bytes of spills with heads of 128): one leaves in 53% of the cycles; ALU
// (conversions) 35%, FMA 29%, LSU 24% of their rates. The next tile's codes are on their way meanwhile: 32 sequences of up to 16384 tokens
// 1299 us, 2546 with each tile's loads in its own loops; 256 rows x 16 heads on 4096 tokens 817 us = 10 TFLOP/s, 2608 where limits and
// visibility were looked up for every token.
// ------------------------------------------------------------------------------------------------------------
template <int DH, int CODE>
struct SimtEngine {
  static constexpr int kRows = 8, kDim = DH, kW = DH / 32;   // dims per lane of the second product
  using T = float;
  struct Shared {
    float q[8][DH];
    float p[kWarps][16][8];
  };
  static constexpr int kCtas = 2;                  // per SM
  static constexpr int kWarpBytes = kRows * DH * 4;
  static constexpr int kExtra = kWarps * kWarpBytes + sizeof(Shared);
  Shared* sh;
  __device__ void place(uint8_t* extra, uint64_t*, int*) { sh = reinterpret_cast<Shared*>(extra + kWarps * kWarpBytes); }
  float o[8][kW], l[8], ref[8];
  int lim[8];                                      // tokens that the rows see
  int lane, warp, rows;
  // A tile's codes, as they are stored: the lane's half of its token's key, its dims of every token's value.
  struct Codes {
    uint4 k[DH / 32];
    uint32_t v[16];
    float ks, vs;
  };

  __device__ void begin(const AttnArgs& a, const Segment& g, int rows_) {
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    rows = rows_;
    const int group = a.group, row0 = g.tile * kRows, lim0 = g.len - g.n + 1;
    for (int i = threadIdx.x; i < 8 * DH; i += kWarps * 32) {
      const int r = i / DH, d = i - r * DH, row = row0 + r, tok = row / group;
      sh->q[r][d] = r < rows ? static_cast<const T*>(a.q)[(int64_t)(g.s + tok) * a.q_stride + (int64_t)(g.kvh * group + row - tok * group) * DH + d] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      l[r] = 0.f;
      ref[r] = -INFINITY;
      lim[r] = lim0 + (row0 + r) / group;
#pragma unroll
      for (int i = 0; i < kW; ++i) o[r][i] = 0.f;
    }
    __syncthreads();
  }
  // key(x, j): the lane's elements 8j .. of its half of its token; value(x, r): the lane's elements of token r; n: tokens of the tile that
  // exist. CODED: all of them, and values that are numbers, so that those a row does not see need no look (their probabilities are zeros)
  template <bool CODED, typename FK, typename FV>
  __device__ void tile(float ks, float vs, int t0, int n, FK key, FV value) {
    const int tok = lane >> 1, half = lane & 1;
    float s[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) s[r] = 0.f;
#pragma unroll (CODED ? DH / 16 : 2)
    for (int j = 0; j < DH / 16; ++j) {
      const int d = half * (DH / 2) + 8 * j;
      float x[8];
      key(x, j);
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < rows) {
          const float4 u = *reinterpret_cast<const float4*>(&sh->q[r][d]), v = *reinterpret_cast<const float4*>(&sh->q[r][d + 4]);
          s[r] += x[0] * u.x + x[1] * u.y + x[2] * u.z + x[3] * u.w + x[4] * v.x + x[5] * v.y + x[6] * v.z + x[7] * v.w;
        }
    }
    bool over = false;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
      const bool seen = r < rows && tok < n && t0 + tok < lim[r];
      s[r] = seen ? s[r] * ks : -INFINITY;
      over |= s[r] > ref[r] + kMove;
    }
    if (__any_sync(0xffffffffu, over)) {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        float m = s[r];
#pragma unroll
        for (int x = 2; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
        const float to = fmaxf(ref[r], m), f = ref[r] == to ? 1.f : exp2f(ref[r] - to);
        ref[r] = to;
        l[r] *= f;
#pragma unroll
        for (int i = 0; i < kW; ++i) o[r][i] *= f;
      }
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      s[r] = exp2f(s[r] - (ref[r] == -INFINITY ? 0.f : ref[r]));
      l[r] += s[r];
      if (half == 0) sh->p[warp][tok][r] = s[r] == 0.f ? 0.f : s[r] * vs;
    }
    __syncwarp();
#pragma unroll (CODED ? 16 : 4)
    for (int k = 0; k < (CODED ? 16 : n); ++k) {
      float v[kW];
      value(v, k);
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < rows) {
          const float p = sh->p[warp][k][r];
          if (CODED || t0 + k < lim[r]) {
#pragma unroll
            for (int i = 0; i < kW; ++i) o[r][i] += p * v[i];
          }
        }
    }
    __syncwarp();
  }
  __device__ void coded(const AttnArgs& a, const Segment& g, int ta, int tb) {
    if (ta >= tb) return;
    const int per = a.page >> 4, sft = a.page_shift - 4, end_page = ((tb - 1) >> sft) + 1;
    PageWindow w;
    w.fill(a, g, ta >> sft, end_page, lane);
    auto load = [&](int t, Codes& c) {
      const int pi = t >> sft;
      if (pi >= w.base + 32) w.fill(a, g, pi, end_page, lane);
      const int id = __shfl_sync(0xffffffffu, w.id, pi - w.base);
      c.ks = __shfl_sync(0xffffffffu, w.ks, pi - w.base);
      c.vs = __shfl_sync(0xffffffffu, w.vs, pi - w.base);
      const int64_t at = ((int64_t)id * a.c.n_kv + g.kvh) * a.page * DH + (int64_t)(t & (per - 1)) * 16 * DH;
      const uint8_t* kp = a.c.codes[0] + at + lane * (DH / 2);
      const uint8_t* vp = a.c.codes[1] + at + kW * lane;
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) c.k[i] = __ldg(reinterpret_cast<const uint4*>(kp) + i);
#pragma unroll
      for (int k = 0; k < 16; ++k)
        c.v[k] = kW == 4 ? __ldg(reinterpret_cast<const uint32_t*>(vp + k * DH)) : (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(vp + k * DH));
    };
    Codes c, next;
    load(ta, c);
#pragma unroll 1
    for (int t = ta; t < tb; ++t) {
      if (t + 1 < tb) load(t + 1, next);                     // on their way while this tile is multiplied
      tile<true>(c.ks * a.scale_log2, c.vs, t * 16, 16,
           [&](float (&x)[8], int j) {
             const uint4 u = c.k[j >> 1];
             float y[4], z[4];
             decode4<CODE>(j & 1 ? u.z : u.x, y);
             decode4<CODE>(j & 1 ? u.w : u.y, z);
#pragma unroll
             for (int i = 0; i < 4; ++i) { x[i] = y[i]; x[4 + i] = z[i]; }
           },
           [&](float (&v)[kW], int k) {
             float y[4];
             decode4<CODE>(c.v[k], y);
#pragma unroll
             for (int i = 0; i < kW; ++i) v[i] = y[i];
           });
      c = next;
    }
  }
  __device__ void opened(const AttnArgs& a, const Segment& g, int ta, int tb, int full, int slot) {
    const int64_t head = ((int64_t)slot * a.c.n_kv + g.kvh) * a.page * DH;
#pragma unroll 1
    for (int t = ta; t < tb; t += kWarps) {
      const int n = min(16, g.len - t * 16);
      const T* kp = static_cast<const T*>(a.c.open[0]) + head + (int64_t)(t * 16 - full + min(lane >> 1, n - 1)) * DH;
      const T* vp = static_cast<const T*>(a.c.open[1]) + head + (int64_t)(t * 16 - full) * DH + kW * lane;
      tile<false>(a.scale_log2, 1.f, t * 16, n, [&](float (&x)[8], int j) { load8(kp + (lane & 1) * (DH / 2) + 8 * j, x); },
           [&](float (&v)[kW], int k) {
#pragma unroll
             for (int i = 0; i < kW; ++i) v[i] = vp[k * DH + i];
           });
    }
  }
  __device__ void leave(float* so, float2* sm) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      float sum = l[r];                              // both lanes of a token have its probability
#pragma unroll
      for (int x = 2; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      if (lane == 0) sm[r] = make_float2(ref[r], sum);
#pragma unroll
      for (int i = 0; i < kW; ++i) so[r * DH + kW * lane + i] = o[r][i];
    }
  }
};

template <int ROWS>
struct Meeting {                                     // where the warps of a CTA leave their results (accumulators: over their rings)
  float2 m[kWarps][ROWS];
  float weight[kWarps][ROWS];
  int64_t at[ROWS];                                  // rows of the output
  uint64_t bars[kWarps][kMostStages];
  Range range;
  int arrived, abort_flag;
};
template <typename E> constexpr int kMeetingBytes = (int)(sizeof(Meeting<E::kRows>) + 1023) / 1024 * 1024;

// A warp's share of a problem's parts (every kWarps-th, in their order) for rows r0 .. r0 + RU - 1, CU parts on their way at a time: a lane
// has DH / 32 dims. The result stands where the warp's own did.
template <int ROWS, int DH, int RU, int CU>
__device__ __forceinline__ void gather_parts(const AttnArgs& a, const Segment& g, int r0, int rows, float* so, float2* sm) {
  constexpr int kStat = ROWS * DH, kSlot = ROWS * (DH + 2), V = DH / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float acc[RU][V], sum[RU], top[RU];
#pragma unroll
  for (int k = 0; k < RU; ++k) {
    sum[k] = 0.f;
    top[k] = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[k][i] = 0.f;
  }
  for (int c0 = g.first + warp; c0 <= g.last; c0 += kWarps * CU) {
    float x[CU][RU][V];
    float2 m[CU][RU];
#pragma unroll
    for (int c = 0; c < CU; ++c) {
      const float* p = a.part + (int64_t)part_slot(min(c0 + c * kWarps, g.last), g.first) * kSlot;
#pragma unroll
      for (int k = 0; k < RU; ++k) {
        const int r = min(r0 + k, rows - 1);
        if (V == 4) {
          const float4 f = __ldcg(reinterpret_cast<const float4*>(p + r * DH) + lane);
          x[c][k][0] = f.x; x[c][k][1] = f.y; x[c][k][2 % V] = f.z; x[c][k][3 % V] = f.w;
        } else {
          const float2 f = __ldcg(reinterpret_cast<const float2*>(p + r * DH) + lane);
          x[c][k][0] = f.x; x[c][k][1] = f.y;
        }
        m[c][k] = __ldcg(reinterpret_cast<const float2*>(p + kStat) + r);
      }
    }
#pragma unroll
    for (int k = 0; k < RU; ++k) {
      float to = top[k];
#pragma unroll
      for (int c = 0; c < CU; ++c)
        if (c0 + c * kWarps <= g.last) to = fmaxf(to, m[c][k].x);
      const float f = part_weight(top[k], to);
      sum[k] *= f;
#pragma unroll
      for (int i = 0; i < V; ++i) acc[k][i] *= f;
      top[k] = to;
#pragma unroll
      for (int c = 0; c < CU; ++c)
        if (c0 + c * kWarps <= g.last) {
          const float w = part_weight(m[c][k].x, to);
          sum[k] += w * m[c][k].y;
#pragma unroll
          for (int i = 0; i < V; ++i) acc[k][i] += w * x[c][k][i];
        }
    }
  }
#pragma unroll
  for (int k = 0; k < RU; ++k)
    if (r0 + k < rows) {
#pragma unroll
      for (int i = 0; i < V; ++i) so[(r0 + k) * DH + V * lane + i] = acc[k][i];
      if (lane == 0) sm[r0 + k] = make_float2(top[k], sum[k]);
    }
}

template <typename E>
__global__ void __launch_bounds__(kWarps * 32, E::kCtas) cache_attn_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int ROWS = E::kRows, DH = E::kDim;
  using T = typename E::T;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Meeting<ROWS>& meet = *reinterpret_cast<Meeting<ROWS>*>(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid < kWarps * kMostStages) tc::mbar_init(&meet.bars[0][0] + tid, 1);
  if (tid == 0) {
    meet.abort_flag = 0;
    tc::fence_barrier_init();
  }
  fl_grid_wait();
  fl_grid_release();
  if (warp == 0) {
    const Range r = find_range<ROWS, kUnit>(a, lane);
    if (lane == 0) meet.range = r;
  }
  __syncthreads();
  const Range range = meet.range;
  E e;
  uint8_t* extra = smem + kMeetingBytes<E>;
  auto left = [&](int w) { return reinterpret_cast<float*>(extra + w * E::kWarpBytes); };
  e.place(extra, &meet.bars[0][0], &meet.abort_flag);
  for_each_segment<ROWS, kUnit>(a, range, [&](const Segment& g) {
    const int rows = rows_of(a, g, ROWS);
    e.begin(a, g, rows);
    // 16-token tiles: a run of the coded ones for each warp, those of the open block in turn; rows see nothing past the last one's limit
    const int full = g.len >> a.page_shift << a.page_shift;
    const int seen = max(0, min(g.len, limit_of(a, g, g.tile * ROWS + rows - 1)));
    const int ta = g.blk0 * (kUnit / 16), tb = min(g.blk1 * (kUnit / 16), (seen + 15) >> 4), tc = max(ta, min(tb, full >> 4));
    e.coded(a, g, ta + (tc - ta) * warp / kWarps, ta + (tc - ta) * (warp + 1) / kWarps);
    if (tc + warp < tb) {
      const int slot = cache_slot(a.c, g.b, a.status);
      if (slot >= 0) e.opened(a, g, tc + warp, tb, full, slot);
    }
    __syncwarp();
    e.leave(left(warp), meet.m[warp]);
    __syncthreads();
    constexpr int kStep = kWarps * 32 / DH;          // rows at a time
    const int d = tid % DH;
    float* part = a.part + (int64_t)part_slot(blockIdx.x, g.first) * ROWS * (DH + 2);
    auto combine = [&](bool last) {                  // the warps' results: to the output, or as the CTA's part
      if (tid < rows) {                              // a row's thread has all that is not a dim's
        float top = -INFINITY, sum = 0.f, f[kWarps];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, meet.m[w][tid].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          f[w] = part_weight(meet.m[w][tid].x, top);
          sum += f[w] * meet.m[w][tid].y;
        }
        const float norm = !last ? 1.f : sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;     // (a sum that is no number stays none)
#pragma unroll
        for (int w = 0; w < kWarps; ++w) meet.weight[w][tid] = f[w] * norm;
        if (last) {
          const int64_t at = out_row(a, g, g.tile * ROWS + tid);
          meet.at[tid] = at;
          if (a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
        } else {
          __stcg(reinterpret_cast<float2*>(part + ROWS * DH) + tid, make_float2(top, sum));
        }
      }
      __syncthreads();
#pragma unroll 4
      for (int r = tid / DH; r < rows; r += kStep) {
        float acc = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) acc += meet.weight[w][r] * left(w)[r * DH + d];
        if (!last) __stcg(part + r * DH + d, acc);
        else if (sizeof(T) == 2) static_cast<__nv_bfloat16*>(a.o)[meet.at[r] * DH + d] = __float2bfloat16_rn(acc);
        else static_cast<float*>(a.o)[meet.at[r] * DH + d] = acc;
      }
    };
    combine(g.whole());
    if (!g.whole()) {
      __syncthreads();
      if (tid == 0) {
        __threadfence();                             // (what the CTA's other threads wrote before the barrier goes with it)
        const int n = g.last - g.first + 1, old = atomicAdd(a.counters + g.first, 1);
        meet.arrived = old == n - 1;
        if (old == n - 1) a.counters[g.first] = 0;
      }
      __syncthreads();
      if (meet.arrived) {
        __threadfence();
        if (rows == 1) {
          gather_parts<ROWS, DH, 1, 8>(a, g, 0, rows, left(warp), meet.m[warp]);
        } else {
          constexpr int kAtOnce = E::kCtas == 2 ? 8 : 4;   // (as the engine's registers allow)
          for (int r = 0; r < rows; r += kAtOnce) gather_parts<ROWS, DH, kAtOnce, 2>(a, g, r, rows, left(warp), meet.m[warp]);
        }
        __syncthreads();
        combine(true);
      }
    }
    tc::fence_proxy_async_smem();                    // the next tiles come where these results stood
    __syncthreads();
  });
  if (meet.abort_flag != 0) {                        // copies may still be on their way: the CTA outlives them
    for (int it = 0; it < (1 << 16); ++it) __nanosleep(256);
    if (tid == 0 && a.status != nullptr) atomicExch(a.status, (int)FL_ERR_TIMEOUT);
  }
}

template <typename E> constexpr size_t kSmemBytes = 1024 + kMeetingBytes<E> + E::kExtra;   // (tiles stand on 1024-byte boundaries)

constexpr int kMostCtas = 3;       // per SM, of any engine

template <typename E>
int launch(fl_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  static_assert(E::kCtas <= kMostCtas, "workspace");
  FL_FUNC_ATTR_ONCE(ctx, cache_attn_kernel<E>, kSmemBytes<E>, true);
  FL_CHECK_CUDA(fl_launch(ctx, cache_attn_kernel<E>, dim3((unsigned)(ctx->sm_count * E::kCtas)), dim3(kWarps * 32), kSmemBytes<E>, st, a));
  return fl_launch_status();
}

template <int DH, int CODE>
int launch_rows(fl_ctx* ctx, const AttnArgs& a, int dtype, int rows, cudaStream_t st) {
  if (dtype == FL_F32) return launch<SimtEngine<DH, CODE>>(ctx, a, st);
  return rows <= 8 ? launch<MmaEngine<DH, CODE, 1>>(ctx, a, st) : launch<MmaEngine<DH, CODE, 2>>(ctx, a, st);
}

int check_call(const fl_paged_kv* cache, int32_t n_heads, int32_t n_tokens, int32_t max_q) {
  const int rc = fl_check_cache(cache);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(n_heads >= 1 && n_heads % cache->n_kv_heads == 0 && n_tokens >= 0 && max_q >= 1);
  if (n_heads / cache->n_kv_heads > 128) return FL_ERR_UNSUPPORTED;
  FL_REQUIRE((int64_t)max_q * (n_heads / cache->n_kv_heads) <= INT32_MAX / 2);
  return FL_OK;
}

// This kernel's counters, its partial results, the chunk kernel's (whose cut problems need no counters).
int64_t counter_bytes(const fl_ctx* ctx) { return ((int64_t)ctx->sm_count * kMostCtas * 4 + 255) / 256 * 256; }
int64_t part_bytes(const fl_ctx* ctx, int head_dim) {
  return ((int64_t)ctx->sm_count * kMostCtas * 2 * kFewRows * (head_dim + 2) * 4 + 255) / 256 * 256;
}
bool has_chunks(const fl_paged_kv* cache, int32_t n_heads, int32_t max_q) {
  return cache->dtype == FL_BF16 && max_q * (n_heads / cache->n_kv_heads) > kFewRows;
}

}  // namespace

extern "C" int fl_cache_attention_workspace_bytes(fl_ctx* ctx, const fl_paged_kv* cache, int32_t n_heads, int32_t n_tokens, int32_t max_q,
                                                  int64_t* bytes) {
  FL_REQUIRE(ctx != nullptr && bytes != nullptr);
  const int rc = check_call(cache, n_heads, n_tokens, max_q);
  if (rc != FL_OK) return rc;
  *bytes = counter_bytes(ctx) + part_bytes(ctx, cache->head_dim);
  if (has_chunks(cache, n_heads, max_q)) *bytes += fl_cache_attn_tc_part_bytes(ctx, cache->head_dim);
  return FL_OK;
}

extern "C" int fl_cache_attention(fl_ctx* ctx, const fl_paged_kv* cache, const void* q, int64_t q_stride, int32_t n_heads,
                                  const int32_t* seq_start, int32_t n_tokens, int32_t max_q, const int32_t* kv_len, float sm_scale, void* o,
                                  float* lse, void* workspace, int64_t workspace_bytes, int32_t* status, void* stream) {
  int64_t need = 0;
  const int rc = fl_cache_attention_workspace_bytes(ctx, cache, n_heads, n_tokens, max_q, &need);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(sm_scale > 0.f && sm_scale <= 3.4028234e38f);
  const int64_t piece = cache->dtype == FL_BF16 ? 8 : 4;
  FL_REQUIRE(q_stride >= (int64_t)n_heads * cache->head_dim && q_stride % piece == 0);
  if (n_tokens == 0) return FL_OK;
  FL_REQUIRE(q != nullptr && o != nullptr && seq_start != nullptr && kv_len != nullptr);
  FL_REQUIRE(fl_aligned16(q) && fl_aligned16(o));
  FL_REQUIRE(workspace != nullptr && (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0);
  if (workspace_bytes < need) return FL_ERR_WORKSPACE;
  AttnArgs a = {};
  a.c = fl_cache_args(cache);
  a.q = q;
  a.q_stride = q_stride;
  a.seq_start = seq_start;
  a.kv_len = kv_len;
  a.o = o;
  a.lse = lse;
  a.counters = static_cast<int32_t*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + counter_bytes(ctx));
  a.status = status;
  a.n_tokens = n_tokens;
  a.n_heads = n_heads;
  a.group = n_heads / cache->n_kv_heads;
  a.max_q = max_q;
  a.page = cache->page;
  a.page_shift = cache->page == 16 ? 4 : cache->page == 32 ? 5 : cache->page == 64 ? 6 : 7;
  a.which = kEvery;
  a.little = kLittle / ((int64_t)cache->n_kv_heads * cache->n_seqs);
  // Two units are worth a CTA of their own: one row over 8192 tokens 16 us so, 19 with eight. A problem's queries, first loads, and
  // result cost what ten units of its tokens do: 32 sequences of up to 16384 tokens take 208 us so, 221 where they count as two.
  a.min_units = 2;
  a.head_units = 10;
  a.scale_log2 = sm_scale * kLog2e;
  if (cache->dtype == FL_BF16) {
    const int64_t code_rows = (int64_t)cache->n_pages * cache->n_kv_heads * cache->page;
    if (!fl_code_tmap(ctx, cache->k_codes, code_rows, cache->head_dim, 16, &a.map[0]) ||
        !fl_code_tmap(ctx, cache->v_codes, code_rows, cache->head_dim, 16, &a.map[1]))
      return FL_ERR_UNSUPPORTED;
  }
  a.max_parts = INT32_MAX;
  const int rows = max_q * a.group;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool chunks = has_chunks(cache, n_heads, max_q);
  if (chunks) a.which = kFew;
  int rc2 = FL_OK;
  // a batch may hold both: where a sequence could have more rows than a decode step's, each kernel takes its own
  if (cache->head_dim == 128)
    rc2 = cache->code == FL_INT8 ? launch_rows<128, FL_INT8>(ctx, a, cache->dtype, rows, st) : launch_rows<128, FL_E4M3>(ctx, a, cache->dtype, rows, st);
  else
    rc2 = cache->code == FL_INT8 ? launch_rows<64, FL_INT8>(ctx, a, cache->dtype, rows, st) : launch_rows<64, FL_E4M3>(ctx, a, cache->dtype, rows, st);
  if (rc2 != FL_OK || !chunks) return rc2;
  a.which = kMany;
  a.part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.part) + part_bytes(ctx, cache->head_dim));
  return fl_launch_cache_attn_tc(ctx, a, cache->head_dim, cache->code, st);
}
