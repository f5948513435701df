// Attention of a prompt's chunk over its paged 8-bit cache on the Blackwell tensor path (bf16 storage).
//
// A problem is (sequence, kv head, 256 rows); rows are (new token, query head of the group), heads fastest, so that shared key heads
// fill the same tiles. The CTAs, one per SM, take equal runs of the chunks of 128 keys of all problems; what a run's border cuts is put
// together by a kernel of its own, which spreads it over the chip. Within a run the kernel is the dense loop's: two tiles of 128 rows that share each
// key and value tile, S = Q K^T and acc += P V by tcgen05 MMAs, softmax by a thread per row.
// What differs: keys and values come as codes. Four warps turn them into f16 operand tiles (exact: see code_pair) as fast as the
// two tiles use them up, and the scales never touch the operands: a block's scale of K goes into the factor of its
// columns' logits, its scale of V into the exponent of their probabilities, P' = 2^(s - ref + log2(2^7 vs / vref)), vref the largest scale
// so far, and the row's sum takes P' back in 32 bits.
// Bound by neither products nor exponentials alone: a chunk takes 6000 cycles where its products take 2000. With clocks read around the waits
// (8200 cycles a chunk) the warps of the codes work 4900 to 5600 of them, the softmax of the two tiles waits 800 and 2000, and Q K^T waits
// 3250 for the other tile to take its S; a warp gets an instruction off in eight to ten cycles, a fifth of them for want of the next one:
// the code of four roles is more than the instruction caches serve, and where it comes to lie moves the time by 3% either way. 2048 rows x
// 16 heads on 32768 tokens: int8 730, e4m3 729, pages of 16 806 us (730 = 727 TFLOP/s; 748 on one cache after another). At 720, with an eighth of
// the products, without the exponentials and with a sixteenth of the codes turned it took 770, 630 and 780.
#include "cache_attn.cuh"

namespace {

using namespace fl_ca;
using namespace fl_tc;

constexpr int kRows = 256, kNC_ = 128, kSlots = 4;
constexpr int kWarpsTc = 16, kThreadsTc = kWarpsTc * 32;
// warps 0-3, 4-7: softmax of a tile; 8: QK^T; 9: PV; 10: the plan; 11: pages and scales; 12-15: codes to operands. Registers of the four
// warpgroups: 2 x 192 + 64 + 64 of 512. int8 / e4m3 / pages of 16 when they were chosen: 716 / 748 / 797 us so, 748 / 737 / 827 with 208 + 48
// + 48, 702 / 767 / 779 with 192 + 56 + 72, 771 / 765 / 798 with 184 + 64 + 80.
constexpr int kQkWarp = 8, kPvWarp = 9, kPlanWarp = 10, kScaleWarp = 11, kCodeWarp = 12;
constexpr int kReaders = 15;           // warps that read the plan: softmax, issuers, scales, codes
constexpr int kRegsSoftmax = 192, kRegsIssue = 64, kRegsCodes = 64;
static_assert(2 * kRegsSoftmax + kRegsIssue + kRegsCodes <= 4 * 128, "more registers than the block is launched with");

struct alignas(16) Factors {   // of a chunk's groups of 16 tokens
  int row[8];               // first row of each in the pools
  uint32_t spoils;          // bit g: group g is of a block without scales that are numbers: its keys are none, and so is what sees them;
                            // bits 8 + g, 24 + g: of a block whose keys, values have scale zero: so are they, whatever the codes (and the
                            // values of a block without a scale, which only rows meet that do not see it or are none already)
  float ks[8], lv[8], iv[8];
  float rv, vref;           // old vref over the new one, the new one: negative where a value of the open block is no number
};
// A CTA's part of a problem, in chunks: tile t takes chunks [blk0, blk0 + cnt[t]). One warp lays the parts out ahead of the others, which
// keep none of it in registers (192 of them hardly hold a row of S and P).
constexpr int kPlans = 4;
struct Plan {
  Segment g;
  int rows, cnt[2], chunks, full;
  int end;                  // nothing more
};

struct __align__(16) Ctl {
  uint64_t plan_full[kPlans], plan_free[kPlans], box_full[4];
  uint64_t q_full[2], kv_full[kSlots], kv_free[kSlots], fac_full[4], fac_free[4], rows_full[4], open_full, s_full[2], s_free[2], p_full[2], pv_done[2];
  alignas(16) Factors fac[4];
  Plan plan[kPlans];
  Range range;
  uint32_t tmem_base, top[2][2][4];    // top: of one open block and the next
  int abort_flag, plan_abort;
};
template <int DH> constexpr int kTile = 128 * DH * 2;             // bytes of an operand tile: 128 rows of f16
template <int DH> constexpr int kBox = 16 * DH;                   // bytes: 16 rows of codes
template <int DH> constexpr size_t kSmemTc = 1024 + (2 + kSlots) * kTile<DH> + 16 * kBox<DH> + sizeof(Ctl);

template <int R> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R)); }
template <int R> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R)); }
__device__ __forceinline__ void named_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }

__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// The powers of two that bring the open block's rows into f16's range, from the largest magnitudes that the four warps found, and
// whether a value is no number.
__device__ __forceinline__ bool open_powers(const uint32_t (&top)[2][4], float* kmul, float* kinv, float* vmul, float* vinv) {
  const volatile uint32_t* k = top[0];
  const volatile uint32_t* v = top[1];
  const uint32_t v0 = v[0], v1 = v[1], v2 = v[2], v3 = v[3];
  to_power(max(max(k[0], k[1]), max(k[2], k[3])), 14, kmul, kinv);
  to_power(max(max(v0 & 0xffffu, v1 & 0xffffu), max(v2 & 0xffffu, v3 & 0xffffu)), 6, vmul, vinv);
  return ((v0 | v1 | v2 | v3) & 0x10000u) != 0;
}

// Bounded waits of the warps that have time (one thread, or a converged warp): the hardware wakes them, they hardly poll.
__device__ __forceinline__ bool patient(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  for (int it = 0; it < (1 << 17); ++it) {
    if (tc::mbar_try_wait_hint(bar, parity, 2000u)) return true;
    if (*abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool patient_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  bool ok = tc::mbar_try_wait(bar, parity);
  if (__all_sync(0xffffffffu, ok)) return true;
  if (!ok) ok = patient(bar, parity, abort_flag);
  return __all_sync(0xffffffffu, ok);
}

// P' of M logits, packed, and the sum of them.
template <int M>
__device__ __forceinline__ float exp_some(const uint32_t* r, float f, float add, uint32_t* p) {
  using namespace fl_codec;
  const f32x2 ff = pair(f, f), aa = pair(add, add);
  f32x2 sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
  for (int u = 0; u < M / 2; ++u) {
    float x0, x1;
    split(fma2(pair_u(r[2 * u], r[2 * u + 1]), ff, aa), x0, x1);
    const float p0 = tc::ex2(x0), p1 = tc::ex2(x1);
    sum[u & 1] = add2(sum[u & 1], pair(p0, p1));
    p[u] = pack_f16(p0, p1);
  }
  float s0, s1;
  split(add2(sum[0], sum[1]), s0, s1);
  return s0 + s1;
}
__device__ __forceinline__ float max16(const uint32_t* r) {
  float m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = max3(__uint_as_float(r[i]), __uint_as_float(r[i + 4]), __uint_as_float(r[i + 8]));
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = fmaxf(m[i], __uint_as_float(r[12 + i]));
  return fmaxf(max3(m[0], m[1], m[2]), m[3]);
}
// Log2 of a probability per unit of a product. Never zero, which would make a number of a hidden column's -inf no number; the
// smallest normal number beside it is lost in the rounding, or leaves products (below 2^37) as good as zero. (As fmaxf(ks * c2, 2^-126) it
// cost 3% of a long chunk.)
__device__ __forceinline__ float logit_unit(float ks, float c2) { return fmaf(ks, c2, 0x1p-126f); }
// 32 columns (block q of a chunk) whose groups of 16 share their factors where pages are of 32 tokens and more.
template <bool FINE>
__device__ __forceinline__ float max_block(const uint32_t (&r)[32], const Factors& f, int q, float c2) {
  if (FINE) return fmaxf(max16(r) * logit_unit(f.ks[2 * q], c2), max16(r + 16) * logit_unit(f.ks[2 * q + 1], c2));
  return max32(r) * logit_unit(f.ks[2 * q], c2);
}
template <bool FINE>
__device__ __forceinline__ float exp_block(const uint32_t (&r)[32], const Factors& f, int q, float c2, float sub, uint32_t (&p)[16]) {
  if (FINE) {
    const float a = exp_some<16>(r, logit_unit(f.ks[2 * q], c2), f.lv[2 * q] - sub, p) * f.iv[2 * q];
    return a + exp_some<16>(r + 16, logit_unit(f.ks[2 * q + 1], c2), f.lv[2 * q + 1] - sub, p + 8) * f.iv[2 * q + 1];
  }
  return exp_some<32>(r, logit_unit(f.ks[2 * q], c2), f.lv[2 * q] - sub, p) * f.iv[2 * q];
}

// FINE: pages of 16 tokens, factors for every 16 columns.
template <int DH, int CODE, bool FINE>
__global__ void __launch_bounds__(kThreadsTc, 1) cache_flash_kernel(const __grid_constant__ AttnArgs a) {
  constexpr uint32_t kAcc = 0, kS = 256, kP = 384;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + (-tc::smem_u32(smem_raw) & 1023u);    // (by an offset: the compiler still knows that it is shared memory)
  uint8_t* q_tiles = smem;
  uint8_t* ring = smem + 2 * kTile<DH>;
  uint8_t* boxes = ring + kSlots * kTile<DH>;
  Ctl& ctl = *reinterpret_cast<Ctl*>(boxes + 16 * kBox<DH>);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < 4; ++s) {
      tc::mbar_init(&ctl.kv_full[s], 2);
      tc::mbar_init(&ctl.box_full[s], 1);
      tc::mbar_init(&ctl.rows_full[s], 1);
      tc::mbar_init(&ctl.kv_free[s], 1);
      tc::mbar_init(&ctl.fac_full[s], 1);
      tc::mbar_init(&ctl.fac_free[s], 1);
    }
    for (int t = 0; t < 2; ++t) {
      tc::mbar_init(&ctl.q_full[t], 4);
      tc::mbar_init(&ctl.s_full[t], 1);
      tc::mbar_init(&ctl.s_free[t], 4);
      tc::mbar_init(&ctl.p_full[t], 4);
      tc::mbar_init(&ctl.pv_done[t], 1);
    }
    tc::mbar_init(&ctl.open_full, 4);
    for (int s = 0; s < kPlans; ++s) {
      tc::mbar_init(&ctl.plan_full[s], 1);
      tc::mbar_init(&ctl.plan_free[s], kReaders);
    }
    ctl.abort_flag = ctl.plan_abort = 0;
    tc::fence_barrier_init();
  }
  fl_grid_wait();
  fl_grid_release();
  if (warp == 0) {
    const Range r = find_range<kRows, kNC_>(a, lane);
    if (lane == 0) ctl.range = r;
  }
  __syncthreads();
  if (ctl.range.u0 == ctl.range.u1) return;                // nothing to do
  if (warp == kQkWarp) {
    tc::tmem_alloc(&ctl.tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = ctl.tmem_base;
  volatile int* abort_flag = &ctl.abort_flag;
  // body(plan) for every part, by a warp or by one of its threads; a part's place is free again when all readers are done with it. After a
  // wait that ran out every part is still gone through, by all warps, so that they meet at the same barriers: the waits for the plan do
  // not look at the flag that such a wait raises.
  volatile int* plan_abort = &ctl.plan_abort;
  auto for_each_plan = [&](bool whole_warp, auto body) {
    for (int s = 0;; ++s) {
      const bool there = whole_warp ? patient_warp(&ctl.plan_full[s % kPlans], (s / kPlans) & 1, plan_abort)
                                    : patient(&ctl.plan_full[s % kPlans], (s / kPlans) & 1, plan_abort);
      const Plan& p = ctl.plan[s % kPlans];
      if (!there || p.end) break;
      body(p);
      if (whole_warp) __syncwarp();
      if (!whole_warp || lane == 0) tc::mbar_arrive(&ctl.plan_free[s % kPlans]);
    }
  };

  if (warp >= kCodeWarp) {
    // ============================================ codes -> operands ============================================
    regs_down<kRegsCodes>();
    // Two warps have the keys, two the values, 64 rows of a tile each. The codes come by TMA, the next chunk's
    // as soon as this one's have been read. One piece of code, its loop half rolled: laid
    // out flat, with loads of their own on their way in registers, the warps of three roles ran out of instructions a third of the time.
    constexpr int kLanes = DH / 16, kStep = 32 / kLanes;  // lanes to a row, rows at a time
    const int cw = warp - kCodeWarp, ct = tid - kCodeWarp * 32, side = cw >> 1, row0 = 64 * (cw & 1);
    const int j = lane % kLanes, r0 = lane / kLanes;      // piece of a row, first row
    const int slab = j >> 2, first = 2 * (j & 3) + slab, second = 2 * (j & 3) + 1 - slab;   // (the order keeps eight lanes on eight banks)
    uint8_t* box = boxes + cw * 4 * kBox<DH>;
    int N = 0, opens = 0;                                 // chunks and open blocks so far
    bool ok = true;                                       // (a wait that ran out: on to the end, past every barrier of the four warps)
    for_each_plan(true, [&](const Plan& pl) {
      const Segment& g = pl.g;
      const int chunks = pl.chunks;
      // rows of the tile that are no codes: the open block's, those past the sequence's end, and blocks without scales or of scale zero
      auto patch = [&](int n, float mul, uint32_t spoils, uint8_t* dst) {
#pragma unroll 1
        for (int i = 0; i < 64 / kStep; ++i) {
          const int r = row0 + r0 + i * kStep, t = n * 128 + r;
          const uint32_t odd = spoils >> (16 * side + (r >> 4)) & 0x101u;
          if (t < pl.full && odd == 0) continue;
          uint4 x, y;
          x = y = make_uint4(0u, 0u, 0u, 0u);
          if (odd & 1u) x = y = make_uint4(0x7e007e00u, 0x7e007e00u, 0x7e007e00u, 0x7e007e00u);
          const int slot = t >= pl.full && t < g.len ? cache_slot(a.c, g.b, a.status) : -1;
          if (slot >= 0) {                                 // a value that is no number is left out here
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.c.open[side]) +
                                                            (((int64_t)slot * a.c.n_kv + g.kvh) * a.page + t - pl.full) * DH + 16 * j);
            const uint4 u = p[slab], v = p[1 - slab];
            uint32_t q[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              if (side == 1) {
                if ((q[k] & 0x7f80u) == 0x7f80u) q[k] &= 0xffff0000u;
                if ((q[k] & 0x7f800000u) == 0x7f800000u) q[k] &= 0xffffu;
              }
              q[k] = scaled_f16(q[k], mul);
            }
            x = make_uint4(q[0], q[1], q[2], q[3]);
            y = make_uint4(q[4], q[5], q[6], q[7]);
          }
          *reinterpret_cast<uint4*>(dst + slab * (128 * 128) + tc::sw128_offset(r, first)) = x;
          *reinterpret_cast<uint4*>(dst + slab * (128 * 128) + tc::sw128_offset(r, second)) = y;
        }
      };
      // the warp's rows of chunk N (tokens without a page: rows of page 0, which patch() passes over)
      auto request = [&](int chunk) {
        if (ok) ok = patient_warp(&ctl.rows_full[chunk & 3], (chunk >> 2) & 1, abort_flag);
        if (lane == 0) tc::mbar_arrive_expect_tx(&ctl.box_full[cw], 4 * kBox<DH>);
        __syncwarp();
        if (lane < 4) tc::tma_tile2d(box + lane * kBox<DH>, &a.map[side], &ctl.box_full[cw], 0, ctl.fac[chunk & 3].row[4 * (cw & 1) + lane]);
        __syncwarp();
      };
      if (chunks > 0) request(N);
#pragma unroll 1
      for (int n = g.blk0; n < g.blk0 + chunks; ++n, ++N) {
        const bool tail = (n + 1) * 128 > pl.full;
        float mul = 1.f;
        if (tail && g.len > pl.full) {                     // the open block: its rows' largest magnitudes, by all four warps
          const int slot = max(0, cache_slot(a.c, g.b, a.status));
          uint32_t top[2] = {0u, 0u};
          bool bad = false;
          const int pieces = (g.len - pl.full) * (DH / 8);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.c.open[s]) + ((int64_t)slot * a.c.n_kv + g.kvh) * a.page * DH);
#pragma unroll 4
            for (int i = ct; i < pieces; i += 128) {
              const uint4 u = p[i];
              const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                top[s] = largest(top[s], q[k]);
                if (s == 1) bad |= (q[k] & 0x7f80u) == 0x7f80u || (q[k] & 0x7f800000u) == 0x7f800000u;
              }
            }
            top[s] = __reduce_max_sync(0xffffffffu, top[s]);
          }
          bad = __any_sync(0xffffffffu, bad);
          if (lane == 0) {
            ctl.top[opens & 1][0][cw] = top[0];
            ctl.top[opens & 1][1][cw] = top[1] | (bad ? 0x10000u : 0u);
            tc::mbar_arrive(&ctl.open_full);               // for the warp of the scales
          }
          named_sync(3, 128);
          float kmul, vmul, inv;
          open_powers(ctl.top[opens & 1], &kmul, &inv, &vmul, &inv);
          mul = side == 0 ? kmul : vmul;
          ++opens;
        }
        const int sl = 2 * (N & 1) + side;                 // K's places and V's: free again after QK^T and after PV
        uint8_t* dst = ring + sl * kTile<DH>;
        uint8_t* at = dst + slab * (128 * 128) + row0 * 128;
        if (ok) ok = patient_warp(&ctl.box_full[cw], N & 1, abort_flag);
        if (N >= 2 && ok) ok = patient_warp(&ctl.kv_free[sl], ((N >> 1) - 1) & 1, abort_flag);
#pragma unroll 1
        for (int h = 0; h < 4; ++h) {
          uint4 w[16 / kStep];
#pragma unroll
          for (int i = 0; i < 16 / kStep; ++i) {
            const int r = (r0 + i * kStep) & 7;            // (eight rows stand like the eight before them)
            w[i] = *reinterpret_cast<const uint4*>(box + h * kBox<DH> + i * kStep / 8 * (8 * DH) +
                                                   (DH == 128 ? r * 128 + ((j ^ r) << 4) : r * 64 + ((j ^ (r >> 1)) << 4)));
          }
          if (h == 3) {
            __syncwarp();                                  // the codes have been read
            if (n + 1 < g.blk0 + chunks) request(N + 1);
          }
#pragma unroll
          for (int i = 0; i < 16 / kStep; ++i) {
            const int r = (r0 + i * kStep) & 7;
            const uint32_t w0 = slab ? w[i].z : w[i].x, w1 = slab ? w[i].w : w[i].y, w2 = slab ? w[i].x : w[i].z, w3 = slab ? w[i].y : w[i].w;
            uint8_t* to = at + h * 2048 + i * kStep / 8 * 1024 + r * 128;
            *reinterpret_cast<uint4*>(to + ((first ^ r) << 4)) =
                make_uint4(code_pair<CODE, 0>(w0), code_pair<CODE, 2>(w0), code_pair<CODE, 0>(w1), code_pair<CODE, 2>(w1));
            *reinterpret_cast<uint4*>(to + ((second ^ r) << 4)) =
                make_uint4(code_pair<CODE, 0>(w2), code_pair<CODE, 2>(w2), code_pair<CODE, 0>(w3), code_pair<CODE, 2>(w3));
          }
        }
        const uint32_t spoils = ctl.fac[N & 3].spoils;
        if (tail || spoils != 0) patch(n, mul, spoils, dst);
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.kv_full[sl]);
      }
    });
  } else if (warp >= kQkWarp) {
    regs_down<kRegsIssue>();
    if (warp == kQkWarp) {
      // ============================================ S = Q K^T ============================================
      if (lane == 0) {
        constexpr uint32_t idesc = idesc_f16(128, kNC_, false);
        const uint64_t q_desc = tc::make_desc_sw128(tc::smem_u32(q_tiles), 16, 1024), k_desc = tc::make_desc_sw128(tc::smem_u32(ring), 16, 1024);
        const uint32_t hi = (uint32_t)(k_desc >> 32), q_lo0 = (uint32_t)q_desc, k_lo0 = (uint32_t)k_desc, s_dst = tmem + kS;
        int N = 0, before = -1;                              // before: tile of the S before this one
        uint32_t done = 0, segs = 0;                         // parity of each tile's chunks and runs so far
        bool ok = true;
        for_each_plan(false, [&](const Plan& run) {
          const int chunks = run.chunks, cnt0 = run.cnt[0], cnt1 = run.cnt[1];
          for (int c = 0; c < chunks && ok; ++c, ++N) {
            const int sl = 2 * (N & 1);
            ok = patient(&ctl.kv_full[sl], (N >> 1) & 1, abort_flag);
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
              if (c >= (t == 0 ? cnt0 : cnt1) || !ok) continue;
              if (c == 0) {
                ok = patient(&ctl.q_full[t], segs >> t & 1, abort_flag);
                segs ^= 1u << t;
              }
              if (ok && before >= 0) ok = patient(&ctl.s_free[before], ~(done >> before) & 1, abort_flag);
              if (!ok) continue;
              tc::tc_fence_after();
              const uint32_t q_lo = q_lo0 + t * (kTile<DH> >> 4), k_lo = k_lo0 + sl * (kTile<DH> >> 4);
#pragma unroll
              for (int kk = 0; kk < DH / 16; ++kk) {
                const uint32_t off = ((kk >> 2) * (128 * 128) + (kk & 3) * 32) >> 4;
                if (kk == 0) tc::mma_ss_lo<false>(s_dst, q_lo + off, hi, k_lo + off, hi, idesc);
                else tc::mma_ss_lo<true>(s_dst, q_lo + off, hi, k_lo + off, hi, idesc);
              }
              tc::mma_commit(&ctl.s_full[t]);
              if (t == 1 || c >= cnt1) tc::mma_commit(&ctl.kv_free[sl]);
              before = t;
              done ^= 1u << t;
            }
          }
        });
      }
      __syncwarp();
    } else if (warp == kScaleWarp) {
      // ============================================ pages and scales ============================================
      // lane l < 8: a chunk's l-th group of 16 tokens; a chunk's loads are on their way while the one before it is published
      int N = 0, opens = 0;
      bool ok = true;
      for_each_plan(true, [&](const Plan& pl) {
        const Segment& g = pl.g;
        const int end = g.blk0 + pl.chunks;
        auto page_of = [&](int n) {
          const int t = n * 128 + 16 * (lane & 7);
          return t < pl.full && n < end ? max(0, cache_page(a.c, g.b, t >> a.page_shift, a.status)) : 0;
        };
        float vref = 0x1p-110f;
        int id1 = page_of(g.blk0), id2 = page_of(g.blk0 + 1);
        float ks1 = __ldg(a.c.scale[0] + (int64_t)id1 * a.c.n_kv + g.kvh), vs1 = __ldg(a.c.scale[1] + (int64_t)id1 * a.c.n_kv + g.kvh);
        for (int n = g.blk0; n < end; ++n, ++N) {
          const float ks2 = __ldg(a.c.scale[0] + (int64_t)id2 * a.c.n_kv + g.kvh), vs2 = __ldg(a.c.scale[1] + (int64_t)id2 * a.c.n_kv + g.kvh);
          const int id3 = page_of(n + 2), t = n * 128 + 16 * (lane & 7);
          Factors& f = ctl.fac[N & 3];
          if (N >= 4 && ok) ok = patient_warp(&ctl.fac_free[N & 3], ((N >> 2) - 1) & 1, abort_flag);
          const bool coded = t < pl.full, spoiled = coded && !(ks1 < INFINITY && vs1 < INFINITY);
          const bool zero = coded && ks1 == 0.f, nought = spoiled || (coded && vs1 == 0.f);
          const uint32_t spoils = __ballot_sync(0xffffffffu, spoiled && lane < 8) | __ballot_sync(0xffffffffu, zero && lane < 8) << 8 |
                                  __ballot_sync(0xffffffffu, nought && lane < 8) << 24;
          if (lane == 0) f.spoils = spoils;
          if (lane < 8) f.row[lane] = coded ? ((id1 * a.c.n_kv + g.kvh) << a.page_shift) + (t & (a.page - 1)) : 0;
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&ctl.rows_full[N & 3]);
          float kinv = 1.f, vinv = 0.f;
          bool odd = false;
          if ((n + 1) * 128 > pl.full && g.len > pl.full) {
            if (ok) ok = patient_warp(&ctl.open_full, opens & 1, abort_flag);
            float mul;
            odd = open_powers(ctl.top[opens & 1], &mul, &kinv, &mul, &vinv);
            ++opens;
          }
          const float k1 = coded ? (spoiled || zero ? 1.f : ks1) : t < g.len ? kinv : 1.f, v1 = coded ? (spoiled ? 0.f : vs1) : t < g.len ? vinv : 0.f;
          const float now = fmaxf(vref, __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v1))));
          // (values that are all zero: any scale.) Below 2^-60 the probabilities' sum would be lost with them; as f16 they are zeros from 2^-40 on
          const float share = v1 == 0.f ? 1.f : fmaxf(v1 / now, 0x1p-60f);
          if (lane < 8) {
            f.ks[lane] = k1;
            f.lv[lane] = log2f(128.f * share);
            f.iv[lane] = 0x1p-7f / share;
          }
          if (lane == 0) {
            f.rv = vref / now;
            f.vref = odd ? -now : now;
          }
          vref = now;
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&ctl.fac_full[N & 3]);
          id1 = id2;
          id2 = id3;
          ks1 = ks2;
          vs1 = vs2;
        }
      });
    } else if (warp == kPlanWarp) {
      // ============================================ the plan ============================================
      int s = 0;
      bool ok = true;
      auto put = [&](bool end, const Segment& g) {
        if (s >= kPlans && ok) ok = patient_warp(&ctl.plan_free[s % kPlans], (s / kPlans - 1) & 1, plan_abort);
        if (!ok) return;
        if (lane == 0) {
          Plan& p = ctl.plan[s % kPlans];
          p.end = end;
          if (!end) {
            p.g = g;
            p.rows = rows_of(a, g, kRows);
            p.full = g.len >> a.page_shift << a.page_shift;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const int last = min(p.rows, (t + 1) * 128) - 1;
              const int seen = last < t * 128 ? 0 : max(0, min(g.len, limit_of(a, g, g.tile * kRows + last)));
              p.cnt[t] = max(0, min(g.blk1, (seen + 127) >> 7) - g.blk0);
            }
            p.chunks = max(p.cnt[0], p.cnt[1]);
          }
          tc::mbar_arrive(&ctl.plan_full[s % kPlans]);
        }
        __syncwarp();
        ++s;
      };
      for_each_segment<kRows, kNC_>(a, ctl.range, [&](const Segment& g) { put(false, g); });
      put(true, Segment{});
    } else if (warp == kPvWarp) {
      // ============================================ acc += P V ============================================
      if (lane == 0) {
        constexpr uint32_t idesc = idesc_f16(128, DH, true);
        const uint64_t v_desc = tc::make_desc_sw128(tc::smem_u32(ring), kNC_ * 128, 1024);   // MN-major
        const uint32_t v_hi = (uint32_t)(v_desc >> 32), v_lo0 = (uint32_t)v_desc;
        int N = 0;
        uint32_t done = 0;
        bool ok = true;
        for_each_plan(false, [&](const Plan& run) {
          const int chunks = run.chunks, cnt0 = run.cnt[0], cnt1 = run.cnt[1];
          for (int c = 0; c < chunks && ok; ++c, ++N) {
            const int sl = 2 * (N & 1) + 1;
            ok = patient(&ctl.kv_full[sl], (N >> 1) & 1, abort_flag);
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
              if (c >= (t == 0 ? cnt0 : cnt1) || !ok) continue;
              ok = patient(&ctl.p_full[t], done >> t & 1, abort_flag);
              if (!ok) continue;
              tc::tc_fence_after();
              const uint32_t v_lo = v_lo0 + sl * (kTile<DH> >> 4), p_src = tmem + kP + t * (kNC_ / 2), acc = tmem + kAcc + t * 128;
#pragma unroll
              for (int kk = 0; kk < kNC_ / 16; ++kk)        // a run's first chunk overwrites the accumulator
                tc::mma_ts_lo(acc, p_src + kk * 8, v_lo + kk * (2048 >> 4), v_hi, idesc, (c == 0 && kk == 0) ? 0u : 1u);
              tc::mma_commit(&ctl.pv_done[t]);
              if (t == 1 || c >= cnt1) {
                tc::mma_commit(&ctl.kv_free[sl]);
                tc::mma_commit(&ctl.fac_free[N & 3]);       // (its P's were made: nobody reads the chunk's factors any more)
              }
              done ^= 1u << t;
            }
          }
        });
      }
      __syncwarp();
    }
  } else {
    // ============================================ softmax ============================================
    regs_up<kRegsSoftmax>();
    const int t = warp >> 2, gt = tid & 127, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + kS, p_addr = tmem + lane_base + kP + t * (kNC_ / 2), acc_addr = tmem + lane_base + kAcc + t * 128;
    uint8_t* stage = q_tiles + t * kTile<DH>;
    int N = 0, done = 0;
    bool ok = true;
    for_each_plan(true, [&](const Plan& run) {
      const Segment& g = run.g;
      const int n_rows = min(128, run.rows - t * 128), cnt = run.cnt[t];
      const int pr = g.tile * kRows + t * 128 + row;        // row of the problem's rows
      const bool row_ok = row < n_rows;
      const int limit = row_ok ? limit_of(a, g, pr) : 0;
      float ell = 0.f, ref = -INFINITY, c2 = 0.f, vref = 1.f;
      if (cnt > 0) {
        // Q: the thread's row, brought into f16's range by a power of two
        uint32_t top = 0;
        const uint4* src = nullptr;
        if (row_ok) {
          const int i = pr / a.group;
          src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (int64_t)(g.s + i) * a.q_stride +
                                               (int64_t)(g.kvh * a.group + pr - i * a.group) * DH);
        }
        uint4 x[DH / 8];
#pragma unroll
        for (int c = 0; c < DH / 8; ++c) {
          x[c] = row_ok ? __ldg(src + c) : make_uint4(0u, 0u, 0u, 0u);
          top = largest(largest(largest(largest(top, x[c].x), x[c].y), x[c].z), x[c].w);
        }
        float mul, inv;
        to_power(top, 14, &mul, &inv);
        c2 = a.scale_log2 * inv;
#pragma unroll
        for (int c = 0; c < DH / 8; ++c)
          *reinterpret_cast<uint4*>(stage + (c >> 3) * (128 * 128) + tc::sw128_offset(row, c & 7)) =
              make_uint4(scaled_f16(x[c].x, mul), scaled_f16(x[c].y, mul), scaled_f16(x[c].z, mul), scaled_f16(x[c].w, mul));
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.q_full[t]);
      }
      for (int c = 0; c < cnt && ok; ++c) {
        const int t0 = (g.blk0 + c) * 128, F = (N + c) & 3;
        if (!warp_wait(&ctl.s_full[t], done & 1, abort_flag) || !warp_wait(&ctl.fac_full[F], ((N + c) >> 2) & 1, abort_flag)) { ok = false; break; }
        tc::tc_fence_after();
        uint32_t r[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tc::tmem_ld32(s_addr + q * 32, r[q]);
        tc::tmem_wait_ld();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.s_free[t]);
        // the keys that a row sees are a prefix of the chunk
        const Factors& fc = ctl.fac[F];
        const int vis = limit - t0;
        if (!__all_sync(0xffffffffu, vis >= 128)) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int u = 0; u < 32; ++u) r[q][u] = q * 32 + u < vis ? r[q][u] : 0xff800000u;
        }
        float cm = max_block<FINE>(r[0], fc, 0, c2);
#pragma unroll
        for (int q = 1; q < 4; ++q) cm = fmaxf(cm, max_block<FINE>(r[q], fc, q, c2));
        const float rv = fc.rv;
        const bool over = cm > -INFINITY && !(cm - ref <= kMove);
        const bool any_over = __any_sync(0xffffffffu, over) || rv != 1.f;
        const float old_ref = ref;
        if (over) ref = fmaxf(ref, cm);
        const float sub = ref == -INFINITY ? 0.f : ref;
        // half of the columns at a time, by one piece of code (see there: the warps of codes)
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          uint32_t p0[16], p1[16];
          const float sum0 = exp_block<FINE>(r[0], fc, 2 * h, c2, sub, p0), sum1 = exp_block<FINE>(r[1], fc, 2 * h + 1, c2, sub, p1);
          if (h == 0) {
            // the P before this one must have been read, and with it every earlier PV has completed
            if (c > 0 && ok) ok = warp_wait(&ctl.pv_done[t], (done - 1) & 1, abort_flag);
            tc::tc_fence_after();
            if (any_over) {
              const float factor = over ? tc::ex2(old_ref - ref) : 1.f, af = factor * rv;
              ell *= factor;
#pragma unroll 1
              for (int q = 0; q < DH / 16 && c > 0; ++q) {
                uint32_t acc[16];
                tc::tmem_ld16(acc_addr + q * 16, acc);
                tc::tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] = __float_as_uint(__uint_as_float(acc[i]) * af);
                tc::tmem_st16(acc_addr + q * 16, acc);
              }
            }
          }
          tc::tmem_st16(p_addr + 32 * h, p0);
          tc::tmem_st16(p_addr + 32 * h + 16, p1);
          ell += sum0 + sum1;
#pragma unroll
          for (int u = 0; u < 32; ++u) {
            r[0][u] = r[2][u];
            r[1][u] = r[3][u];
          }
        }
        vref = fc.vref;
        tc::tmem_wait_st();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.p_full[t]);
        ++done;
      }
      N += run.chunks;
      // ---- the run's result: O = acc vref 2^-7 / l, or the accumulator, its reference and its sum as a part of the problem's -------
      const int full = run.full;
      const bool whole = g.whole();
      if (cnt > 0 && ok) ok = warp_wait(&ctl.pv_done[t], (done - 1) & 1, abort_flag);
      tc::tc_fence_after();
      float* part = a.part + (int64_t)part_slot(blockIdx.x, g.first) * kRows * (DH + 2);
      const float unit = fabsf(vref) * 0x1p-7f;
      auto weight = [](float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; };
      // 16 dims from c0 on of the thread's row
      auto mine = [&](int c0, float (&v)[16]) {
        uint32_t av[16];
        if (cnt > 0) {
          tc::tmem_ld16(acc_addr + c0, av);
          tc::tmem_wait_ld();
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = cnt > 0 ? __uint_as_float(av[i]) * unit : 0.f;
        if (vref < 0.f && row_ok) {                                // values that are no numbers, for the rows that see them
          const int slot = cache_slot(a.c, g.b, a.status);
          const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(a.c.open[1]) + ((int64_t)max(slot, 0) * a.c.n_kv + g.kvh) * a.page * DH + c0;
          const int end = min(limit, min(g.blk1 * 128, g.len));
          for (int k = max(full, g.blk0 * 128); k < end; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float z = __bfloat162float(p[(int64_t)(k - full) * DH + i]);
              if (!(fabsf(z) < INFINITY)) v[i] += z;
            }
        }
      };
      auto emit = [&](auto source, float l, float top) {
        const float w = weight(l);
        named_sync(1 + t, 128);                             // every QK^T has retired, Q's place is free
#pragma unroll 1
        for (int c0 = 0; c0 < DH; c0 += 16) {
          float v[16];
          source(c0, v);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float pv[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) pv[i] = w * v[q * 8 + i];
            *reinterpret_cast<uint4*>(stage + row * (2 * DH) + (((c0 / 8 + q) ^ (row & 7)) << 4)) = pack8(pv);
          }
        }
        if (row_ok && a.lse != nullptr && ok) a.lse[out_row(a, g, pr)] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
        named_sync(1 + t, 128);
        if (ok)
#pragma unroll 4
          for (int k = 0; k < DH / 8; ++k) {
            const int idx = k * 128 + gt, rr = idx / (DH / 8), cc = idx % (DH / 8);
            if (rr < n_rows)
              *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o) + out_row(a, g, g.tile * kRows + t * 128 + rr) * DH + cc * 8) =
                  *reinterpret_cast<const uint4*>(stage + rr * (2 * DH) + ((cc ^ (rr & 7)) << 4));
          }
        named_sync(1 + t, 128);                             // the next run's Q comes here
      };
      if (whole) {
        if (n_rows > 0) emit(mine, ell, ref);
        return;
      }
      // parts: [dims / 4][rows] of four, so that a warp's rows stand side by side; then (reference, sum)
      float4* po = reinterpret_cast<float4*>(part);
      float2* ps = reinterpret_cast<float2*>(part + kRows * DH);
      if (n_rows > 0) {
#pragma unroll 1
        for (int c0 = 0; c0 < DH; c0 += 16) {
          float v[16];
          mine(c0, v);
          if (row_ok) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              __stcg(po + (c0 / 4 + q) * kRows + t * 128 + row, make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]));
          }
        }
        if (row_ok) __stcg(ps + t * 128 + row, make_float2(ref, ell));
      }
    });
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == kQkWarp) {
    if (ctl.abort_flag) {
      if (lane == 0) tc::mma_commit(&ctl.pv_done[0]);
      __syncwarp();
      for (int it = 0; it < (1 << 16); ++it) __nanosleep(256);
    }
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
  if (tid == 0 && (ctl.abort_flag || ctl.plan_abort) && a.status != nullptr) atomicExch(a.status, (int)FL_ERR_TIMEOUT);
}

// The problems that the borders of the runs cut: block x has the one that begins in CTA x's run and goes on after it, if there is one; of it
// 32 rows (y), a lane's row and a warp's 32 dims. The parts are added in their order.
template <int DH>
__global__ void __launch_bounds__(DH) cache_join_kernel(const __grid_constant__ AttnArgs a) {
  __shared__ Range range;
  fl_grid_wait();
  fl_grid_release();
  const int lane = threadIdx.x & 31, c0 = (threadIdx.x >> 5) * 32, row = blockIdx.y * 32 + lane;
  if (threadIdx.x < 32) {
    const Range r = find_range<kRows, kNC_>(a, lane);
    if (lane == 0) range = r;
  }
  __syncthreads();
  for_each_segment<kRows, kNC_>(a, range, [&](const Segment& g) {
    if (g.whole() || g.first != (int)blockIdx.x || row >= rows_of(a, g, kRows)) return;
    auto part_of = [&](int c) { return a.part + (int64_t)part_slot(min(c, g.last), g.first) * kRows * (DH + 2); };
    float v[32], top = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = 0.f;
    for (int c = g.first; c <= g.last; c += 2) {
      float4 f[2][8];
      float2 m[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        m[k] = __ldcg(reinterpret_cast<const float2*>(part_of(c + k) + kRows * DH) + row);
        const float4* p = reinterpret_cast<const float4*>(part_of(c + k)) + (c0 / 4) * kRows + row;
#pragma unroll
        for (int q = 0; q < 8; ++q) f[k][q] = __ldcg(p + q * kRows);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (c + k > g.last) break;
        const float to = fmaxf(top, m[k].x), old = part_weight(top, to), w = part_weight(m[k].x, to);
        top = to;
        l = l * old + w * m[k].y;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          v[4 * q] = v[4 * q] * old + w * f[k][q].x;
          v[4 * q + 1] = v[4 * q + 1] * old + w * f[k][q].y;
          v[4 * q + 2] = v[4 * q + 2] * old + w * f[k][q].z;
          v[4 * q + 3] = v[4 * q + 3] * old + w * f[k][q].w;
        }
      }
    }
    const float w = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    const int64_t at = out_row(a, g, g.tile * kRows + row);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = v[8 * q + i] * w;
      *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o) + at * DH + c0 + 8 * q) = pack8(x);
    }
    if (c0 == 0 && a.lse != nullptr) a.lse[at] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
  });
}

template <int DH, int CODE, bool FINE>
int launch(fl_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  auto kern = cache_flash_kernel<DH, CODE, FINE>;
  if ((size_t)ctx->max_smem_optin < kSmemTc<DH>) return FL_ERR_UNSUPPORTED;
  FL_FUNC_ATTR_ONCE(ctx, kern, (kSmemTc<DH>), true);
  // the warpgroups' shares are taken from what the block is launched with: with fewer registers than counted on, one would wait for ever
  static const int regs = [] {
    cudaFuncAttributes f;
    return cudaFuncGetAttributes(&f, cache_flash_kernel<DH, CODE, FINE>) == cudaSuccess ? f.numRegs : 0;
  }();
  if (4 * regs < 2 * kRegsSoftmax + kRegsIssue + kRegsCodes) return FL_ERR_CUDA;
  FL_CHECK_CUDA(fl_launch(ctx, kern, dim3((unsigned)ctx->sm_count), dim3(kThreadsTc), kSmemTc<DH>, st, a));
  FL_CHECK_CUDA(fl_launch(ctx, cache_join_kernel<DH>, dim3((unsigned)ctx->sm_count, kRows / 32), dim3(DH), 0, st, a));
  return fl_launch_status();
}
template <int DH, int CODE>
int launch_page(fl_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  return a.page == 16 ? launch<DH, CODE, true>(ctx, a, st) : launch<DH, CODE, false>(ctx, a, st);
}

}  // namespace

int64_t fl_cache_attn_tc_part_bytes(const fl_ctx* ctx, int head_dim) { return (int64_t)ctx->sm_count * 2 * kRows * (head_dim + 2) * 4; }

int fl_launch_cache_attn_tc(fl_ctx* ctx, const AttnArgs& args, int head_dim, int code, cudaStream_t st) {
  AttnArgs a = args;
  // (a problem's Q, first chunk and result count as four chunks, two are worth a CTA; with one for the ends the times above are the same)
  a.min_units = 2;
  a.head_units = 4;
  a.max_parts = 16;
  if (head_dim == 128) return code == FL_INT8 ? launch_page<128, FL_INT8>(ctx, a, st) : launch_page<128, FL_E4M3>(ctx, a, st);
  return code == FL_INT8 ? launch_page<64, FL_INT8>(ctx, a, st) : launch_page<64, FL_E4M3>(ctx, a, st);
}
