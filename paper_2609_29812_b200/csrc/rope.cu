// Rotary positions: the table of cosines and sines, and the rotation of the rows of a projection.
#include "rope.cuh"

#include <cmath>

namespace {

struct Freqs {
  double f[64];   // turns per position of each pair
};

// The angle in turns keeps its fraction in binary64 (a position of 2^24 costs 24 of 53 bits); sincospi is exact in its reduction.
// Bound by binary64 arithmetic: 32768 positions x 64 pairs 20 us, 131072 67 (writing them takes 10). A program makes its table once.
__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ Freqs fr, int half, double magnitude, int64_t n, float2* table) {
  fl_grid_wait();
  fl_grid_release();
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t p = i / half;
    const double t = (double)p * fr.f[i - p * half];
    double s, c;
    sincospi(2.0 * (t - rint(t)), &s, &c);
    table[i] = make_float2((float)(magnitude * c), (float)(magnitude * s));
  }
}

struct RotArgs {
  const void* x;
  void* y;
  int64_t x_stride, y_stride;
  const int32_t* pos;
  int pos0, n, n_heads, head_dim;
  RopeArgs rope;
  float sign;
  int32_t* status;
};

// The row of the table for token t; a position outside the table is reported and its row not followed.
__device__ __forceinline__ const float* table_row(const RotArgs& a, int t) {
  int p = a.pos != nullptr ? __ldg(a.pos + t) : a.pos0 + t;
  if ((unsigned)p >= (unsigned)a.rope.n_pos) {
    if (a.status != nullptr) atomicExch(a.status, (int)FL_ERR_INVALID_ARG);
    p = 0;
  }
  return a.rope.table + (int64_t)p * a.rope.rot_dim;
}

// A thread has 16 elements, 8 pairs, of HPT heads of a token, all their loads in flight at once; the (cos, sin) of its pairs serve
// all of them. Bound by HBM, each element read and written once: the rows of a 32768-token prompt of 16 heads 44 us = 6.3 TB/s, in binary32 105
// = 5.2 TB/s (100 registers a thread, two CTAs an SM where bf16 has four).
template <typename T, int MODE, int HPT>
__global__ void __launch_bounds__(256) rotate_rows_kernel(const __grid_constant__ RotArgs a) {
  fl_grid_wait();
  fl_grid_release();
  const int shift = a.head_dim == 128 ? 3 : 2, items = 1 << shift;        // items per head
  const int groups = (a.n_heads + HPT - 1) / HPT;
  const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int j = (int)id & (items - 1);
  const int64_t r = id >> shift;
  const int t = (int)(r / groups), h0 = (int)(r - (int64_t)t * groups) * HPT;
  if (t >= a.n) return;
  const RopeItem it = rope_item<MODE>(j, a.rope.rot_dim);
  const T* x = static_cast<const T*>(a.x) + (int64_t)t * a.x_stride + (int64_t)h0 * a.head_dim;
  T* y = static_cast<T*>(a.y) + (int64_t)t * a.y_stride + (int64_t)h0 * a.head_dim;
  Piece<T> u[HPT], v[HPT];                                                // as they are stored: half the registers that numbers take
#pragma unroll
  for (int k = 0; k < HPT; ++k)
    if (HPT == 1 || h0 + k < a.n_heads) {
      get_piece(u[k], x + k * a.head_dim + it.a);
      get_piece(v[k], x + k * a.head_dim + it.b);
    }
  float c[8], s[8];
  if (it.turns) rope_load(table_row(a, t), j, a.sign, c, s);
#pragma unroll
  for (int k = 0; k < HPT; ++k)
    if (HPT == 1 || h0 + k < a.n_heads) {
      if (it.turns) {
        float f[8], g[8];
        open_piece(u[k], f);
        open_piece(v[k], g);
        rope_apply<MODE>(f, g, c, s);
        close_piece(u[k], f);
        close_piece(v[k], g);
      }
      put_piece(y + k * a.head_dim + it.a, u[k]);
      put_piece(y + k * a.head_dim + it.b, v[k]);
    }
}

// Any even rot_dim, any alignment: a thread has one pair, or one element that stays; the same rows with 20 or 50 elements turned take 263, 249
// us (floor 42): single elements to and fro, and two divisions for each.
template <typename T>
__global__ void __launch_bounds__(256) rotate_rows_any_kernel(const __grid_constant__ RotArgs a) {
  fl_grid_wait();
  fl_grid_release();
  const int half = a.rope.rot_dim >> 1, per_head = a.head_dim - half;
  const int64_t n = (int64_t)a.n * a.n_heads * per_head;
  for (int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; id < n; id += (int64_t)gridDim.x * blockDim.x) {
    const int64_t r = id / per_head;
    const int e = (int)(id - r * per_head), t = (int)(r / a.n_heads), h = (int)(r - (int64_t)t * a.n_heads);
    const T* x = static_cast<const T*>(a.x) + (int64_t)t * a.x_stride + (int64_t)h * a.head_dim;
    T* y = static_cast<T*>(a.y) + (int64_t)t * a.y_stride + (int64_t)h * a.head_dim;
    if (e < half) {
      const float* row = table_row(a, t);
      const int i0 = a.rope.layout == FL_ROPE_HALF ? e : 2 * e, i1 = a.rope.layout == FL_ROPE_HALF ? e + half : 2 * e + 1;
      float u = load1(x + i0), v = load1(x + i1);
      rope_pair(u, v, row[2 * e], a.sign * row[2 * e + 1]);
      store1(y + i0, u);
      store1(y + i1, v);
    } else {
      y[e + half] = x[e + half];
    }
  }
}

template <typename T, int MODE>
int launch_rotate(fl_ctx* ctx, const RotArgs& a, cudaStream_t st) {
  // Four heads per thread share its (cos, sin), and quarter the table's traffic; one head per thread where that would leave SMs short
  // of threads.
  const int64_t threads = (int64_t)a.n * (a.head_dim / 16);
  const bool four = threads * ((a.n_heads + 3) / 4) >= (int64_t)ctx->sm_count * 1024;
  const int64_t total = threads * (four ? (a.n_heads + 3) / 4 : a.n_heads), blocks = (total + 255) / 256;
  FL_REQUIRE(blocks <= INT32_MAX);
  FL_CHECK_CUDA(fl_launch(ctx, four ? rotate_rows_kernel<T, MODE, 4> : rotate_rows_kernel<T, MODE, 1>, dim3((unsigned)blocks), dim3(256), 0, st, a));
  return fl_launch_status();
}

template <typename T>
int rotate(fl_ctx* ctx, const RotArgs& a, int mode, cudaStream_t st) {
  const int64_t piece = 16 / (int64_t)sizeof(T);
  if (mode == kRopeAny || !fl_aligned16(a.x) || !fl_aligned16(a.y) || a.x_stride % piece != 0 || a.y_stride % piece != 0) {
    const int64_t n = (int64_t)a.n * a.n_heads * (a.head_dim - a.rope.rot_dim / 2), most = (int64_t)ctx->sm_count * 64;
    const int64_t blocks = (n + 255) / 256;
    FL_CHECK_CUDA(fl_launch(ctx, rotate_rows_any_kernel<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a));
    return fl_launch_status();
  }
  return mode == kRopeHalf ? launch_rotate<T, kRopeHalf>(ctx, a, st) : launch_rotate<T, kRopePairs>(ctx, a, st);
}

}  // namespace

extern "C" int fl_rope_table(fl_ctx* ctx, const fl_rope_spec* spec, float* table, int32_t n_pos, void* stream) {
  FL_REQUIRE(ctx != nullptr && spec != nullptr && table != nullptr && fl_aligned16(table));
  FL_REQUIRE(n_pos >= 1);
  const int rot = spec->rot_dim;
  FL_REQUIRE(rot >= 2 && rot % 2 == 0 && rot <= 128);
  FL_REQUIRE(spec->base > 1.0 && std::isfinite(spec->base));
  FL_REQUIRE(spec->kind >= FL_ROPE_PLAIN && spec->kind <= FL_ROPE_YARN);
  if (spec->kind != FL_ROPE_PLAIN) FL_REQUIRE(spec->factor >= 1.0 && std::isfinite(spec->factor));
  const double pi = 3.14159265358979323846;
  double base = spec->base, lo = 0.0, hi = 0.0, magnitude = 1.0;
  if (spec->kind == FL_ROPE_NTK) {
    FL_REQUIRE(rot > 2);
    base *= std::pow(spec->factor, rot / (rot - 2.0));
  }
  if (spec->kind == FL_ROPE_YARN) {
    FL_REQUIRE(spec->slow > 0.0 && spec->fast > spec->slow && std::isfinite(spec->fast) && spec->trained >= 1);
    // the pair that turns t times within the trained positions
    auto pair_of = [&](double t) { return rot * std::log(spec->trained / (2 * pi * t)) / (2 * std::log(spec->base)); };
    lo = std::fmax(0.0, std::floor(pair_of(spec->fast)));
    hi = std::fmin(rot - 1.0, std::ceil(pair_of(spec->slow)));
    magnitude = 0.1 * std::log(spec->factor) + 1.0;
  }
  Freqs fr;
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot);
    if (spec->kind == FL_ROPE_LINEAR) f /= spec->factor;
    if (spec->kind == FL_ROPE_YARN) {
      const double g = std::fmin(1.0, std::fmax(0.0, (i - lo) / std::fmax(hi - lo, 1e-3)));
      f = f * (1.0 - g) + f / spec->factor * g;
    }
    fr.f[i] = f / (2 * pi);
  }
  const int64_t n = (int64_t)n_pos * (rot / 2), blocks = (n + 255) / 256, most = (int64_t)ctx->sm_count * 32;
  FL_CHECK_CUDA(fl_launch(ctx, rope_table_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0,
                          static_cast<cudaStream_t>(stream), fr, rot / 2, magnitude, n, reinterpret_cast<float2*>(table)));
  return fl_launch_status();
}

extern "C" int fl_rotate_rows(fl_ctx* ctx, const void* x, int64_t x_stride, const int32_t* pos, int32_t pos0, int32_t n, int32_t n_heads,
                              int32_t head_dim, int32_t dtype, const fl_rope* rope, int32_t inverse, void* y, int64_t y_stride,
                              int32_t* status, void* stream) {
  FL_REQUIRE(ctx != nullptr && rope != nullptr);
  FL_REQUIRE(n >= 0 && n_heads >= 1 && head_dim >= 1);
  FL_REQUIRE(dtype == FL_BF16 || dtype == FL_F32);
  if (head_dim != 64 && head_dim != 128) return FL_ERR_UNSUPPORTED;
  const int rc = fl_check_rope(rope, head_dim);
  if (rc != FL_OK) return rc;
  FL_REQUIRE(x_stride >= (int64_t)n_heads * head_dim && y_stride >= (int64_t)n_heads * head_dim);
  FL_REQUIRE(pos != nullptr || (pos0 >= 0 && (int64_t)pos0 + n <= rope->n_pos));
  if (n == 0) return FL_OK;
  FL_REQUIRE(x != nullptr && y != nullptr);
  FL_REQUIRE(x != y || x_stride == y_stride);
  const uintptr_t es = dtype == FL_BF16 ? 2 : 4;
  FL_REQUIRE(reinterpret_cast<uintptr_t>(x) % es == 0 && reinterpret_cast<uintptr_t>(y) % es == 0);
  const RotArgs a = {x, y, x_stride, y_stride, pos, pos0, n, n_heads, head_dim, {rope->table, rope->n_pos, rope->rot_dim, rope->layout},
                     inverse ? -1.f : 1.f, status};
  const int mode = fl_rope_mode(rope);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == FL_BF16 ? rotate<__nv_bfloat16>(ctx, a, mode, st) : rotate<float>(ctx, a, mode, st);
}
