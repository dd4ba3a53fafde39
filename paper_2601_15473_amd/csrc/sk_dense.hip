// What stands around a dense layer's products: the second launch of a forward product that was split over its contraction, and dz = dy act'(z) with the bias's gradient ahead
// of the two backward ones,  dx = dz W,  dW = dz^T x.
//
// Bound by memory.  dz of 4096 x 4096 behind gelu 19 us for 101 MB (5.3 TB/s; level for two to eight rows ahead and three to eight work-groups a CU), 16384 x 11008 behind silu 228 to 257 us for
// 1.08 GB; the runs' sums 2 to 5 us, a launch.  In bf16 z comes back rounded (the derivative at z off by 2^-8 z act''(z): 0.0006 of dz, where dz's own rounding, as an operand of both products, is 0.0017; z in
// fp32 would be twice the bytes here and in the forward pass), and the bias's sums are of dz before its rounding.
//
// Tried and slower: the bias's gradient on the weight's product, whose operand dz is, as MFMAs against ones (46 us for 36) or on the vector unit (48), where without an activation
// its two launches here take 8 ([4001 x 1024]^T . [4001 x 4096]); dx beside dW in one launch on staged 128 x 128 tiles (84 for 38 + 37, 4096 tokens, 1024 -> 4096).
#include "sk_activation.h"
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

// y = act(z) + residual with z the sum of the product's fp32 slabs, in order, and the bias; z itself, rounded, where a backward pass wants it.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void dense_finish_kernel(const DenseArgs p) {
  const int pieces = p.out / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id / pieces;
  const int at = (int)(id - row * pieces) * 8;
  if (row >= p.tokens) return;
  const int64_t n = (int64_t)p.tokens * p.out;
  const float* const slab = p.slabs + row * p.out + at;
  float4 sum[2];
  const float* const both[2] = {slab, slab + 4};
  sum_slabs<2>(sum, both, n, p.splits);
  float z[8] = {sum[0].x, sum[0].y, sum[0].z, sum[0].w, sum[1].x, sum[1].y, sum[1].z, sum[1].w}, add[8];
  if (p.bias) {
    load_values<T, 8>(add, static_cast<const T*>(p.bias) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] += add[i];
  }
  if (ACT != ACT_NONE && p.z) store_values<T, 8>(static_cast<T*>(p.z) + row * p.out + at, z);
#pragma unroll
  for (int i = 0; i < 8; ++i) { z[i] = activation<ACT, sizeof(T) == 4>(z[i]); add[i] = 0.f; }
  if (p.residual) load_values<T, 8>(add, static_cast<const T*>(p.residual) + row * p.residual_stride + at);
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] += add[i];
  store_values<T, 8>(static_cast<T*>(p.y) + row * p.out + at, z);
}

// dz = dy act'(z) and its column sums: a work-group has 512 columns (eight a lane) of a run of rows, its four waves every fourth row each, their sums
// joined in the waves' order.  Without an activation dz is dy, and only the sums are formed.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void dense_dz_kernel(const DenseArgs p, int rows_per_run) {
  constexpr int AHEAD = 4;
  __shared__ float part[4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = blockIdx.x * 512 + lane * 8;
  const int64_t begin = (int64_t)blockIdx.y * rows_per_run, end = begin + rows_per_run < p.tokens ? begin + rows_per_run : p.tokens;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (at < p.out) {
    for (int64_t row = begin + wave; row < end; row += 4 * AHEAD) {
      float d[AHEAD][8], z[AHEAD][8];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {   // (past the run: its last row again, for nothing)
        const int64_t r = row + 4 * a < end ? row + 4 * a : end - 1;
        load_values<T, 8>(d[a], static_cast<const T*>(p.dy) + r * p.out + at);
        if constexpr (ACT != ACT_NONE) load_values<T, 8>(z[a], static_cast<const T*>(p.z) + r * p.out + at);
      }
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        const int64_t r = row + 4 * a;
        if (r >= end) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (ACT != ACT_NONE) d[a][i] *= activation_slope<ACT, sizeof(T) == 4>(z[a][i]);
          sum[i] += d[a][i];
        }
        if constexpr (ACT != ACT_NONE) store_values<T, 8>(static_cast<T*>(p.dz) + r * p.out + at, d[a]);
      }
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += 256)
    if (blockIdx.x * 512 + c < p.out) p.partial[(int64_t)blockIdx.y * p.out + blockIdx.x * 512 + c] = ((part[0][c] + part[1][c]) + part[2][c]) + part[3][c];
}

// The runs' sums added up: 32 columns a work-group, runs dealt over 32 threads a column and joined in order.
template <typename T>
__global__ __launch_bounds__(1024) void dense_dbias_kernel(const float* __restrict__ partial, T* __restrict__ dbias, int columns, int runs) {
  __shared__ float sums[32][33];
  const int c = threadIdx.x & 31, part = threadIdx.x >> 5, column = blockIdx.x * 32 + c;
  float s = 0.f;
  if (column < columns)
#pragma unroll 4
    for (int g = part; g < runs; g += 32) s += partial[(int64_t)g * columns + column];
  sums[part][c] = s;
  __syncthreads();
  if (part == 0 && column < columns) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][c];
    store_one(dbias + column, s);
  }
}

template <typename F>
hipError_t by_activation(int act, F&& f) {
  switch (act) {
    case ACT_NONE: return f(IntC<ACT_NONE>{});
    case ACT_RELU: return f(IntC<ACT_RELU>{});
    case ACT_GELU: return f(IntC<ACT_GELU>{});
    case ACT_GELU_TANH: return f(IntC<ACT_GELU_TANH>{});
    case ACT_SILU: return f(IntC<ACT_SILU>{});
    default: return hipErrorInvalidValue;
  }
}

template <typename T>
hipError_t finish(const DenseArgs& a, hipStream_t s) {
  note_matrix(a.slabs, (int64_t)a.splits * a.tokens, a.out, a.out, 4, false);
  note_matrix(a.bias, 1, a.out, a.out, sizeof(T), false);
  if (a.activation != ACT_NONE) note_matrix(a.z, a.tokens, a.out, a.out, sizeof(T), true);
  if (a.residual) note_matrix(a.residual, a.tokens, a.out, a.residual_stride, sizeof(T), false);
  note_matrix(a.y, a.tokens, a.out, a.out, sizeof(T), true);
  const int64_t groups = ((int64_t)a.tokens * (a.out / 8) + 255) / 256;
  return by_activation(a.activation, [&](auto act) {
    return launch_kernel("dense_finish_kernel", Work{0.0, (4.0 * a.splits + 3.0 * sizeof(T)) * a.tokens * a.out}, dense_finish_kernel<T, decltype(act)::value>, dim3((unsigned)groups), dim3(256), s, a);
  });
}

template <typename T>
hipError_t dz(const DenseArgs& a, hipStream_t s) {
  const bool act = a.activation != ACT_NONE;
  if (!act && !a.partial) return hipSuccess;
  const ColumnRuns r(a.tokens, a.out);
  note_matrix(a.dy, a.tokens, a.out, a.out, sizeof(T), false);
  if (act) {
    note_matrix(a.z, a.tokens, a.out, a.out, sizeof(T), false);
    note_matrix(a.dz, a.tokens, a.out, a.out, sizeof(T), true);
  }
  note_matrix(a.partial, r.runs, a.out, a.out, 4, true);
  return by_activation(a.activation, [&](auto t) {
    return launch_kernel("dense_dz_kernel", Work{0.0, (act ? 3.0 : 1.0) * a.tokens * a.out * sizeof(T)}, dense_dz_kernel<T, decltype(t)::value>,
                         dim3((unsigned)r.groups, (unsigned)r.runs), dim3(256), s, a, r.rows);
  });
}

template <typename T>
hipError_t dbias(const DenseArgs& a, hipStream_t s) {
  if (!a.partial) return hipSuccess;
  const ColumnRuns r(a.tokens, a.out);
  note_matrix(a.partial, r.runs, a.out, a.out, 4, false);
  note_matrix(a.dbias, 1, a.out, a.out, sizeof(T), true);
  return launch_kernel("dense_dbias_kernel", Work{0.0, 4.0 * r.runs * a.out}, dense_dbias_kernel<T>, dim3((unsigned)((a.out + 31) / 32)), dim3(1024), s,
                       static_cast<const float*>(a.partial), static_cast<T*>(a.dbias), a.out, r.runs);
}

}  // namespace

hipError_t launch_dense_finish(const DenseArgs& a, bool f32, hipStream_t s) { return f32 ? finish<float>(a, s) : finish<bf16>(a, s); }
hipError_t launch_dense_dz(const DenseArgs& a, bool f32, hipStream_t s) { return f32 ? dz<float>(a, s) : dz<bf16>(a, s); }
hipError_t launch_dense_dbias(const DenseArgs& a, bool f32, hipStream_t s) { return f32 ? dbias<float>(a, s) : dbias<bf16>(a, s); }

}  // namespace sk
