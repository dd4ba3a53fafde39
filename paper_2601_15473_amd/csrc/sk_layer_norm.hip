// Layer norm of rows, with a residual added first, and its gradients.
//
//   s = x + residual,  mu = mean s,  r = 1 / sqrt(mean (s - mu)^2 + eps),  u = (s - mu) r,  y = u w + b
//   g = dy w,  dx = ds + r (g - mean g - u mean(g u)),  dw = sum dy u,  db = sum dy
//
// Bound by memory: a row is read once into registers, eight values to a lane and piece, and both of its sums are taken there (the mean first, the
// squares about it second: a stream whose mean is large beside its spread loses nothing).  y is formed of the sum before s is rounded, and so are the gradients of the weights: s as it was
// stored, off by up to 2^-9 of it, would make dw 0.0024 to 0.0027 off 64 bits where one rounding of an exact result is 0.0017.  Four bits more a value, a quarter of a tensor each way, leave
// 2^-12 of it (s in fp32 would be a whole one).
// Bf16, 16383 rows of 4096 with a residual: forward 94 us for 570 MB (6.1 TB/s; a copy reaches 5.1), back 120 us for 570 MB (4.8) and 5 for the sum of the partial
// sums, of which the four bits are 6 and 8; 4096 rows of 768 8.1, 9.4 and 3.7.  What carried it: every load of a row ahead of its first sum, the weights' among them (forward 99 -> 93, eight rows of 8192 6.4 -> 4.5), and the
// next row's loads under this one's sums (back 180 -> 112).
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

constexpr int PIECE = 8;   // values

// What a piece's rounding to bf16 left off, in 16ths of a step, four bits a value (the far half of a step is 8 of them: one less).  On the numbers' bits: a step
// of the magnitude is one of the bits, across powers of two too, so that the fp32 bits less the rounded ones are what was left, and adding them gives it back.
__device__ __forceinline__ unsigned rest_of(const float (&v)[PIECE]) {
  unsigned rest = 0;
#pragma unroll
  for (int i = 0; i < PIECE; i += 2) {
    const unsigned rounded = pack_bf16x2(v[i], v[i + 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int left = (int)(__builtin_bit_cast(unsigned, v[i + h]) - (h ? rounded & 0xffff0000u : rounded << 16));
      const int q = (left + 0x800) >> 12;
      rest |= (unsigned)((q < -8 ? -8 : q > 7 ? 7 : q) & 15) << (4 * (i + h));
    }
  }
  return rest;
}
__device__ __forceinline__ void add_rest(float (&v)[PIECE], unsigned rest) {
#pragma unroll
  for (int i = 0; i < PIECE; ++i)
    v[i] = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v[i]) + ((unsigned)((int)(rest << (28 - 4 * i)) >> 28) << 12));
}

// The sum of a row's lanes, L of a wave or all of a work-group's (`shared`: a float a wave, another place for each sum).  Every lane gets it.
template <int L>
__device__ __forceinline__ float sum_row(float v, float* shared) {
#pragma unroll
  for (int m = 1; m < (L < 64 ? L : 64); m <<= 1) v += __shfl_xor(v, m);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < L / 64; ++w) v += shared[w];
  }
  return v;
}

// A row's pieces as they lie in memory, for loads that are not waited for yet.
template <typename T, int N>
struct Raw {
  uint4 v[N][sizeof(T) / 2];
  template <int L>
  __device__ __forceinline__ void load(const T* row, int lane, int width) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = (n * L + lane) * PIECE;
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h) v[n][h] = at < width ? reinterpret_cast<const uint4*>(row + at)[h] : make_uint4(0u, 0u, 0u, 0u);
    }
  }
  __device__ __forceinline__ void values(float (&f)[PIECE], int n) const {
    const unsigned u[4] = {v[n][0].x, v[n][0].y, v[n][0].z, v[n][0].w};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __builtin_bit_cast(float, u[i] << 16);
        f[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
      }
    } else {
      const uint4 w = v[n][sizeof(T) / 2 - 1];
      const unsigned x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = __builtin_bit_cast(float, u[i]);
        f[4 + i] = __builtin_bit_cast(float, x[i]);
      }
    }
  }
};

// L lanes to a row, N pieces to a lane: piece n of a lane is the row's n L + lane.
template <typename T, int L, int N>
__global__ __launch_bounds__(L > 256 ? L : 256) void layer_norm_fwd_kernel(const LayerNormArgs p) {
  constexpr int THREADS = L > 256 ? L : 256, ROWS = THREADS / L;
  __shared__ float shared[2][L > 64 ? L / 64 : 1];
  const int lane = threadIdx.x % L;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / L;
  if (row >= p.rows) return;   // (L > 64: a work-group's threads all, or none)
  // everything that the row needs, asked for at once
  Raw<T, N> x, residual, weight, bias;
  x.template load<L>(static_cast<const T*>(p.x) + row * p.x_stride, lane, p.width);
  if (p.residual) residual.template load<L>(static_cast<const T*>(p.residual) + row * p.residual_stride, lane, p.width);
  if (p.weight) weight.template load<L>(static_cast<const T*>(p.weight), lane, p.width);
  if (p.bias) bias.template load<L>(static_cast<const T*>(p.bias), lane, p.width);
  float v[N][PIECE];
#pragma unroll
  for (int n = 0; n < N; ++n) x.values(v[n], n);
  if (p.residual) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float add[PIECE];
      residual.values(add, n);
#pragma unroll
      for (int i = 0; i < PIECE; ++i) v[n][i] += add[i];
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < PIECE; ++i) sum += v[n][i];
  const float mean = sum_row<L>(sum, shared[0]) / p.width;
  sum = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
    if ((n * L + lane) * PIECE < p.width)
#pragma unroll
      for (int i = 0; i < PIECE; ++i) sum += (v[n][i] - mean) * (v[n][i] - mean);
  const float r = 1.f / sqrtf(sum_row<L>(sum, shared[1]) / p.width + p.eps);
  if (p.stats && lane == 0) *reinterpret_cast<float2*>(p.stats + row * 2) = make_float2(mean, r);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int at = (n * L + lane) * PIECE;
    if (at >= p.width) continue;
    if (p.s) store_values<T, PIECE>(static_cast<T*>(p.s) + row * p.width + at, v[n]);
    if constexpr (sizeof(T) == 2)
      if (p.rest) p.rest[(row * p.width + at) / PIECE] = rest_of(v[n]);
    float w[PIECE], b[PIECE], y[PIECE];
#pragma unroll
    for (int i = 0; i < PIECE; ++i) { w[i] = 1.f; b[i] = 0.f; }
    if (p.weight) weight.values(w, n);
    if (p.bias) bias.values(b, n);
#pragma unroll
    for (int i = 0; i < PIECE; ++i) y[i] = (v[n][i] - mean) * r * w[i] + b[i];
    store_values<T, PIECE>(static_cast<T*>(p.y) + row * p.width + at, y);
  }
}

// Gradients: work-groups walk over the rows with their lanes' terms of dw and db in registers, and leave one row of each, [group][dw, db][width].
// What the next row needs is on its way while this one's sums are formed.  Where a row takes 1024 lanes, there are 128 registers a lane, and the terms' sums do not fit beside the row: those
// rows are a work-group each, and the weights' gradients have a launch that reads s and dy again (with all of it in one, spilled, 4096 rows of 16384 302 us for 119 + 72,
// 2048 of 32768 814 for 132 + 71).  Rows past 16384 still do not fit in some forms: spilled are 3 registers of a lane in bf16 with ds and the four bits, in fp32 39 forward, 76 back with ds and
// 2 without (2048 of 32768 with a residual in fp32: forward 293 us, 3.7 TB/s; rows of 16384, which fit, 220 for 4096 of them, 4.9).
template <typename T, int L, int N, bool SUM, bool REST>
__global__ __launch_bounds__(L > 256 ? L : 256) void layer_norm_bwd_kernel(const LayerNormArgs p) {
  constexpr int THREADS = L > 256 ? L : 256, ROWS = THREADS / L, WAVES = L > 64 ? L / 64 : 1;
  constexpr bool WIDE = L > 256;
  __shared__ float shared[2][2 * WAVES];
  __shared__ float rows[ROWS > 1 ? THREADS * N * PIECE : 1];
  const int lane = threadIdx.x % L, sub = threadIdx.x / L;
  float dw[WIDE ? 1 : N][PIECE], db[WIDE ? 1 : N][PIECE];
  Raw<T, N> weight;
  if (p.weight) weight.template load<L>(static_cast<const T*>(p.weight), lane, p.width);
#pragma unroll
  for (int n = 0; n < (WIDE ? 1 : N); ++n)
#pragma unroll
    for (int i = 0; i < PIECE; ++i) dw[n][i] = db[n][i] = 0.f;
  struct Row {
    Raw<T, N> s, dy, ds;
    unsigned rest[N];
    float2 stat;
  };
  auto fetch = [&](Row& r, int64_t row) {   // (past the last row: it again, for nothing)
    const int64_t at = row < p.rows ? row : p.rows - 1;
    r.stat = *reinterpret_cast<const float2*>(p.stats + at * 2);
    r.s.template load<L>(static_cast<const T*>(p.x) + at * p.x_stride, lane, p.width);
    if constexpr (REST)
#pragma unroll
      for (int n = 0; n < N; ++n) r.rest[n] = (n * L + lane) * PIECE < p.width ? p.rest[at * (p.width / PIECE) + n * L + lane] : 0u;
    r.dy.template load<L>(static_cast<const T*>(p.dy) + at * p.width, lane, p.width);
    if constexpr (SUM) r.ds.template load<L>(static_cast<const T*>(p.ds) + at * p.width, lane, p.width);
  };
  int turn = 0;
  auto one = [&](const Row& r, int64_t row) {
    const bool there = row < p.rows;   // (ROWS > 1: the lanes of a row that is not there go along with zeros)
    float u[N][PIECE], g[N][PIECE], sums[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const bool in = there && (n * L + lane) * PIECE < p.width;
      float w[PIECE];
#pragma unroll
      for (int i = 0; i < PIECE; ++i) w[i] = 1.f;
      if (p.weight) weight.values(w, n);
      r.s.values(u[n], n);
      if constexpr (REST) add_rest(u[n], r.rest[n]);
      r.dy.values(g[n], n);
#pragma unroll
      for (int i = 0; i < PIECE; ++i) {
        u[n][i] = in ? (u[n][i] - r.stat.x) * r.stat.y : 0.f;
        const float d = in ? g[n][i] : 0.f;
        if constexpr (!WIDE) {
          dw[n][i] += d * u[n][i];
          db[n][i] += d;
        }
        g[n][i] = d * w[i];
        sums[0] += g[n][i];
        sums[1] += g[n][i] * u[n][i];
      }
    }
#pragma unroll
    for (int m = 1; m < (L < 64 ? L : 64); m <<= 1) {
      sums[0] += __shfl_xor(sums[0], m);
      sums[1] += __shfl_xor(sums[1], m);
    }
    if constexpr (L > 64) {   // (two places in turn: what is written now was read two barriers ago)
      float* const place = shared[turn];
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
        place[threadIdx.x >> 6] = sums[0];
        place[WAVES + (threadIdx.x >> 6)] = sums[1];
      }
      __syncthreads();
      sums[0] = sums[1] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) { sums[0] += place[w]; sums[1] += place[WAVES + w]; }
    }
    const float mg = sums[0] / p.width, mgu = sums[1] / p.width;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = (n * L + lane) * PIECE;
      float dx[PIECE];
#pragma unroll
      for (int i = 0; i < PIECE; ++i) dx[i] = r.stat.y * (g[n][i] - mg - u[n][i] * mgu);
      if constexpr (SUM) {
        float add[PIECE];
        r.ds.values(add, n);
#pragma unroll
        for (int i = 0; i < PIECE; ++i) dx[i] += add[i];
      }
      if (there && at < p.width) store_values<T, PIECE>(static_cast<T*>(p.dx) + row * p.width + at, dx);
    }
  };
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + sub;
  Row here;
  if constexpr (WIDE) {   // a row to a work-group
    fetch(here, row);
    one(here, row);
    return;
  } else {
    Row next;
    fetch(here, row);
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < p.rows; row0 += 2 * step) {
      fetch(next, row + step);
      one(here, row);
      if (row0 + step >= p.rows) break;
      fetch(here, row + 2 * step);
      one(next, row + step);
      row += 2 * step;
    }
  }
  if constexpr (!WIDE) {
    if (!p.partial) return;
    float* const out = p.partial + (int64_t)blockIdx.x * 2 * p.width;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float (&d)[N][PIECE] = which ? db : dw;
      if constexpr (ROWS > 1) {   // the rows side by side, added in their order
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < PIECE; ++i) rows[sub * (L * N * PIECE) + (n * L + lane) * PIECE + i] = d[n][i];
        __syncthreads();
        for (int c = threadIdx.x; c < p.width; c += THREADS) {
          float t = 0.f;
#pragma unroll
          for (int q = 0; q < ROWS; ++q) t += rows[q * (L * N * PIECE) + c];
          out[which * p.width + c] = t;
        }
      } else {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int at = (n * L + lane) * PIECE;
          if (at < p.width) store_values<float, PIECE>(out + which * p.width + at, d[n]);
        }
      }
    }
  }
}

// The weights' gradients of wide rows: a work-group has 512 columns (eight a lane) of a run of rows, its four waves every fourth row each, their sums joined in the waves' order.
template <typename T, bool REST>
__global__ __launch_bounds__(256) void layer_norm_columns_kernel(const LayerNormArgs p, int rows_per_run) {
  constexpr int AHEAD = 4;
  __shared__ float part[2][4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = blockIdx.x * 512 + lane * PIECE;
  const int64_t begin = (int64_t)blockIdx.y * rows_per_run, end = begin + rows_per_run < p.rows ? begin + rows_per_run : p.rows;
  float dw[PIECE], db[PIECE];
#pragma unroll
  for (int i = 0; i < PIECE; ++i) dw[i] = db[i] = 0.f;
  if (at < p.width)
    for (int64_t row = begin + wave; row < end; row += 4 * AHEAD) {
      float s[AHEAD][PIECE], d[AHEAD][PIECE];
      float2 stat[AHEAD];
      unsigned rest[AHEAD];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {   // (past the run: its last row again, for nothing)
        const int64_t r = row + 4 * a < end ? row + 4 * a : end - 1;
        load_values<T, PIECE>(s[a], static_cast<const T*>(p.x) + r * p.x_stride + at);
        load_values<T, PIECE>(d[a], static_cast<const T*>(p.dy) + r * p.width + at);
        stat[a] = *reinterpret_cast<const float2*>(p.stats + r * 2);
        if constexpr (REST) rest[a] = p.rest[(r * p.width + at) / PIECE];
      }
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        if (row + 4 * a >= end) break;
        if constexpr (REST) add_rest(s[a], rest[a]);
#pragma unroll
        for (int i = 0; i < PIECE; ++i) {
          dw[i] += d[a][i] * ((s[a][i] - stat[a].x) * stat[a].y);
          db[i] += d[a][i];
        }
      }
    }
#pragma unroll
  for (int i = 0; i < PIECE; ++i) {
    part[0][wave][lane * PIECE + i] = dw[i];
    part[1][wave][lane * PIECE + i] = db[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 1024; c += 256) {
    const int which = c >> 9, column = blockIdx.x * 512 + (c & 511);
    const float(&of)[4][512] = part[which];
    if (column < p.width) p.partial[((int64_t)blockIdx.y * 2 + which) * p.width + column] = ((of[0][c & 511] + of[1][c & 511]) + of[2][c & 511]) + of[3][c & 511];
  }
}

// The work-groups' rows summed: 32 columns a work-group, rows dealt over 32 threads a column and joined in order.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_sum_kernel(const LayerNormArgs p, int groups) {
  __shared__ float sums[32][33];
  const int c = threadIdx.x & 31, part = threadIdx.x >> 5, column = blockIdx.x * 32 + c, columns = 2 * p.width;
  float s = 0.f;
  if (column < columns)
#pragma unroll 8
    for (int g = part; g < groups; g += 32) s += p.partial[(int64_t)g * columns + column];
  sums[part][c] = s;
  __syncthreads();
  if (part == 0 && column < columns) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][c];
    if (column < p.width) {
      if (p.dweight) store_one(static_cast<T*>(p.dweight) + column, s);
    } else if (p.dbias) {
      store_one(static_cast<T*>(p.dbias) + column - p.width, s);
    }
  }
}

double values_of(const LayerNormArgs& a) { return (double)a.rows * a.width; }

template <typename T, int L, int N>
hipError_t fwd(const LayerNormArgs& a, hipStream_t s) {
  constexpr int THREADS = L > 256 ? L : 256, ROWS = THREADS / L;
  note_matrix(a.x, a.rows, a.width, a.x_stride, sizeof(T), false);
  if (a.residual) note_matrix(a.residual, a.rows, a.width, a.residual_stride, sizeof(T), false);
  note_matrix(a.weight, 1, a.width, a.width, sizeof(T), false);
  note_matrix(a.bias, 1, a.width, a.width, sizeof(T), false);
  note_matrix(a.y, a.rows, a.width, a.width, sizeof(T), true);
  note_matrix(a.s, a.rows, a.width, a.width, sizeof(T), true);
  note_matrix(a.rest, a.rows, a.width / PIECE, a.width / PIECE, 4, true);
  note_matrix(a.stats, a.rows, 2, 2, 4, true);
  const int tensors = 2 + (a.residual != nullptr) + (a.s != nullptr);
  return launch_kernel("layer_norm_fwd_kernel", Work{8 * values_of(a), tensors * values_of(a) * sizeof(T)}, layer_norm_fwd_kernel<T, L, N>,
                       dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), dim3(THREADS), s, a);
}

template <typename T, int L, int N>
hipError_t bwd(const LayerNormArgs& a, hipStream_t s) {
  constexpr int THREADS = L > 256 ? L : 256;
  const int groups = layer_norm_groups(a.rows, a.width);
  note_matrix(a.x, a.rows, a.width, a.x_stride, sizeof(T), false);
  note_matrix(a.rest, a.rows, a.width / PIECE, a.width / PIECE, 4, false);
  note_matrix(a.weight, 1, a.width, a.width, sizeof(T), false);
  note_matrix(a.stats, a.rows, 2, 2, 4, false);
  note_matrix(a.dy, a.rows, a.width, a.width, sizeof(T), false);
  note_matrix(a.ds, a.rows, a.width, a.width, sizeof(T), false);
  note_matrix(a.dx, a.rows, a.width, a.width, sizeof(T), true);
  if (L <= 256) note_matrix(a.partial, groups, 2 * a.width, 2 * a.width, 4, true);
  auto kernel = a.ds ? layer_norm_bwd_kernel<T, L, N, true, false> : layer_norm_bwd_kernel<T, L, N, false, false>;
  if constexpr (sizeof(T) == 2)
    if (a.rest) kernel = a.ds ? layer_norm_bwd_kernel<T, L, N, true, true> : layer_norm_bwd_kernel<T, L, N, false, true>;
  hipError_t e = launch_kernel("layer_norm_bwd_kernel", Work{14 * values_of(a), ((a.ds ? 4 : 3) * sizeof(T) + (a.rest ? 0.5 : 0.0)) * values_of(a)},
                               kernel, dim3(L > 256 ? (unsigned)a.rows : groups), dim3(THREADS), s, a);
  if (e != hipSuccess || !a.partial) return e;
  if constexpr (L > 256) {
    const ColumnRuns r(a.rows, a.width);
    note_matrix(a.x, a.rows, a.width, a.x_stride, sizeof(T), false);
    note_matrix(a.rest, a.rows, a.width / PIECE, a.width / PIECE, 4, false);
    note_matrix(a.dy, a.rows, a.width, a.width, sizeof(T), false);
    note_matrix(a.stats, a.rows, 2, 2, 4, false);
    note_matrix(a.partial, groups, 2 * a.width, 2 * a.width, 4, true);
    auto columns = layer_norm_columns_kernel<T, false>;
    if constexpr (sizeof(T) == 2)
      if (a.rest) columns = layer_norm_columns_kernel<T, true>;
    e = launch_kernel("layer_norm_columns_kernel", Work{5 * values_of(a), (2 * sizeof(T) + (a.rest ? 0.5 : 0.0)) * values_of(a)}, columns, dim3((unsigned)r.groups, (unsigned)r.runs), dim3(256), s, a, r.rows);
    if (e != hipSuccess) return e;
  }
  note_matrix(a.partial, groups, 2 * a.width, 2 * a.width, 4, false);
  note_matrix(a.dweight, 1, a.width, a.width, sizeof(T), true);
  note_matrix(a.dbias, 1, a.width, a.width, sizeof(T), true);
  return launch_kernel("layer_norm_sum_kernel", Work{0.0, 8.0 * groups * a.width}, layer_norm_sum_kernel<T>, dim3((2 * a.width + 31) / 32), dim3(1024), s, a, groups);
}

template <typename T, bool BACK>
hipError_t by_width(const LayerNormArgs& a, hipStream_t s) {
  auto go = [&](auto l, auto n) {
    if constexpr (BACK) return bwd<T, decltype(l)::value, decltype(n)::value>(a, s);
    else return fwd<T, decltype(l)::value, decltype(n)::value>(a, s);
  };
  const int pieces = a.width / PIECE;
  switch (layer_norm_lanes(a.width)) {
    case 8: return go(IntC<8>{}, IntC<1>{});
    case 16: return go(IntC<16>{}, IntC<1>{});
    case 32: return go(IntC<32>{}, IntC<1>{});
    case 64: return pieces <= 64 ? go(IntC<64>{}, IntC<1>{}) : go(IntC<64>{}, IntC<2>{});
    case 256: return pieces <= 256 ? go(IntC<256>{}, IntC<1>{}) : pieces <= 512 ? go(IntC<256>{}, IntC<2>{}) : pieces <= 768 ? go(IntC<256>{}, IntC<3>{}) : go(IntC<256>{}, IntC<4>{});
    default: return pieces <= 2048 ? go(IntC<1024>{}, IntC<2>{}) : pieces <= 4096 ? go(IntC<1024>{}, IntC<4>{}) : hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_layer_norm_fwd(const LayerNormArgs& a, bool f32, hipStream_t s) {
  return f32 ? by_width<float, false>(a, s) : by_width<bf16, false>(a, s);
}
hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, bool f32, hipStream_t s) {
  return f32 ? by_width<float, true>(a, s) : by_width<bf16, true>(a, s);
}

}  // namespace sk
