// RMS norm of every query and key head with the position rotation in the same pass, and its gradients.
//
//   r = 1 / sqrt(mean x^2 + eps),  n = x w r,  (a, b) -> (a cos - b sin, b cos + a sin) on the pairs of n
//   dn = the rotation back on dy,  dw = sum dn x r,  g = dn w,  dx = r (g - x r^2 mean(g x))
//
// Bound by memory, one pass over it each way (r is computed again from x, which the gradient needs anyway): 16384 tokens of 32 + 8 heads of 128 in
// bf16, 341 MB, forward 62 us = 5.5 TB/s; back 108 us for 513 MB = 4.7 TB/s (a copy: 5.2) and 5 for the sum of the weights' gradients.  Heads of
// several steps loaded before the first is used took the forward pass from 65 to 63 us and the backward pass from 108 to 115, where registers cost waves.
//
// A head's D values lie on L lanes (D / 8, rounded up to a power of two), eight to a lane: four rotated pairs, so that
// neither the rotation nor the products with the weights cross lanes, only the sum of squares does.  Halves: lane i has values 4 i ..
// + 3 of the first half of its part of the head (the rotated part or the rest, which is two halves under a turn of zero)
// and the same of the second; interleaved: values 8 i .. + 7.
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

// Where a lane's four pairs are: first values a .. a + 3 and second b .. b + 3 (halves), or a .. a + 7 in turn.
struct Pairs {
  int a, b, column;      // column: of the tables, -1 where nothing turns
  bool there;
};
template <bool INTERLEAVED>
__device__ __forceinline__ Pairs pairs_of(int piece, int D, int rotary) {
  Pairs q;
  const int at = piece * 4, half = rotary / 2;
  q.there = at < D / 2;
  q.column = at < half ? at : -1;
  if (INTERLEAVED) {
    q.a = 2 * at;
    q.b = 2 * at + 4;
  } else if (at < half) {
    q.a = at;
    q.b = half + at;
  } else {
    q.a = half + at;                     // rotary + (at - half)
    q.b = half + at + (D - rotary) / 2;
  }
  return q;
}

// x[0..3] the pairs' first values, x[4..7] their second
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void load_pairs(float (&x)[8], const T* p, const Pairs& q) {
  if (INTERLEAVED) {
    float v[8];
    load_values<T, 8>(v, p + q.a);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = v[2 * i]; x[4 + i] = v[2 * i + 1]; }
  } else {
    float a[4], b[4];
    load_values<T, 4>(a, p + q.a);
    load_values<T, 4>(b, p + q.b);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
  }
}
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void store_pairs(T* p, const float (&x)[8], const Pairs& q) {
  if (INTERLEAVED) {
    const float v[8] = {x[0], x[4], x[1], x[5], x[2], x[6], x[3], x[7]};
    store_values<T, 8>(p + q.a, v);
  } else {
    const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
    store_values<T, 4>(p + q.a, a);
    store_values<T, 4>(p + q.b, b);
  }
}

template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int m = 1; m < L; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

__device__ __forceinline__ int64_t table_row(const NormRopeArgs& p, int64_t t) {
  const int64_t at = p.pos64 ? static_cast<const int64_t*>(p.positions)[t] : static_cast<const int32_t*>(p.positions)[t];
  return at < 0 ? 0 : at < p.table_rows ? at : p.table_rows - 1;
}
__device__ __forceinline__ void load_turn(float (&cs)[4], float (&sn)[4], const NormRopeArgs& p, int64_t t, const Pairs& q) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  if (q.there && q.column >= 0) {
    const int64_t at = table_row(p, t) * (p.rotary / 2) + q.column;
    load_values<float, 4>(cs, p.cos + at);
    load_values<float, 4>(sn, p.sin + at);
  }
}

// A wave takes one token's heads, 64 / L at a time, so that the turn is loaded once for all of them, or with `parts` > 1 (few tokens) a part
// of them: eight tokens of 72 heads 3.7 us, a launch's own time.
template <typename T, int L, bool INTERLEAVED>
__global__ __launch_bounds__(256) void norm_rope_fwd_kernel(const NormRopeArgs p, int parts) {
  constexpr int HEADS = 64 / L;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = id / parts;
  const int part = (int)(id - t * parts);
  if (t >= p.tokens) return;
  const Pairs q = pairs_of<INTERLEAVED>(lane % L, p.D, p.rotary);
  float cs[4], sn[4];
  load_turn(cs, sn, p, t, q);
  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 0.f;
  if (q.there) {
    load_pairs<T, INTERLEAVED>(wq, static_cast<const T*>(p.wq), q);
    if (p.kv_heads > 0) load_pairs<T, INTERLEAVED>(wk, static_cast<const T*>(p.wk), q);
  }
  const int heads = p.heads + p.kv_heads;
  for (int h0 = part * HEADS; h0 < heads; h0 += parts * HEADS) {
    const int h = h0 + lane / L;
    const bool key = h >= p.heads, there = q.there && h < heads;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    const T* const in = key ? static_cast<const T*>(p.k) + t * p.ks[0] + (h - p.heads) * p.ks[1] : static_cast<const T*>(p.q) + t * p.qs[0] + h * p.qs[1];
    if (there) load_pairs<T, INTERLEAVED>(x, in, q);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
    ss = sum_lanes<L>(ss);
    const float r = 1.f / sqrtf(ss / p.D + p.eps);
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[i] * r * (key ? wk[i] : wq[i]), b = x[4 + i] * r * (key ? wk[4 + i] : wq[4 + i]);
      y[i] = a * cs[i] - b * sn[i];
      y[4 + i] = b * cs[i] + a * sn[i];
    }
    T* const out = key ? static_cast<T*>(p.k_out) + t * p.kos[0] + (h - p.heads) * p.kos[1] : static_cast<T*>(p.q_out) + t * p.qos[0] + h * p.qos[1];
    if (there) store_pairs<T, INTERLEAVED>(out, y, q);
  }
}

// Gradients: a wave walks over tokens with its lanes' terms of the weights' gradients in registers; a work-group leaves one row
// of them, [group][queries, keys][D].  The weights' columns are the lane's own all the way.
template <typename T, int L, bool INTERLEAVED>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(const NormRopeArgs p) {
  constexpr int HEADS = 64 / L;
  __shared__ float sums[4][64][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Pairs q = pairs_of<INTERLEAVED>(lane % L, p.D, p.rotary);
  float w[2][8], dw[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[0][i] = w[1][i] = dw[0][i] = dw[1][i] = 0.f;
  if (q.there) {
    load_pairs<T, INTERLEAVED>(w[0], static_cast<const T*>(p.wq), q);
    if (p.kv_heads > 0) load_pairs<T, INTERLEAVED>(w[1], static_cast<const T*>(p.wk), q);
  }
  for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < p.tokens; t += (int64_t)gridDim.x * 4) {
    float cs[4], sn[4];
    load_turn(cs, sn, p, t, q);
#pragma unroll
    for (int key = 0; key < 2; ++key) {
      const int heads = key ? p.kv_heads : p.heads;
      const T* const in = key ? static_cast<const T*>(p.k) + t * p.ks[0] : static_cast<const T*>(p.q) + t * p.qs[0];
      const int64_t head_stride = key ? p.ks[1] : p.qs[1];
      const T* const grad = (key ? static_cast<const T*>(p.dk_out) : static_cast<const T*>(p.dq_out)) + t * heads * p.D;
      T* const out = (key ? static_cast<T*>(p.k_out) : static_cast<T*>(p.q_out)) + t * heads * p.D;
      for (int h0 = 0; h0 < heads; h0 += HEADS) {
        const int h = h0 + lane / L;
        const bool there = q.there && h < heads;
        float x[8], g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = g[i] = 0.f;
        if (there) {
          load_pairs<T, INTERLEAVED>(x, in + h * head_stride, q);
          load_pairs<T, INTERLEAVED>(g, grad + (int64_t)h * p.D, q);
        }
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
        ss = sum_lanes<L>(ss);
        const float r = there ? 1.f / sqrtf(ss / p.D + p.eps) : 0.f;   // (a head that is not there: not 1 / 0 where eps is 0)
        float gx = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // the rotation back, then the norm's
          const float a = g[i] * cs[i] + g[4 + i] * sn[i], b = g[4 + i] * cs[i] - g[i] * sn[i];
          dw[key][i] += a * x[i] * r;
          dw[key][4 + i] += b * x[4 + i] * r;
          g[i] = a * w[key][i];
          g[4 + i] = b * w[key][4 + i];
          gx += g[i] * x[i] + g[4 + i] * x[4 + i];
        }
        gx = sum_lanes<L>(gx) / p.D * r * r;
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = r * (g[i] - x[i] * gx);
        if (there) store_pairs<T, INTERLEAVED>(out + (int64_t)h * p.D, g, q);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) { sums[wave][lane][i] = dw[0][i]; sums[wave][lane][8 + i] = dw[1][i]; }
  __syncthreads();
  // (lane, value) of the first head's lanes over the work-group's heads and waves, in that order
  for (int at = threadIdx.x; at < L * 16; at += 256) {
    const int l = at / 16, v = at % 16;
    float s = 0.f;
#pragma unroll
    for (int wv = 0; wv < 4; ++wv)
#pragma unroll
      for (int h = 0; h < HEADS; ++h) s += sums[wv][h * L + l][v];
    const Pairs u = pairs_of<INTERLEAVED>(l, p.D, p.rotary);
    const int i = v & 7, column = INTERLEAVED ? u.a + 2 * (i & 3) + (i >> 2) : i < 4 ? u.a + i : u.b + i - 4;
    if (u.there) p.partial[((int64_t)blockIdx.x * 2 + v / 8) * p.D + column] = s;
  }
}

// The work-groups' rows summed: 32 columns a work-group, rows dealt over 32 threads a column and joined in order.
template <typename T>
__global__ __launch_bounds__(1024) void norm_rope_sum_kernel(const NormRopeArgs p, int groups) {
  __shared__ float sums[32][33];
  const int c = threadIdx.x & 31, part = threadIdx.x >> 5, column = blockIdx.x * 32 + c, columns = 2 * p.D;
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
    if (column < p.D) store_one(static_cast<T*>(p.dwq) + column, s);
    else if (p.kv_heads > 0) store_one(static_cast<T*>(p.dwk) + column - p.D, s);
  }
}

void note_io(const NormRopeArgs& a, int esize, bool back) {
  if (!tracing()) return;
  note_matrix(a.q, 1, (a.tokens - 1) * a.qs[0] + (a.heads - 1) * a.qs[1] + a.D, 0, esize, false);
  if (a.kv_heads > 0) note_matrix(a.k, 1, (a.tokens - 1) * a.ks[0] + (a.kv_heads - 1) * a.ks[1] + a.D, 0, esize, false);
  note_matrix(a.wq, 1, a.D, a.D, esize, false);
  if (a.kv_heads > 0) note_matrix(a.wk, 1, a.D, a.D, esize, false);
  if (a.rotary > 0) {
    note_matrix(a.cos, a.table_rows, a.rotary / 2, a.rotary / 2, 4, false);
    note_matrix(a.sin, a.table_rows, a.rotary / 2, a.rotary / 2, 4, false);
    note_matrix(a.positions, 1, a.tokens, a.tokens, a.pos64 ? 8 : 4, false);
  }
  if (back) {
    note_matrix(a.dq_out, a.tokens * a.heads, a.D, a.D, esize, false);
    if (a.kv_heads > 0) note_matrix(a.dk_out, a.tokens * a.kv_heads, a.D, a.D, esize, false);
    note_matrix(a.q_out, a.tokens * a.heads, a.D, a.D, esize, true);
    if (a.kv_heads > 0) note_matrix(a.k_out, a.tokens * a.kv_heads, a.D, a.D, esize, true);
  } else {
    note_matrix(a.q_out, 1, (a.tokens - 1) * a.qos[0] + (a.heads - 1) * a.qos[1] + a.D, 0, esize, true);
    if (a.kv_heads > 0) note_matrix(a.k_out, 1, (a.tokens - 1) * a.kos[0] + (a.kv_heads - 1) * a.kos[1] + a.D, 0, esize, true);
  }
}
double values_of(const NormRopeArgs& a) { return (double)a.tokens * (a.heads + a.kv_heads) * a.D; }

template <typename T, int L, bool INTERLEAVED>
hipError_t fwd(const NormRopeArgs& a, hipStream_t s) {
  constexpr int HEADS = 64 / L;
  const int rounds = (a.heads + a.kv_heads + HEADS - 1) / HEADS;
  // few tokens: a token's heads over several waves, up to about two waves a SIMD
  int64_t parts = (2 * 4 * NUM_CUS + a.tokens - 1) / a.tokens;
  parts = parts < 1 ? 1 : parts > rounds ? rounds : parts;
  note_io(a, sizeof(T), false);
  return launch_kernel("norm_rope_fwd_kernel", Work{8 * values_of(a), 2 * values_of(a) * sizeof(T)}, norm_rope_fwd_kernel<T, L, INTERLEAVED>,
                       dim3((unsigned)((a.tokens * parts + 3) / 4)), dim3(256), s, a, (int)parts);
}

template <typename T, int L, bool INTERLEAVED>
hipError_t bwd(const NormRopeArgs& a, hipStream_t s) {
  const int groups = (int)(a.tokens + 3 < 4 * NORM_ROPE_MAX_GROUPS ? (a.tokens + 3) / 4 : NORM_ROPE_MAX_GROUPS);
  note_io(a, sizeof(T), true);
  note_matrix(a.partial, 1, (int64_t)groups * 2 * a.D, 0, 4, true);
  hipError_t e = launch_kernel("norm_rope_bwd_kernel", Work{12 * values_of(a), 3 * values_of(a) * sizeof(T)}, norm_rope_bwd_kernel<T, L, INTERLEAVED>,
                               dim3(groups), dim3(256), s, a);
  if (e != hipSuccess) return e;
  note_matrix(a.partial, 1, (int64_t)groups * 2 * a.D, 0, 4, false);
  note_matrix(a.dwq, 1, a.D, 0, sizeof(T), true);
  if (a.kv_heads > 0) note_matrix(a.dwk, 1, a.D, 0, sizeof(T), true);
  return launch_kernel("norm_rope_sum_kernel", Work{0.0, 8.0 * groups * a.D}, norm_rope_sum_kernel<T>, dim3((2 * a.D + 31) / 32), dim3(1024), s, a, groups);
}

template <typename T, bool INTERLEAVED, bool BACK>
hipError_t by_lanes(const NormRopeArgs& a, hipStream_t s) {
  auto go = [&](auto l) {
    if constexpr (BACK) return bwd<T, decltype(l)::value, INTERLEAVED>(a, s);
    else return fwd<T, decltype(l)::value, INTERLEAVED>(a, s);
  };
  if (a.D <= 32) return go(IntC<4>{});
  if (a.D <= 64) return go(IntC<8>{});
  if (a.D <= 128) return go(IntC<16>{});
  return go(IntC<32>{});
}

}  // namespace

hipError_t launch_norm_rope_fwd(const NormRopeArgs& a, bool f32, hipStream_t s) {
  if (f32) return a.interleaved ? by_lanes<float, true, false>(a, s) : by_lanes<float, false, false>(a, s);
  return a.interleaved ? by_lanes<bf16, true, false>(a, s) : by_lanes<bf16, false, false>(a, s);
}

hipError_t launch_norm_rope_bwd(const NormRopeArgs& a, bool f32, hipStream_t s) {
  if (f32) return a.interleaved ? by_lanes<float, true, true>(a, s) : by_lanes<float, false, true>(a, s);
  return a.interleaved ? by_lanes<bf16, true, true>(a, s) : by_lanes<bf16, false, true>(a, s);
}

}  // namespace sk
