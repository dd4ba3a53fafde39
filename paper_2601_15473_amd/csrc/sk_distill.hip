// The loss of logits against a teacher's largest logits and against labels, and its gradient.
//
//   p = softmax(t / tau) over the teacher's entries,  q = softmax(z / tau),
//   loss = (1 - w) tau^2 sum_k p_k (log p_k - log q_k) + w (log sum exp z - z_label)
//   dz_j = g [ (1 - w) tau (q_j - p_j) + w (softmax(z)_j - [j = label]) ]
//
// Bound by memory: forward z is read once, with the largest value so far and the sums of exponentials below it carried along (rescaled once in
// some values), back it is read again and dz written (what the gradient is scaled by is known then only).  The entries are few: one thread each.
//
// A row begins wherever the vocabulary's size puts it: its values are taken 16 bytes at a time at the places where memory has them, and one by one
// in the pieces that it shares with its neighbours.
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int LISTS = 256;   // entries that a work-group has in LDS at once

__device__ __forceinline__ int64_t index_of(const void* p, int wide, int64_t at) {
  return wide ? static_cast<const int64_t*>(p)[at] : (int64_t)static_cast<const int32_t*>(p)[at];
}

// A row's 16-byte pieces: piece i has the row's values i E - lead .. + E - 1.
template <typename T>
struct RowPieces {
  static constexpr int E = 16 / sizeof(T);
  const T* row;
  int lead, n, pieces;
  __device__ __forceinline__ RowPieces(const T* r, int width) : row(r), lead((int)((reinterpret_cast<uintptr_t>(r) & 15) / sizeof(T))), n(width), pieces((lead + width + E - 1) / E) {}
  __device__ __forceinline__ bool whole(int i) const { return i * E >= lead && i * E - lead + E <= n; }
  // values outside the row: `outside`
  __device__ __forceinline__ void load(float (&v)[E], int i, float outside) const {
    const int at = i * E - lead;
    if (i < pieces && whole(i)) {
      load_values<T, E>(v, row + at);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = i < pieces && at + e >= 0 && at + e < n ? load_one(row + at + e) : outside;
    }
  }
};

struct Sums {
  float top, soft, hard;   // the largest logit, the sums of exp((z - top) / tau) and exp(z - top)
};
__device__ __forceinline__ float below(float x, float top, float c) { return __builtin_amdgcn_exp2f((x - top) * c); }
// (a row of -infinities so far has nothing to rescale)
template <bool HARD>
__device__ __forceinline__ void raise(Sums& s, float top, float c) {
  if (top == s.top) return;
  if (s.top != -INFINITY) {
    s.soft *= below(s.top, top, c);
    if (HARD) s.hard *= below(s.top, top, LOG2E);
  }
  s.top = top;
}
template <bool HARD>
__device__ __forceinline__ void join(Sums& s, Sums o, float c) {
  const float top = fmaxf(s.top, o.top);
  raise<HARD>(s, top, c);
  raise<HARD>(o, top, c);
  s.soft += o.soft;
  if (HARD) s.hard += o.hard;
}

// The sum (of 64 bits) of a work-group's threads, in all of them.
template <int THREADS>
__device__ __forceinline__ double sum_threads(double v, double* shared) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  if constexpr (THREADS > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += shared[w];
  }
  return v;
}
template <int THREADS>
__device__ __forceinline__ float max_threads(float v, double* shared) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m));
  if constexpr (THREADS > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = -INFINITY;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v = fmaxf(v, (float)shared[w]);
  }
  return v;
}

// An entry of the teacher's list: where it stands, and how large it is.  One outside the vocabulary or of -infinity is not there.
struct Entry {
  int id;
  float t;
  bool there;
};
template <typename T>
__device__ __forceinline__ Entry entry_of(const DistillArgs& p, int64_t row, int k) {
  Entry e{-1, -INFINITY, false};
  if (k >= p.top) return e;
  const int64_t id = index_of(p.ids, p.ids64, row * p.top + k);
  e.t = load_one(static_cast<const T*>(p.teacher) + row * p.top + k);
  e.there = id >= 0 && id < p.vocabulary && e.t != -INFINITY;
  if (e.there) e.id = (int)id;
  return e;
}
// The largest of a row's entries, and the sum of their exponentials below it (0: there is none)
template <typename T, int THREADS>
__device__ __forceinline__ float teacher_sum(const DistillArgs& p, int64_t row, float c, float& high, double* shared) {
  high = -INFINITY;
  for (int k = threadIdx.x; k < p.top; k += THREADS) {
    const Entry e = entry_of<T>(p, row, k);
    if (e.there) high = fmaxf(high, e.t);   // (a NaN is no largest, and comes out in the sum)
  }
  high = max_threads<THREADS>(high, shared);
  double sum = 0.0;
  for (int k = threadIdx.x; k < p.top; k += THREADS) {
    const Entry e = entry_of<T>(p, row, k);
    if (e.there) sum += below(e.t, high, c);
  }
  return (float)sum_threads<THREADS>(sum, shared);
}

// THREADS to a row
template <typename T, int THREADS, bool HARD>
__global__ __launch_bounds__(THREADS) void distill_fwd_kernel(const DistillArgs p) {
  constexpr int E = RowPieces<T>::E, AHEAD = 4;
  __shared__ double shared[THREADS / 64];
  __shared__ Sums waves[THREADS / 64];
  const int64_t row = blockIdx.x;
  const T* const z = static_cast<const T*>(p.logits) + row * p.logits_stride;
  const RowPieces<T> pieces(z, p.vocabulary);
  const float c = LOG2E / p.temperature;
  Sums s{-INFINITY, 0.f, 0.f};
  for (int i = threadIdx.x; i < pieces.pieces; i += AHEAD * THREADS) {
    float v[AHEAD][E];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) pieces.load(v[a], i + a * THREADS, -INFINITY);
    float top = s.top;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, v[a][e]);
    raise<HARD>(s, top, c);
    const float from = top == -INFINITY ? 0.f : top;   // (nothing but -infinities: their exponentials are zeros)
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s.soft += below(v[a][e], from, c);
        if (HARD) s.hard += below(v[a][e], from, LOG2E);
      }
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    Sums o;
    o.top = __shfl_xor(s.top, m);
    o.soft = __shfl_xor(s.soft, m);
    o.hard = HARD ? __shfl_xor(s.hard, m) : 0.f;
    join<HARD>(s, o, c);
  }
  if constexpr (THREADS > 64) {
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
    __syncthreads();
    s = waves[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) join<HARD>(s, waves[w], c);
  }
  const float tau = p.temperature, weight = p.label_weight;
  // the teacher's part: log p - log q is a difference of numbers much larger than it, in 64 bits
  float high;
  const float total = teacher_sum<T, THREADS>(p, row, c, high, shared);
  double loss = 0.0;
  const bool some = total != 0.f;   // (NaN: there is something)
  if (some && weight != 1.f) {
    const double logs = log((double)s.soft) - log((double)total);
    for (int k = threadIdx.x; k < p.top; k += THREADS) {
      const Entry e = entry_of<T>(p, row, k);
      if (!e.there) continue;
      const float share = below(e.t, high, c) / total;
      if (share == 0.f) continue;     // (what it would be the logarithm of may be anything)
      loss += (double)share * ((((double)e.t - (double)high) - ((double)load_one(z + e.id) - (double)s.top)) / (double)tau + logs);
    }
    loss = sum_threads<THREADS>(loss, shared) * ((1.0 - (double)weight) * (double)tau * (double)tau);
  }
  if (threadIdx.x != 0) return;
  if (p.labels && weight != 0.f) {
    const int64_t label = index_of(p.labels, p.labels64, row);
    if (label >= 0 && label < p.vocabulary)
      loss += (double)weight * (log((double)(HARD ? s.hard : s.soft)) + ((double)s.top - (double)load_one(z + label)));
  }
  p.loss[row] = (float)loss;
  if (p.stats) *reinterpret_cast<float4*>(p.stats + row * 4) = make_float4(s.top, 1.f / s.soft, 1.f / (HARD ? s.hard : s.soft), 0.f);
}

// The row of dz by its pieces first, then the values at the teacher's entries and at the label once more with what they have subtracted: by one thread each,
// the first of those with the same place, behind a wait for the work-group's stores.
template <typename T, int THREADS, bool HARD>
__global__ __launch_bounds__(THREADS) void distill_bwd_kernel(const DistillArgs p) {
  constexpr int E = RowPieces<T>::E, AHEAD = 4;
  __shared__ double shared[THREADS / 64];
  __shared__ int ids[LISTS];
  __shared__ float less[LISTS];
  const int64_t row = blockIdx.x;
  const T* const z = static_cast<const T*>(p.logits) + row * p.logits_stride;
  T* const out = static_cast<T*>(p.dlogits) + row * p.vocabulary;
  const RowPieces<T> pieces(z, p.vocabulary);
  const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;   // (pieces of both are the same)
  const float tau = p.temperature, c = LOG2E / tau;
  const float4 stat = *reinterpret_cast<const float4*>(p.stats + row * 4);
  const float top = stat.x, g = p.dloss[row];
  float high;
  const float total = teacher_sum<T, THREADS>(p, row, c, high, shared);
  int64_t label = -1;
  if (p.labels && p.label_weight != 0.f) {
    label = index_of(p.labels, p.labels64, row);
    if (label < 0 || label >= p.vocabulary) label = -1;
  }
  const bool teaches = total != 0.f && p.label_weight != 1.f, counts = teaches || label >= 0;
  const float share = teaches ? g * (1.f - p.label_weight) * tau : 0.f;   // of the entries
  const float right = label >= 0 ? g * p.label_weight : 0.f;              // of the label
  // what q and softmax(z) are multiplied by, over their sums
  const float soft = HARD ? share * stat.y : (share + right) * stat.y, hard = HARD ? right * stat.z : 0.f;
  auto dense = [&](float v) { return soft * below(v, top, c) + (HARD ? hard * below(v, top, LOG2E) : 0.f); };
  for (int i = threadIdx.x; i < pieces.pieces; i += AHEAD * THREADS) {
    float v[AHEAD][E];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) pieces.load(v[a], i + a * THREADS, 0.f);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int piece = i + a * THREADS, at = piece * E - pieces.lead;
      if (piece >= pieces.pieces) break;
#pragma unroll
      for (int e = 0; e < E; ++e) v[a][e] = counts ? dense(v[a][e]) : 0.f;
      if (together && pieces.whole(piece)) {
        store_values<T, E>(out + at, v[a]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (at + e >= 0 && at + e < p.vocabulary) store_one(out + at + e, v[a][e]);
      }
    }
  }
  if (!counts) return;
  // (a piece's store and a place's of another wave: the first has to have arrived)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  const int n = teaches ? p.top : 0;
  const float each = teaches ? share / total : 0.f;
  // the list's entries, the label behind them, against all of them a stretch at a time
  for (int k0 = 0; k0 <= n; k0 += THREADS) {
    const int k = k0 + (int)threadIdx.x;
    int id = -1;
    if (k < n) id = entry_of<T>(p, row, k).id;
    else if (k == n) id = (int)label;
    float sum = 0.f;
    bool first = id >= 0;
    for (int j0 = 0; j0 <= n; j0 += LISTS) {
      __syncthreads();
      for (int j = threadIdx.x; j < LISTS; j += THREADS) {
        int other = -1;
        float w = 0.f;
        if (j0 + j < n) {
          const Entry e = entry_of<T>(p, row, j0 + j);
          other = e.id;
          if (e.there) w = below(e.t, high, c) * each;
        } else if (j0 + j == n) {
          other = (int)label;
          w = right;
        }
        ids[j] = other;
        less[j] = w;
      }
      __syncthreads();
      const int m = n + 1 - j0 < LISTS ? n + 1 - j0 : LISTS;
      for (int j = 0; j < m; ++j) {
        const bool same = ids[j] == id;
        sum += same ? less[j] : 0.f;
        if (same && j0 + j < k) first = false;
      }
    }
    if (first) store_one(out + id, dense(load_one(z + id)) - sum);
  }
}

double values_of(const DistillArgs& a) { return (double)a.rows * a.vocabulary; }
void note_io(const DistillArgs& a, int esize, bool back) {
  if (!tracing()) return;
  note_matrix(a.logits, a.rows, a.vocabulary, a.logits_stride, esize, false);
  note_matrix(a.teacher, a.rows, a.top, a.top, esize, false);
  note_matrix(a.ids, a.rows, a.top, a.top, a.ids64 ? 8 : 4, false);
  note_matrix(a.labels, 1, a.rows, a.rows, a.labels64 ? 8 : 4, false);
  note_matrix(a.stats, a.rows, 4, 4, 4, !back);
  if (back) {
    note_matrix(a.dloss, 1, a.rows, a.rows, 4, false);
    note_matrix(a.dlogits, a.rows, a.vocabulary, a.vocabulary, esize, true);
  } else {
    note_matrix(a.loss, 1, a.rows, a.rows, 4, true);
  }
}

template <typename T, int THREADS, bool HARD, bool BACK>
hipError_t go(const DistillArgs& a, hipStream_t s) {
  note_io(a, sizeof(T), BACK);
  if constexpr (BACK)
    return launch_kernel("distill_bwd_kernel", Work{4 * values_of(a), 2 * values_of(a) * sizeof(T)}, distill_bwd_kernel<T, THREADS, HARD>, dim3((unsigned)a.rows), dim3(THREADS), s, a);
  else
    return launch_kernel("distill_fwd_kernel", Work{4 * values_of(a), values_of(a) * sizeof(T)}, distill_fwd_kernel<T, THREADS, HARD>, dim3((unsigned)a.rows), dim3(THREADS), s, a);
}

template <typename T, bool HARD, bool BACK>
hipError_t by_size(const DistillArgs& a, hipStream_t s) {
  if (a.vocabulary <= 2048) return go<T, 64, HARD, BACK>(a, s);
  return go<T, 256, HARD, BACK>(a, s);
}
template <bool BACK>
hipError_t by_type(const DistillArgs& a, bool f32, hipStream_t s) {
  // (one sum serves both parts where the temperature is 1, or where one of them is not there)
  const bool hard = a.labels && a.label_weight != 0.f && a.temperature != 1.f;
  if (f32) return hard ? by_size<float, true, BACK>(a, s) : by_size<float, false, BACK>(a, s);
  return hard ? by_size<bf16, true, BACK>(a, s) : by_size<bf16, false, BACK>(a, s);
}

}  // namespace

hipError_t launch_distill_fwd(const DistillArgs& a, bool f32, hipStream_t s) { return by_type<false>(a, f32, s); }
hipError_t launch_distill_bwd(const DistillArgs& a, bool f32, hipStream_t s) { return by_type<true>(a, f32, s); }

}  // namespace sk
