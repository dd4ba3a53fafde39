// The loss of logits against a teacher's largest logits and against labels, and its gradient.
//
//   p = softmax(t / tau) over the teacher's entries,  q = softmax(z / tau),
//   loss = (1 - w) tau^2 sum_k p_k (log p_k - log q_k) + w (log sum exp z - z_label)
//   dz_j = g [ (1 - w) tau (q_j - p_j) + w (softmax(z)_j - [j = label]) ]
//
// Bound by memory: forward z is read once, with the largest value so far and the sums of exponentials below it carried along (rescaled once in
// some values), back it is read again and dz written (what the gradient is scaled by is known then only).  The entries are few: one thread each.
// Bf16, 8192 rows of 65536: forward 179 us with one exponential a value (1.07 GB, 6.0 TB/s), 265 with two, back 398 with lists of 128 (2.15 GB, 5.4; a copy reaches 5.1).  Behind a backward pass
// the forward one takes 215 and 267: it shares the memory with what that pass left to be written back.  Fp32, 8192 rows of 32000: 177 forward (5.9 TB/s), 725 with the gradient.
//
// A row begins wherever the vocabulary's size puts it: its values are taken 16 bytes at a time at the places where memory has them, and one by one
// in the pieces that it shares with its neighbours.  dz's rows are dense.  Where one of them lies otherwise to a 16-byte boundary than its row of logits (an odd vocabulary as a part of
// a padded head's columns), its values are stored one by one: no slower, 4001 rows of 32001 bf16 176 us forward and back from dense rows, 175 from rows 32008 apart, in fp32 405 and 408.
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ int64_t index_of(const void* p, int wide, int64_t at) {
  return wide ? static_cast<const int64_t*>(p)[at] : (int64_t)static_cast<const int32_t*>(p)[at];
}

// A row as its values before the first 16-byte boundary, its whole pieces, and its values behind the last.
template <typename T>
struct RowPieces {
  static constexpr int E = 16 / sizeof(T);
  int before, pieces, behind, body;   // body: values up to the last whole piece
  __device__ __forceinline__ RowPieces(const T* row, int width) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    before = off == 0 ? 0 : E - off;
    if (before > width) before = width;
    pieces = (width - before) / E;
    body = before + pieces * E;
    behind = width - body;
  }
  // The place of the lone value that falls to a thread (there are less than 2 E of them), or -1
  __device__ __forceinline__ int lone(int thread) const {
    return thread < before ? thread : thread >= E && thread < E + behind ? body + thread - E : -1;
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
// THREADS to a row.  A thread's first entry of the teacher's list, the student's logit there and the label's are asked for ahead of the row, and what is
// left to do behind it is two sums over the work-group.
template <typename T, int THREADS, bool HARD>
__global__ __launch_bounds__(THREADS) void distill_fwd_kernel(const DistillArgs p) {
  constexpr int E = RowPieces<T>::E, AHEAD = 2, WAVES = THREADS / 64;
  __shared__ Sums waves[WAVES];
  __shared__ float highs[WAVES];
  __shared__ double parts[2][WAVES];
  const int64_t row = blockIdx.x;
  const T* const z = static_cast<const T*>(p.logits) + row * p.logits_stride;
  const RowPieces<T> pieces(z, p.vocabulary);
  const float tau = p.temperature, weight = p.label_weight, c = LOG2E / tau;
  const bool teaches = weight != 1.f;
  // groups of pieces THREADS apart, the next one's loads under this one's exponentials
  const uint4* const body = reinterpret_cast<const uint4*>(z + pieces.before);
  uint4 here[AHEAD], next[AHEAD];
  auto fetch = [&](uint4 (&raw)[AHEAD], int i) {   // (past the row: its last piece, for nothing)
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) raw[a] = body[i + a * THREADS < pieces.pieces ? i + a * THREADS : pieces.pieces - 1];
  };
  int64_t label = p.labels && weight != 0.f ? index_of(p.labels, p.labels64, row) : -1;
  const Entry mine = entry_of<T>(p, row, teaches ? (int)threadIdx.x : p.top);
  if (pieces.pieces > 0) fetch(here, threadIdx.x);
  if (label >= p.vocabulary) label = -1;
  const float at_label = label >= 0 ? load_one(z + label) : 0.f, at_mine = mine.there ? load_one(z + mine.id) : 0.f;

  Sums s{-INFINITY, 0.f, 0.f};
  auto take = [&](auto n_c, const uint4* raw) {   // n pieces
    constexpr int A = decltype(n_c)::value;
    float v[A][E], top = s.top;
#pragma unroll
    for (int a = 0; a < A; ++a) load_values<T, E>(v[a], reinterpret_cast<const T*>(raw + a));
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, v[a][e]);
    raise<HARD>(s, top, c);
    const float from = top == -INFINITY ? 0.f : top;   // (nothing but -infinities: their exponentials are zeros)
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s.soft += below(v[a][e], from, c);
        if (HARD) s.hard += below(v[a][e], from, LOG2E);
      }
  };
  int i = threadIdx.x;
  if (pieces.pieces > 0) {
    constexpr int GROUP = AHEAD * THREADS, LAST = (AHEAD - 1) * THREADS;
    while (i + GROUP + LAST < pieces.pieces) {   // two whole groups
      fetch(next, i + GROUP);
      take(IntC<AHEAD>{}, here);
      fetch(here, i + 2 * GROUP);
      take(IntC<AHEAD>{}, next);
      i += 2 * GROUP;
    }
    if (i + LAST < pieces.pieces) {
      take(IntC<AHEAD>{}, here);
      i += GROUP;
    }
    for (; i < pieces.pieces; i += THREADS) {
      const uint4 one = body[i];
      take(IntC<1>{}, &one);
    }
  }
  if (const int at = pieces.lone(threadIdx.x); at >= 0) {
    const float v = load_one(z + at);
    join<HARD>(s, Sums{v, v == -INFINITY ? 0.f : below(v, v, c), v == -INFINITY ? 0.f : below(v, v, c)}, c);   // (1, or NaN of a NaN or an infinity)
  }
  // the teacher's largest entry (a NaN is no largest, and comes out in the sum), with the row's sums
  float high = mine.there ? fmaxf(mine.t, -INFINITY) : -INFINITY;
  if (teaches)
    for (int k = threadIdx.x + THREADS; k < p.top; k += THREADS) {
      const Entry e = entry_of<T>(p, row, k);
      if (e.there) high = fmaxf(high, e.t);
    }
  // The work-group's largest values, then its sums below the largest: one exponential a thread and sum, and one a wave.  (Joined a pair at a time, every pair with its own, and by all
  // threads, that took 8192 rows of 65536 230 us for 217, 16384 of 1000 30 for 26.)
  const float own = s.top;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    s.top = fmaxf(s.top, __shfl_xor(s.top, m));
    high = fmaxf(high, __shfl_xor(high, m));
  }
  auto rescale = [&](float from) {   // (a thread or wave of -infinities has nothing to rescale)
    const bool any = from != -INFINITY;
    s.soft *= any ? below(from, s.top, c) : 1.f;
    if (HARD) s.hard *= any ? below(from, s.top, LOG2E) : 1.f;
  };
  rescale(own);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    s.soft += __shfl_xor(s.soft, m);
    if (HARD) s.hard += __shfl_xor(s.hard, m);
  }
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) {
      waves[threadIdx.x >> 6] = s;
      highs[threadIdx.x >> 6] = high;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      s.top = fmaxf(s.top, waves[w].top);
      high = fmaxf(high, highs[w]);
    }
    if (threadIdx.x < 64) {   // (the first thread has use for them)
      const Sums o = waves[threadIdx.x % WAVES];
      s.soft = o.soft;
      s.hard = o.hard;
      rescale(o.top);
#pragma unroll
      for (int m = 1; m < WAVES; m <<= 1) {
        s.soft += __shfl_xor(s.soft, m);
        if (HARD) s.hard += __shfl_xor(s.hard, m);
      }
    }
  }
  // With e_k = exp((t_k - high) / tau): the sum of e_k, and that of e_k (t_k - high - (z_k - top)).  log p - log q is a difference of numbers much
  // larger than it: in 64 bits.
  double total = 0.0, apart = 0.0;
  auto add = [&](float t, float at) {
    const float e = below(t, high, c);
    total += (double)e;
    if (e != 0.f) apart += (double)e * (((double)t - (double)high) - ((double)at - (double)s.top));   // (what does not weigh may be anywhere)
  };
  if (teaches && (int)(threadIdx.x & ~63u) < p.top) {   // (a wave without entries has nothing to add up)
    if (mine.there) add(mine.t, at_mine);
    for (int k = threadIdx.x + THREADS; k < p.top; k += THREADS) {
      const Entry e = entry_of<T>(p, row, k);
      if (e.there) add(e.t, load_one(z + e.id));
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      total += __shfl_xor(total, m);
      apart += __shfl_xor(apart, m);
    }
  }
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) {
      parts[0][threadIdx.x >> 6] = total;
      parts[1][threadIdx.x >> 6] = apart;
    }
    __syncthreads();
  }
  if (threadIdx.x != 0) return;
  if constexpr (WAVES > 1) {
    total = apart = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { total += parts[0][w]; apart += parts[1][w]; }
  }
  double loss = 0.0;
  if (total != 0.0)   // (NaN: there is something)
    loss = (apart / total / (double)tau + log((double)s.soft) - log(total)) * ((1.0 - (double)weight) * (double)tau * (double)tau);
  if (label >= 0) loss += (double)weight * (log((double)(HARD ? s.hard : s.soft)) + ((double)s.top - (double)at_label));
  p.loss[row] = (float)loss;
  if (p.stats) {
    float4* const stats = reinterpret_cast<float4*>(p.stats + row * DISTILL_STATS);
    stats[0] = make_float4(s.top, 1.f / s.soft, 1.f / (HARD ? s.hard : s.soft), high);
    stats[1] = make_float4(total != 0.0 ? (float)(1.0 / total) : 0.f, 0.f, 0.f, 0.f);
  }
}

// What the entries and the label subtract, by place, for the thread that writes the place: lists in LDS, chained by thread.
// (A place that is named twice stands in them once, with the sum in the list's order: what order the chains come out in changes nothing.)
struct alignas(16) Places {
  static constexpr int MOST = 256;
  int id[MOST], next[MOST];
  float less[MOST];
};

// dz by pieces; what is subtracted at a place is by the thread that has its piece, before it goes.  (As a pass over the entries behind the row, whose lines had left
// the L2, 128 of them cost 8192 rows of 65536 90 us of 484.)  Lists that do not fit LDS are taken that way, a stretch at a time, behind a wait for the
// work-group's stores; every entry looks through the whole list for its place, so that long ones cost their square: 1024 rows of 32000, bf16, forward and back, lists of 128 61 us,
// 512 94, 1024 197, 2048 553, 4096 1900, 8192 7070, of which the forward pass is 20 to 93.
template <typename T, int THREADS, bool HARD>
__global__ __launch_bounds__(THREADS) void distill_bwd_kernel(const DistillArgs p) {
  constexpr int E = RowPieces<T>::E, AHEAD = 2, NONE = 0x7fffffff;
  __shared__ Places places;
  __shared__ int heads[THREADS];
  const int64_t row = blockIdx.x;
  const T* const z = static_cast<const T*>(p.logits) + row * p.logits_stride;
  T* const out = static_cast<T*>(p.dlogits) + row * p.vocabulary;
  const RowPieces<T> pieces(z, p.vocabulary);
  const bool together = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;   // (pieces of both are the same)
  const float tau = p.temperature, c = LOG2E / tau;
  // what does not wait for anything, on its way at once: the first pieces, and the thread's first entry
  const uint4* const body = reinterpret_cast<const uint4*>(z + pieces.before);
  uint4 here[AHEAD], next[AHEAD];
  auto fetch = [&](uint4 (&raw)[AHEAD], int i) {   // (past the row: its last piece, for nothing)
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) raw[a] = body[i + a * THREADS < pieces.pieces ? i + a * THREADS : pieces.pieces - 1];
  };
  const Entry mine = entry_of<T>(p, row, threadIdx.x);
  if (pieces.pieces > 0) fetch(here, threadIdx.x);
  const float4 stat = reinterpret_cast<const float4*>(p.stats + row * DISTILL_STATS)[0];
  const float top = stat.x, high = stat.w, rest = p.stats[row * DISTILL_STATS + 4], g = p.dloss[row];   // rest: 1 / the sum of the teacher's exponentials, 0 where there is none
  int label = -1;
  if (p.labels && p.label_weight != 0.f) {
    const int64_t at = index_of(p.labels, p.labels64, row);
    if (at >= 0 && at < p.vocabulary) label = (int)at;
  }
  const bool teaches = rest != 0.f, counts = teaches || label >= 0;
  const float share = teaches ? g * (1.f - p.label_weight) * tau : 0.f;   // of the entries
  const float right = label >= 0 ? g * p.label_weight : 0.f;              // of the label
  // what q and softmax(z) are multiplied by, over their sums
  const float soft = HARD ? share * stat.y : (share + right) * stat.y, hard = HARD ? right * stat.z : 0.f;
  auto dense = [&](float v) { return soft * below(v, top, c) + (HARD ? hard * below(v, top, LOG2E) : 0.f); };

  // The list: the teacher's entries, the label behind them.
  const int n = teaches ? p.top : 0;
  const float each = teaches ? share * rest : 0.f;
  const bool chained = n + 1 <= Places::MOST;
  auto stretch = [&](int j0) {   // entries j0 .. of the list into LDS
    __syncthreads();
    for (int j = threadIdx.x; j < Places::MOST; j += THREADS) {
      int id = -1;
      float w = 0.f;
      if (j0 + j < n) {
        const Entry e = j0 + j == (int)threadIdx.x ? mine : entry_of<T>(p, row, j0 + j);
        id = e.id;
        if (e.there) w = below(e.t, high, c) * each;
      } else if (j0 + j == n) {
        id = label;
        w = right;
      }
      places.id[j] = id;
      places.less[j] = w;
    }
    __syncthreads();
  };
  // What is subtracted at entry k's place by the stretch in LDS; whether no entry before k has it
  auto gather = [&](int j0, int k, int id, float& sum, bool& first) {
    const int m = n + 1 - j0 < Places::MOST ? n + 1 - j0 : Places::MOST;
    for (int j = 0; j < m; j += 4) {   // (ids of -1 behind the last)
      const int4 four = *reinterpret_cast<const int4*>(places.id + j);
      if (four.x != id && four.y != id && four.z != id && four.w != id) continue;
      const int all[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (all[e] != id) continue;
        sum += places.less[j + e];
        if (j0 + j + e < k) first = false;
      }
    }
  };
  // The piece that a place is in (the lone values: one behind the last), and the thread that writes it
  auto piece_of = [&](int id) { return id < pieces.before || id >= pieces.body ? pieces.pieces : (id - pieces.before) / E; };
  auto writer_of = [&](int id) { return id < pieces.before ? id : id >= pieces.body ? E + id - pieces.body : (id - pieces.before) / E % THREADS; };
  int pending = NONE;
  auto look = [&](int from) {   // the thread's next piece from `from` on
    pending = NONE;
    for (int k = heads[threadIdx.x]; k >= 0; k = places.next[k]) {
      const int at = piece_of(places.id[k]);
      if (at >= from && at < pending) pending = at;
    }
  };
  if (chained && counts) {
    heads[threadIdx.x] = -1;
    stretch(0);
    float sum[(Places::MOST + THREADS - 1) / THREADS];
    bool first[(Places::MOST + THREADS - 1) / THREADS];
#pragma unroll
    for (int q = 0; q < (Places::MOST + THREADS - 1) / THREADS; ++q) {
      const int k = q * THREADS + (int)threadIdx.x;
      sum[q] = 0.f;
      first[q] = k <= n && places.id[k] >= 0;
      if (q * THREADS <= n) gather(0, k, first[q] ? places.id[k] : -2, sum[q], first[q]);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < (Places::MOST + THREADS - 1) / THREADS; ++q) {
      const int k = q * THREADS + (int)threadIdx.x;
      if (!first[q]) continue;
      places.less[k] = sum[q];
      places.next[k] = atomicExch(&heads[writer_of(places.id[k])], k);
    }
    __syncthreads();
    look(0);
  }
  auto give = [&](auto n_c, const uint4* raw, int i) {   // n pieces from i on
    constexpr int A = decltype(n_c)::value;
    float v[A][E];
#pragma unroll
    for (int a = 0; a < A; ++a) load_values<T, E>(v[a], reinterpret_cast<const T*>(raw + a));
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
      for (int e = 0; e < E; ++e) v[a][e] = counts ? dense(v[a][e]) : 0.f;
    if (pending <= i + (A - 1) * THREADS) {
      for (int k = heads[threadIdx.x]; k >= 0; k = places.next[k]) {
        const int id = places.id[k], at = piece_of(id) - i;      // (a multiple of THREADS)
        if (at < 0 || at > (A - 1) * THREADS) continue;
        const int place = at / THREADS * E + (id - pieces.before) % E;
        const float w = places.less[k];
#pragma unroll
        for (int a = 0; a < A; ++a)
#pragma unroll
          for (int e = 0; e < E; ++e) v[a][e] -= place == a * E + e ? w : 0.f;
      }
      look(i + (A - 1) * THREADS + 1);
    }
#pragma unroll
    for (int a = 0; a < A; ++a) {
      T* const to = out + pieces.before + (i + a * THREADS) * E;
      if (together) {
        store_values<T, E>(to, v[a]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) store_one(to + e, v[a][e]);
      }
    }
  };
  int i = threadIdx.x;
  if (pieces.pieces > 0) {
    constexpr int GROUP = AHEAD * THREADS, LAST = (AHEAD - 1) * THREADS;
    while (i + GROUP + LAST < pieces.pieces) {   // two whole groups
      fetch(next, i + GROUP);
      give(IntC<AHEAD>{}, here, i);
      fetch(here, i + 2 * GROUP);
      give(IntC<AHEAD>{}, next, i + GROUP);
      i += 2 * GROUP;
    }
    if (i + LAST < pieces.pieces) {
      give(IntC<AHEAD>{}, here, i);
      i += GROUP;
    }
    for (; i < pieces.pieces; i += THREADS) {
      const uint4 one = body[i];
      give(IntC<1>{}, &one, i);
    }
  }
  if (const int at = pieces.lone(threadIdx.x); at >= 0) {
    float v = counts ? dense(load_one(z + at)) : 0.f;
    if (pending != NONE)
      for (int k = heads[threadIdx.x]; k >= 0; k = places.next[k])
        if (places.id[k] == at) v -= places.less[k];
    store_one(out + at, v);
  }
  if (chained || !counts) return;
  // (a piece's store and a place's of another wave: the first has to have arrived)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int k0 = 0; k0 <= n; k0 += THREADS) {
    const int k = k0 + (int)threadIdx.x;
    const int id = k < n ? entry_of<T>(p, row, k).id : k == n ? label : -1;
    float sum = 0.f;
    bool first = id >= 0;
    for (int j0 = 0; j0 <= n; j0 += Places::MOST) {
      stretch(j0);
      gather(j0, k, first ? id : -2, sum, first);
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
  note_matrix(a.stats, a.rows, DISTILL_STATS, DISTILL_STATS, 4, !back);
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

// Threads to a row.  Short rows are the price of what each has behind (forward) or ahead of (back) its values, and many small work-groups hide it better;
// long ones want few rows at a time.  Bf16, us, 64 : 256 : 512 threads: forward 16384 rows of 1000 26 : 43 : 74, 3000 of 9000 22 : 20 : 22, 4001 of 32001 84 : 81 : 80,
// 8192 of 65536 241 : 227 : 215; back 16384 of 200 20 : 27 : 53, 16384 of 1000 80 : 67 : 121, 4001 of 32001 114 : 96 : 96, 8192 of 65536 466 : 413 : 398.
// Few rows (less than two waves a SIMD at 64 threads): 256, forward 100 of 32000 16 : 9 : 9.
template <typename T, bool HARD, bool BACK>
hipError_t by_size(const DistillArgs& a, hipStream_t s) {
  if (a.vocabulary <= (BACK ? 512 : 6144) && (a.rows >= 8 * NUM_CUS || a.vocabulary <= 512)) return go<T, 64, HARD, BACK>(a, s);
  if (a.vocabulary <= 49152) return go<T, 256, HARD, BACK>(a, s);
  return go<T, 512, HARD, BACK>(a, s);
}
template <typename T, bool BACK>
hipError_t by_sums(const DistillArgs& a, hipStream_t s) {
  // (one sum serves both parts where the temperature is 1, or where one of them is not there)
  return a.labels && a.label_weight != 0.f && a.temperature != 1.f ? by_size<T, true, BACK>(a, s) : by_size<T, false, BACK>(a, s);
}

}  // namespace

hipError_t launch_distill_fwd(const DistillArgs& a, bool f32, hipStream_t s) { return f32 ? by_sums<float, false>(a, s) : by_sums<bf16, false>(a, s); }
hipError_t launch_distill_bwd(const DistillArgs& a, bool f32, hipStream_t s) { return f32 ? by_sums<float, true>(a, s) : by_sums<bf16, true>(a, s); }

}  // namespace sk
