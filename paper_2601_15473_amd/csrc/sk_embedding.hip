// Token embedding with scaling, and its gradient by sorted tokens.
//
// The gradient in three launches: (1) a work-group sorts up to 16384 tokens by id in LDS, while the others fill the
// gradient with zeros; (more tokens: sorted runs, put into one order by a second launch); (2) every run of 32 sorted tokens is
// summed by id, ids wholly inside written, the others' sums left in the workspace; (3) those are added up in order.
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

constexpr int RUN = EMBEDDING_RUN, CHUNK = EMBEDDING_CHUNK;
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, SORT_STEPS = RUN / SORT_THREADS;

__device__ __forceinline__ int64_t id_at(const EmbeddingArgs& p, int64_t t) {
  return p.ids64 ? static_cast<const int64_t*>(p.ids)[t] : static_cast<const int32_t*>(p.ids)[t];
}

template <typename T>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const EmbeddingArgs p) {
  const int per_row = p.width / 8;
  const int64_t pieces = p.tokens * per_row, stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += stride) {
    const int64_t t = i / per_row, c = (i - t * per_row) * 8, id = id_at(p, t);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (id >= 0 && id < p.rows) {
      load_values<T, 8>(v, static_cast<const T*>(p.table) + id * p.width + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= p.scale;
    }
    store_values<T, 8>(static_cast<T*>(p.out) + t * p.width + c, v);
  }
}

// Stable sort of one run by id, least digits of 8 bits first: wave w has a contiguous part, in which a
// lane's place among equal digits is what its wave has counted before plus the equal lanes below it.
struct SortRoom {
  unsigned key[RUN];
  unsigned short from[RUN];
  unsigned count[SORT_WAVES][256];
  unsigned start[256];
  unsigned wave_total[4];
};

__device__ __forceinline__ void sort_run(const EmbeddingArgs& p, SortRoom& m, int run, int digits, unsigned* keys, unsigned* order) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t first = (int64_t)run * RUN;
  const int n = p.tokens - first < RUN ? (int)(p.tokens - first) : RUN;
  const int steps = (n + SORT_THREADS - 1) / SORT_THREADS, begin = wave * steps * 64;
  for (int i = tid; i < n; i += SORT_THREADS) {
    const int64_t id = id_at(p, first + i);
    m.key[i] = id >= 0 && id < p.rows ? (unsigned)id : (unsigned)p.rows;   // (ids without a row come last)
    m.from[i] = (unsigned short)i;
  }
  unsigned key[SORT_STEPS], place[SORT_STEPS];
  unsigned short from[SORT_STEPS];
  for (int digit = 0; digit < digits; ++digit) {
    for (int i = tid; i < SORT_WAVES * 256; i += SORT_THREADS) (&m.count[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s) {
      if (s < steps) {
        const int i = begin + s * 64 + lane;
        const bool there = i < n;
        key[s] = there ? m.key[i] : 0u;
        from[s] = there ? m.from[i] : 0;
        const unsigned d = (key[s] >> (8 * digit)) & 255u;
        uint64_t same = __ballot(there);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
          const uint64_t set = __ballot((d >> b) & 1u);
          same &= ((d >> b) & 1u) ? set : ~set;
        }
        const int below = __popcll(same & ((1ull << lane) - 1));
        unsigned before = 0;
        if (there) before = m.count[wave][d];
        __builtin_amdgcn_wave_barrier();
        if (there && below == 0) m.count[wave][d] = before + (unsigned)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        place[s] = before + below;
      }
    }
    __syncthreads();
    unsigned total = 0, sum = 0;
    if (tid < 256) {   // a digit's waves in turn, then the digits
      for (int w = 0; w < SORT_WAVES; ++w) {
        const unsigned c = m.count[w][tid];
        m.count[w][tid] = total;
        total += c;
      }
      sum = total;
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const unsigned u = __shfl_up(sum, k);
        if (lane >= k) sum += u;
      }
      if (lane == 63) m.wave_total[wave] = sum;
    }
    __syncthreads();
    if (tid < 256) {
      unsigned base = 0;
      for (int w = 0; w < wave; ++w) base += m.wave_total[w];
      m.start[tid] = base + sum - total;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s) {
      if (s < steps && begin + s * 64 + lane < n) {
        const unsigned d = (key[s] >> (8 * digit)) & 255u;
        const unsigned to = m.start[d] + m.count[wave][d] + place[s];
        m.key[to] = key[s];
        m.from[to] = from[s];
      }
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += SORT_THREADS) {
    keys[first + i] = m.key[i];
    order[first + i] = (unsigned)first + m.from[i];
  }
}

__global__ __launch_bounds__(SORT_THREADS) void embedding_sort_kernel(const EmbeddingArgs p, int runs, int digits, int64_t bytes) {
  __shared__ SortRoom room;
  if ((int)blockIdx.x < runs) {
    sort_run(p, room, blockIdx.x, digits, runs > 1 ? p.keys_runs : p.keys, runs > 1 ? p.order_runs : p.order);
  } else {
    const int64_t stride = (int64_t)(gridDim.x - runs) * SORT_THREADS;
    for (int64_t i = (int64_t)(blockIdx.x - runs) * SORT_THREADS + threadIdx.x; i < bytes / 16; i += stride)
      static_cast<uint4*>(p.out)[i] = make_uint4(0, 0, 0, 0);
  }
}

// Keys of keys[0 .. n - 1] (sorted) below `key`, or with `equal` not above it.
__device__ __forceinline__ int64_t keys_below(const unsigned* keys, int64_t n, unsigned key, bool equal) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (keys[mid] < key || (equal && keys[mid] == key)) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// A token's place among all runs: its own run's tokens before it, and the other runs' that go before it.
__global__ __launch_bounds__(256) void embedding_merge_kernel(const EmbeddingArgs p, int runs) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.tokens) return;
  const int run = (int)(i / RUN);
  const unsigned key = p.keys_runs[i];
  int64_t to = i - (int64_t)run * RUN;
  for (int r = 0; r < runs; ++r) {
    if (r == run) continue;
    const int64_t first = (int64_t)r * RUN, n = p.tokens - first < RUN ? p.tokens - first : RUN;
    to += keys_below(p.keys_runs + first, n, key, r < run);
  }
  p.keys[to] = key;
  p.order[to] = p.order_runs[i];
}

// Eight columns a thread, `threads` of them to a chunk.
template <typename T>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbeddingArgs p, int threads, int blocks, int64_t chunks) {
  const int per = 256 / threads, sub = threadIdx.x / threads;
  const int64_t id = blockIdx.x / blocks;
  const int64_t chunk = id * per + sub;
  const int column = ((int)(blockIdx.x - id * blocks) * threads + threadIdx.x - sub * threads) * 8;
  if (sub >= per || chunk >= chunks || column >= p.width) return;
  const int64_t first = chunk * CHUNK;
  const int n = p.tokens - first < CHUNK ? (int)(p.tokens - first) : CHUNK;
  const unsigned* const keys = p.keys + first;
  const unsigned* const order = p.order + first;
  bool head = first > 0 && keys[-1] == keys[0];   // of an id that began before
  const bool open = first + n < p.tokens && keys[n] == keys[n - 1];
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  constexpr int AT_ONCE = 8;
  for (int i0 = 0; i0 < n; i0 += AT_ONCE) {
    float v[AT_ONCE][8];
    unsigned key[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {   // (past the chunk: its last token again)
      const int i = i0 + k < n ? i0 + k : n - 1;
      key[k] = keys[i];
      load_values<T, 8>(v[k], static_cast<const T*>(p.dy) + (int64_t)order[i] * p.width + column);
    }
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int i = i0 + k;
      if (i >= n) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[k][j];
      const bool last = i == n - 1;
      if (!last && (k + 1 < AT_ONCE ? key[k + 1 < AT_ONCE ? k + 1 : 0] : keys[i + 1]) == key[k]) continue;
      if (head || (last && open)) {
        store_values<float, 8>(p.partial + (chunk * 2 + (head ? 0 : 1)) * p.width + column, acc);
      } else if (key[k] < p.rows) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] *= p.scale;
        store_values<T, 8>(static_cast<T*>(p.out) + (int64_t)key[k] * p.width + column, acc);
      }
      head = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    }
  }
}

// The id that begins in a chunk and goes on behind it: its chunks' sums, dealt over four waves and joined in their order.
template <typename T>
__global__ __launch_bounds__(256) void embedding_join_kernel(const EmbeddingArgs p, int blocks) {
  __shared__ float4 sums[4][64];
  const int64_t chunk = blockIdx.x / blocks, first = chunk * CHUNK, next = first + CHUNK;
  const unsigned key = p.keys[next - 1];
  if (p.keys[next] != key || key >= p.rows || (first > 0 && p.keys[first] == key && p.keys[first - 1] == key)) return;   // (uniform)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int column = ((int)(blockIdx.x - chunk * blocks) * 64 + lane) * 4;
  const bool there = column < p.width;
  const int64_t last = (next + keys_below(p.keys + next, p.tokens - next, key, true) - 1) / CHUNK;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (there) {
#pragma unroll 4
    for (int64_t c = chunk + wave; c <= last; c += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p.partial + (c * 2 + (c == chunk ? 1 : 0)) * p.width + column);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && there) {
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const float4 v = sums[w][lane];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const float out[4] = {s.x * p.scale, s.y * p.scale, s.z * p.scale, s.w * p.scale};
    store_values<T, 4>(static_cast<T*>(p.out) + (int64_t)key * p.width + column, out);
  }
}

template <typename T>
hipError_t fwd(const EmbeddingArgs& a, hipStream_t s) {
  const int64_t pieces = a.tokens * (a.width / 8), groups = (pieces + 255) / 256;
  note_matrix(a.ids, 1, a.tokens, a.tokens, a.ids64 ? 8 : 4, false);
  note_matrix(a.table, a.rows, a.width, a.width, sizeof(T), false);
  note_matrix(a.out, a.tokens, a.width, a.width, sizeof(T), true);
  return launch_kernel("embedding_fwd_kernel", Work{0.0, 2.0 * a.tokens * a.width * sizeof(T)}, embedding_fwd_kernel<T>,
                       dim3((unsigned)(groups < 16 * NUM_CUS ? groups : 16 * NUM_CUS)), dim3(256), s, a);
}

template <typename T>
hipError_t bwd(const EmbeddingArgs& a, hipStream_t s) {
  const int runs = (int)((a.tokens + RUN - 1) / RUN);
  int digits = 1;
  while (digits < 4 && (uint64_t)a.rows >> (8 * digits) != 0) ++digits;
  const int64_t bytes = a.rows * a.width * (int64_t)sizeof(T);
  const int64_t chunks = (a.tokens + CHUNK - 1) / CHUNK;
  unsigned* const keys = runs > 1 ? a.keys_runs : a.keys;
  unsigned* const order = runs > 1 ? a.order_runs : a.order;
  note_matrix(a.ids, 1, a.tokens, a.tokens, a.ids64 ? 8 : 4, false);
  note_matrix(keys, 1, a.tokens, a.tokens, 4, true);
  note_matrix(order, 1, a.tokens, a.tokens, 4, true);
  note_matrix(a.out, a.rows, a.width, a.width, sizeof(T), true);
  const int64_t fill = (bytes / 16 + SORT_THREADS * 8 - 1) / (SORT_THREADS * 8);
  hipError_t e = launch_kernel("embedding_sort_kernel", Work{0.0, (double)bytes}, embedding_sort_kernel,
                               dim3((unsigned)(runs + (fill < NUM_CUS * 4 ? fill : NUM_CUS * 4))), dim3(SORT_THREADS), s, a, runs, digits, bytes);
  if (e != hipSuccess) return e;
  if (runs > 1) {
    note_matrix(keys, 1, a.tokens, a.tokens, 4, false);
    note_matrix(order, 1, a.tokens, a.tokens, 4, false);
    note_matrix(a.keys, 1, a.tokens, a.tokens, 4, true);
    note_matrix(a.order, 1, a.tokens, a.tokens, 4, true);
    e = launch_kernel("embedding_merge_kernel", Work{0.0, 16.0 * a.tokens}, embedding_merge_kernel, dim3((unsigned)((a.tokens + 255) / 256)), dim3(256), s, a, runs);
    if (e != hipSuccess) return e;
  }
  note_matrix(a.keys, 1, a.tokens, a.tokens, 4, false);
  note_matrix(a.order, 1, a.tokens, a.tokens, 4, false);
  note_matrix(a.dy, a.tokens, a.width, a.width, sizeof(T), false);
  note_matrix(a.out, a.rows, a.width, a.width, sizeof(T), true);
  note_matrix(a.partial, chunks * 2, a.width, a.width, 4, true);
  const int columns = a.width / 8, threads = columns < 256 ? columns : 256, blocks = (columns + threads - 1) / threads, per = 256 / threads;
  e = launch_kernel("embedding_sum_kernel", Work{0.0, 2.0 * a.tokens * a.width * sizeof(T)}, embedding_sum_kernel<T>,
                    dim3((unsigned)((chunks + per - 1) / per * blocks)), dim3(256), s, a, threads, blocks, chunks);
  if (e != hipSuccess || chunks == 1) return e;
  note_matrix(a.keys, 1, a.tokens, a.tokens, 4, false);
  note_matrix(a.partial, chunks * 2, a.width, a.width, 4, false);
  note_matrix(a.out, a.rows, a.width, a.width, sizeof(T), true);
  const int join_blocks = (a.width + 255) / 256;
  return launch_kernel("embedding_join_kernel", Work{0.0, 0.0}, embedding_join_kernel<T>, dim3((unsigned)((chunks - 1) * join_blocks)), dim3(256), s, a, join_blocks);
}

}  // namespace

hipError_t launch_embedding_fwd(const EmbeddingArgs& a, bool f32, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_embedding_bwd(const EmbeddingArgs& a, bool f32, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace sk
