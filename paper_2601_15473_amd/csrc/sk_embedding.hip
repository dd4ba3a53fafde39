// Token embedding with scaling, and its gradient by sorted tokens: y_t = scale table[id_t], dtable_v = scale sum of dY_t over the t with
// id_t = v, in the order of t (no atomics: the same bits every run).  Both are bound by memory: 16384 tokens of 4096 features in bf16 forward 40 us
// (268 MB moved, fewer read where tokens repeat), on 65536 rows the gradient 77 + 69 + 7 us, 537 of whose 730 MB are its zeros: they leave at 6.9 TB/s, but
// half of them only as far as the Infinity Cache, which the rows of dY then push them out of.
//
// The gradient in three launches: (1) a work-group sorts up to 16384 tokens by id in LDS, while the others fill the
// gradient with zeros; (more tokens: sorted runs, put into one order by a second launch); (2) every run of 16 or 32 sorted tokens is
// summed by id, ids wholly inside written, the others' sums left in the workspace; (3) those are added up in order.
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

constexpr int RUN = EMBEDDING_RUN;
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, SORT_STEPS = RUN / SORT_THREADS, FILL_PIECES = 4 * SORT_THREADS;

__device__ __forceinline__ int64_t id_at(const EmbeddingArgs& p, int64_t t) {
  return p.ids64 ? static_cast<const int64_t*>(p.ids)[t] : static_cast<const int32_t*>(p.ids)[t];
}

// `threads` of a work-group to a row, 16 bytes a thread and step; four steps are on their way at once, of ROWS rows (narrow ones, whose ids are
// the first trip to memory of two).
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const EmbeddingArgs p, int threads) {
  constexpr int V = 16 / sizeof(T), STEPS = 4 / ROWS;
  const int subs = 256 / threads, sub = threadIdx.x / threads, first = (threadIdx.x - sub * threads) * V, step = threads * V;
  const int64_t t0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * subs * ROWS + sub;
  const T* from[ROWS];
  bool there[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t t = t0 + r * subs, id = id_at(p, t < p.tokens ? t : p.tokens - 1);
    there[r] = id >= 0 && id < p.rows;
    from[r] = static_cast<const T*>(p.table) + (there[r] ? id : 0) * p.width;
  }
  for (int c0 = first; c0 < p.width; c0 += STEPS * step) {
    float v[ROWS][STEPS][V];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int k = 0; k < STEPS; ++k) load_values<T, V>(v[r][k], from[r] + (c0 + k * step < p.width ? c0 + k * step : c0));
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const int64_t t = t0 + r * subs;
#pragma unroll
        for (int j = 0; j < V; ++j) v[r][k][j] = there[r] ? v[r][k][j] * p.scale : 0.f;
        if (t < p.tokens && c0 + k * step < p.width) store_values<T, V>(static_cast<T*>(p.out) + t * p.width + c0 + k * step, v[r][k]);
      }
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
  const int64_t first = (int64_t)run * p.run;
  const int n = p.tokens - first < p.run ? (int)(p.tokens - first) : p.run;
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
    // 64 KB at a time
    const int64_t pieces = bytes / 16, stride = (int64_t)(gridDim.x - runs) * FILL_PIECES;
    for (int64_t i0 = (int64_t)(blockIdx.x - runs) * FILL_PIECES; i0 < pieces; i0 += stride)
#pragma unroll
      for (int k = 0; k < FILL_PIECES; k += SORT_THREADS)
        if (i0 + k + threadIdx.x < pieces) static_cast<uint4*>(p.out)[i0 + k + threadIdx.x] = make_uint4(0, 0, 0, 0);
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
  const int run = (int)(i / p.run);
  const unsigned key = p.keys_runs[i];
  int64_t to = i - (int64_t)run * p.run;
  for (int r = 0; r < runs; ++r) {
    if (r == run) continue;
    const int64_t first = (int64_t)r * p.run, n = p.tokens - first < p.run ? p.tokens - first : p.run;
    to += keys_below(p.keys_runs + first, n, key, r < run);
  }
  p.keys[to] = key;
  p.order[to] = p.order_runs[i];
}

// G lanes of a wave, 16 bytes each, sum a chunk's columns: its tokens and their order in one load, then 16 rows on their way at a time.
template <typename T, int G, int CHUNK>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbeddingArgs p, int blocks, int64_t chunks) {
  constexpr int V = 16 / sizeof(T), AT_ONCE = 16, HELD = (CHUNK + G - 1) / G;
  const int lane = threadIdx.x & 63, l = lane % G;
  const int64_t unit = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / G) + lane / G;   // (all of a chunk's column blocks in a row)
  const int64_t chunk = unit / blocks;
  const int column = ((int)(unit - chunk * blocks) * G + l) * V;
  const bool there = chunk < chunks && column < p.width;
  const int64_t first = (chunk < chunks ? chunk : 0) * CHUNK;
  const int n = p.tokens - first < CHUNK ? (int)(p.tokens - first) : CHUNK;
  unsigned key[HELD], from[HELD];
#pragma unroll
  for (int h = 0; h < HELD; ++h) {   // (past the chunk: its last token again)
    const int i = h * G + l < n ? h * G + l : n - 1;
    key[h] = p.keys[first + i];
    from[h] = p.order[first + i];
  }
  const unsigned before = first > 0 ? p.keys[first - 1] : ~0u, behind = first + n < p.tokens ? p.keys[first + n] : ~0u;   // (no key: ids are below 2^31)
  auto held = [&](const unsigned (&v)[HELD], int i) { return (unsigned)__shfl((int)v[i / G], i % G, G); };
  const T* const dy = static_cast<const T*>(p.dy) + (there ? column : 0);
  bool head = before == held(key, 0);   // of an id that began before
  float acc[V];
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] = 0.f;
#pragma unroll
  for (int i0 = 0; i0 < CHUNK; i0 += AT_ONCE) {
    if (i0 > 0 && i0 >= n) break;
    float v[AT_ONCE][V];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) load_values<T, V>(v[k], dy + (int64_t)held(from, i0 + k) * p.width);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int i = i0 + k;
      if (i >= n) break;
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += v[k][j];
      const unsigned now = held(key, i), next = i == n - 1 ? behind : held(key, i + 1 < CHUNK ? i + 1 : i);
      if (next == now && i < n - 1) continue;
      if (head || next == now) {
        if (there) store_values<float, V>(p.partial + (chunk * 2 + (head ? 0 : 1)) * p.width + column, acc);
      } else if (now < p.rows && there) {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] *= p.scale;
        store_values<T, V>(static_cast<T*>(p.out) + (int64_t)now * p.width + column, acc);
      }
      head = false;
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] = 0.f;
    }
  }
}

// The id that begins in a chunk and goes on behind it: its chunks' sums, dealt over four waves and joined in their order.  Most chunks have
// none: the launch's own time and two trips to memory (16384 tokens of 4096 features 7 us, 11 with the id's end looked for by halves).
template <typename T>
__global__ __launch_bounds__(256) void embedding_join_kernel(const EmbeddingArgs p, int blocks, int run) {
  __shared__ float4 sums[4][64];
  const int64_t chunk = blockIdx.x / blocks, first = chunk * run, next = first + run;
  const unsigned key = p.keys[next - 1];
  if (p.keys[next] != key || key >= p.rows || (first > 0 && p.keys[first] == key && p.keys[first - 1] == key)) return;   // (uniform)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int column = ((int)(blockIdx.x - chunk * blocks) * 64 + lane) * 4;
  const bool there = column < p.width;
  int64_t last = chunk;   // the id's last chunk: those that begin with it, a lane to each
  for (uint64_t same = ~0ull; same == ~0ull;) {
    const int64_t at = (last + 1 + lane) * run;
    same = __ballot(at < p.tokens && p.keys[at < p.tokens ? at : 0] == key);
    last += same == ~0ull ? 64 : __builtin_ctzll(~same);
  }
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
  int threads = 8;
  while (threads < 256 && threads * 16 < a.width * (int)sizeof(T)) threads *= 2;
  note_matrix(a.ids, 1, a.tokens, a.tokens, a.ids64 ? 8 : 4, false);
  note_matrix(a.table, a.rows, a.width, a.width, sizeof(T), false);
  note_matrix(a.out, a.tokens, a.width, a.width, sizeof(T), true);
  // rows to a thread: as many as leave it four steps, and every CU eight work-groups
  const int steps = (a.width * (int)sizeof(T) / 16 + threads - 1) / threads, subs = 256 / threads;
  const int most = (int)(a.tokens / (8 * NUM_CUS * subs)), rows = steps == 1 && most >= 4 ? 4 : steps <= 2 && most >= 2 ? 2 : 1;
  const int64_t groups = (a.tokens + subs * rows - 1) / (subs * rows), along = groups < 1 << 23 ? groups : 1 << 23;   // (a dimension takes 2^32 threads)
  return launch_kernel("embedding_fwd_kernel", Work{0.0, 2.0 * a.tokens * a.width * sizeof(T)},
                       rows == 4 ? embedding_fwd_kernel<T, 4> : rows == 2 ? embedding_fwd_kernel<T, 2> : embedding_fwd_kernel<T, 1>,
                       dim3((unsigned)along, (unsigned)((groups + along - 1) / along)), dim3(256), s, a, threads);
}

template <typename T>
hipError_t bwd(const EmbeddingArgs& a, hipStream_t s) {
  const int runs = (int)((a.tokens + a.run - 1) / a.run);
  int digits = 1;
  while (digits < 4 && (uint64_t)a.rows >> (8 * digits) != 0) ++digits;
  const int64_t bytes = a.rows * a.width * (int64_t)sizeof(T);
  const int chunk = embedding_chunk(a.tokens, a.width, sizeof(T));
  const int64_t chunks = (a.tokens + chunk - 1) / chunk;
  unsigned* const keys = runs > 1 ? a.keys_runs : a.keys;
  unsigned* const order = runs > 1 ? a.order_runs : a.order;
  note_matrix(a.ids, 1, a.tokens, a.tokens, a.ids64 ? 8 : 4, false);
  note_matrix(keys, 1, a.tokens, a.tokens, 4, true);
  note_matrix(order, 1, a.tokens, a.tokens, 4, true);
  note_matrix(a.out, a.rows, a.width, a.width, sizeof(T), true);
  const int64_t fill = (bytes / 16 + FILL_PIECES - 1) / FILL_PIECES;
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
  auto sum = [&](auto g) {
    constexpr int G = decltype(g)::value;
    const int blocks = (a.width * (int)sizeof(T) / 16 + G - 1) / G;
    return launch_kernel("embedding_sum_kernel", Work{0.0, 2.0 * a.tokens * a.width * sizeof(T)}, chunk == 32 ? embedding_sum_kernel<T, G, 32> : embedding_sum_kernel<T, G, 16>,
                         dim3((unsigned)((chunks * blocks + 4 * (64 / G) - 1) / (4 * (64 / G)))), dim3(256), s, a, blocks, chunks);
  };
  const int lanes = a.width * (int)sizeof(T) / 16;
  e = lanes <= 8 ? sum(IntC<8>{}) : lanes <= 16 ? sum(IntC<16>{}) : lanes <= 32 ? sum(IntC<32>{}) : sum(IntC<64>{});
  if (e != hipSuccess || chunks == 1) return e;
  note_matrix(a.keys, 1, a.tokens, a.tokens, 4, false);
  note_matrix(a.partial, chunks * 2, a.width, a.width, 4, false);
  note_matrix(a.out, a.rows, a.width, a.width, sizeof(T), true);
  const int join_blocks = (a.width + 255) / 256;
  return launch_kernel("embedding_join_kernel", Work{0.0, 0.0}, embedding_join_kernel<T>, dim3((unsigned)((chunks - 1) * join_blocks)), dim3(256), s, a, join_blocks, chunk);
}

}  // namespace

hipError_t launch_embedding_fwd(const EmbeddingArgs& a, bool f32, hipStream_t s) { return f32 ? fwd<float>(a, s) : fwd<bf16>(a, s); }
hipError_t launch_embedding_bwd(const EmbeddingArgs& a, bool f32, hipStream_t s) { return f32 ? bwd<float>(a, s) : bwd<bf16>(a, s); }

}  // namespace sk
