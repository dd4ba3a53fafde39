// Attention and its gradients in fp32, the accuracy path, and which type's kernels a call goes to (see sk_attention.h for the
// operands' layouts).
//
// Forward, a wave to 32 rows (query, head of the group): s^T = K q^T has a row's scores in its own lane (and the lane 32
// further), so the running maximum and sum of the softmax are registers; o^T += V^T p^T.  Backward, no atomics: dq by the same walk
// over the keys with p from lse, dk and dv by a walk over the queries for 32 keys a wave.  Tiles of 32 keys (queries) go through
// registers into LDS, one at a time: with fp32 products at a sixteenth of the bf16 ones' rate a wave has 4096 cycles of them a tile at 64 features,
// and the matrix unit is the bound (16 sequences of 512, eight heads of 64, forward and backward: 389 us, 77 TFLOP/s of the 14 flops a pair and feature,
// 99 of what is executed, where the library's product reaches 146).
#include "sk_attention.h"

namespace sk {
namespace {

constexpr int ROWS = 32;   // rows of a staged tile

// Rows row0 .. + 31 of `base` (rows `stride` elements apart, D values each) into LDS, zeros at and past row `rows` and past D.
template <int DP>
__device__ __forceinline__ void stage(float* tile, const float* base, int64_t stride, int row0, int rows, int D, int tid) {
  typedef Mma<float> M;
  constexpr int PIECES = DP / M::E, LD = DP + M::E;
#pragma unroll
  for (int i = 0; i < ROWS * PIECES / 256; ++i) {
    const int piece = i * 256 + tid, row = piece / PIECES, c = piece % PIECES * M::E;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (row0 + row < rows && c < D) v = *reinterpret_cast<const uint4*>(base + (row0 + row) * stride + c);
    *reinterpret_cast<uint4*>(tile + row * LD + c) = v;
  }
}

// A lane's row as fragments of a product's second operand: zeros past D and where the row is not there.
template <int DP>
__device__ __forceinline__ void load_row(typename Mma<float>::Frag (&f)[DP / Mma<float>::STEP], const float* row, bool there, int D, int lane) {
  typedef Mma<float> M;
#pragma unroll
  for (int ks = 0; ks < DP / M::STEP; ++ks) {
    const int c = ks * M::STEP + (lane >> 5) * M::E;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (there && c < D) v = *reinterpret_cast<const uint4*>(row + c);
    f[ks] = __builtin_bit_cast(typename M::Frag, v);
  }
}

// [DP x 32] with a row of the result to a lane, as rows of D values; nothing where `row` is null
template <int DP>
__device__ __forceinline__ void store_row(float* row, const f32x16 (&acc)[DP / 32], float scale, int D, int lane) {
  if (row == nullptr) return;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = d * 32 + 8 * g + 4 * (lane >> 5);
      if (c < D) *reinterpret_cast<f32x4*>(row + c) = f32x4{acc[d][4 * g] * scale, acc[d][4 * g + 1] * scale, acc[d][4 * g + 2] * scale, acc[d][4 * g + 3] * scale};
    }
}

// Work-group -> (sequence, key head, tile); neighbours on one XCD share keys and values.
__device__ __forceinline__ void locate(const AttentionArgs& p, int tiles, int& b, int& hk, int& tile) {
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  tile = id % tiles;
  hk = id / tiles % p.kv_heads;
  b = id / tiles / p.kv_heads;
}

// A lane's row of the packed rows (query, head of the group) of a key head.
struct Row {
  int i, h;
  bool there;
  __device__ __forceinline__ Row(const AttentionArgs& p, int r, int hk) {
    i = r / p.group;
    h = hk * p.group + (r - i * p.group);
    there = i < p.q_len;
  }
};

template <int DP>
__global__ __launch_bounds__(256) void attention_fwd_f32_kernel(const AttentionArgs p, int tiles) {
  typedef Mma<float> M;
  constexpr int KS = DP / M::STEP, LD = DP + M::E;
  __shared__ __align__(16) float k_tile[ROWS * LD];
  __shared__ __align__(16) float v_tile[ROWS * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int b, hk, tile;
  locate(p, tiles, b, hk, tile);
  const Sequence q(p, b);
  const int r0 = tile * 128;
  const Row row(p, r0 + wave * 32 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  const int keys = q.seen(r0 / p.group, (r0 + 127) / p.group);

  typename M::Frag qf[KS];
  load_row<DP>(qf, static_cast<const float*>(p.q) + b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], row.there && row.i < q.n, p.D, lane);
  f32x16 o[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) o[d] = zeros();
  float top = -INFINITY, sum = 0.f;
  const float c = p.scale * LOG2E;
  const float* const kb = static_cast<const float*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const float* const vb = static_cast<const float*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  for (int j0 = 0; j0 < keys; j0 += ROWS) {
    __syncthreads();
    stage<DP>(k_tile, kb, p.ks[1], j0, q.m, p.D, tid);
    stage<DP>(v_tile, vb, p.vs[1], j0, q.m, p.D, tid);
    __syncthreads();
    f32x16 s = zeros();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s = M::mma(M::along(k_tile, LD, 0, ks, lane), qf[ks], s);
    float m = top;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = j0 + acc_row(r, lane) < limit ? s[r] * c : -INFINITY;
      m = fmaxf(m, s[r]);
    }
    m = fmaxf(m, other_half(m));
    const float base = m == -INFINITY ? 0.f : m;   // (a row that has seen nothing: exp2(-inf) are its weights)
    const float keep = __builtin_amdgcn_exp2f(top - base);
    top = m;
    sum *= keep;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(s[r] - base);
      sum += s[r];
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] *= keep;
#pragma unroll
      for (int t = 0; t < 32 / M::STEP; ++t) o[d] = M::mma(M::across(v_tile, LD, 0, t, d * 32, lane), M::of_acc(s, t), o[d]);
    }
  }
  sum += other_half(sum);
  zeros_unless(sum != 0.f, o);
  if (row.there) {
    store_row<DP>(static_cast<float*>(p.o) + (((int64_t)b * p.q_len + row.i) * p.heads + row.h) * p.D, o, sum == 0.f ? 0.f : 1.f / sum, p.D, lane);
    if (p.lse != nullptr && lane < 32)
      p.lse[((int64_t)b * p.heads + row.h) * p.q_len + row.i] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
  }
}

template <int DP>
__global__ __launch_bounds__(256) void attention_dq_f32_kernel(const AttentionArgs p, int tiles) {
  typedef Mma<float> M;
  constexpr int KS = DP / M::STEP, LD = DP + M::E;
  __shared__ __align__(16) float k_tile[ROWS * LD];
  __shared__ __align__(16) float v_tile[ROWS * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int b, hk, tile;
  locate(p, tiles, b, hk, tile);
  const Sequence q(p, b);
  const int r0 = tile * 128;
  const Row row(p, r0 + wave * 32 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  const int keys = q.seen(r0 / p.group, (r0 + 127) / p.group);
  const bool counts = limit > 0;   // (of a row that sees nothing, not what came back for it either)

  typename M::Frag qf[KS], gf[KS];
  const int64_t at = (((int64_t)b * p.q_len + row.i) * p.heads + row.h) * p.D;
  const int64_t stat = ((int64_t)b * p.heads + row.h) * p.q_len + row.i;
  load_row<DP>(qf, static_cast<const float*>(p.q) + b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], counts, p.D, lane);
  load_row<DP>(gf, static_cast<const float*>(p.d_o) + at, counts, p.D, lane);
  float delta = 0.f;
  {
    typename M::Frag of[KS];
    load_row<DP>(of, static_cast<const float*>(p.o_in) + at, counts, p.D, lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) delta -= M::dot(of[ks], gf[ks]);
  }
  delta += other_half(delta);
  // (a row that sees nothing has no probabilities, whatever its lse says)
  const float lse = counts ? p.lse[stat] * LOG2E : INFINITY;
  if (row.there && lane < 32) {
    p.lse2[stat] = lse;
    p.delta[stat] = delta;
  }
  f32x16 dq[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dq[d] = zeros();
  const float c = p.scale * LOG2E;
  const float* const kb = static_cast<const float*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const float* const vb = static_cast<const float*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  for (int j0 = 0; j0 < keys; j0 += ROWS) {
    __syncthreads();
    stage<DP>(k_tile, kb, p.ks[1], j0, q.m, p.D, tid);
    stage<DP>(v_tile, vb, p.vs[1], j0, q.m, p.D, tid);
    __syncthreads();
    f32x16 s = zeros(), g = zeros();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      s = M::mma(M::along(k_tile, LD, 0, ks, lane), qf[ks], s);
      g = M::mma(M::along(v_tile, LD, 0, ks, lane), gf[ks], g);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float w = j0 + acc_row(r, lane) < limit ? __builtin_amdgcn_exp2f(s[r] * c - lse) : 0.f;
      s[r] = w * (g[r] + delta);
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int t = 0; t < 32 / M::STEP; ++t) dq[d] = M::mma(M::across(k_tile, LD, 0, t, d * 32, lane), M::of_acc(s, t), dq[d]);
  }
  zeros_unless(counts, dq);
  store_row<DP>(row.there ? static_cast<float*>(p.dq) + at : nullptr, dq, p.scale, p.D, lane);
}

template <int DP>
__global__ __launch_bounds__(256) void attention_dkv_f32_kernel(const AttentionArgs p, int tiles) {
  typedef Mma<float> M;
  constexpr int KS = DP / M::STEP, LD = DP + M::E;
  __shared__ __align__(16) float q_tile[ROWS * LD];
  __shared__ __align__(16) float g_tile[ROWS * LD];
  __shared__ float lse_tile[ROWS], delta_tile[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int b, hk, tile;
  locate(p, tiles * p.parts, b, hk, tile);
  const int part = tile / tiles;
  tile -= part * tiles;
  const Sequence q(p, b);
  const int j0 = tile * 128, j = j0 + wave * 32 + (lane & 31);
  const bool there = j < q.m;
  // the first query that sees key j, and the work-group's first (no earlier one, whose dO need not be a number if it sees nothing)
  const int first = q.causal ? j - q.shift + 1 : 0;
  const int i_begin = j0 >= q.m ? q.n : q.causal && j0 - q.shift + 1 > 0 ? j0 - q.shift + 1 : 0;

  typename M::Frag kf[KS], vf[KS];
  load_row<DP>(kf, static_cast<const float*>(p.k) + b * p.ks[0] + j * p.ks[1] + hk * p.ks[2], there, p.D, lane);
  load_row<DP>(vf, static_cast<const float*>(p.v) + b * p.vs[0] + j * p.vs[1] + hk * p.vs[2], there, p.D, lane);
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = zeros();
  const float c = p.scale * LOG2E;
  // this part's tiles of all heads' (one head's behind the other's)
  const int per_head = q.n > i_begin ? (q.n - i_begin + ROWS - 1) / ROWS : 0, all = per_head * p.group;
  const int begin = (int)((int64_t)all * part / p.parts), end = (int)((int64_t)all * (part + 1) / p.parts);
  for (int gh = 0; gh < p.group; ++gh) {
    const int h = hk * p.group + gh;
    const float* const qb = static_cast<const float*>(p.q) + b * p.qs[0] + h * p.qs[2];
    const float* const gb = static_cast<const float*>(p.d_o) + ((int64_t)b * p.q_len * p.heads + h) * p.D;
    const float* const lse = p.lse2 + ((int64_t)b * p.heads + h) * p.q_len;
    const float* const delta = p.delta + ((int64_t)b * p.heads + h) * p.q_len;
    const int from = begin - gh * per_head > 0 ? begin - gh * per_head : 0, to = end - gh * per_head < per_head ? end - gh * per_head : per_head;
    for (int step = from; step < to; ++step) {
      const int i0 = i_begin + step * ROWS;
      __syncthreads();
      stage<DP>(q_tile, qb, p.qs[1], i0, q.n, p.D, tid);
      stage<DP>(g_tile, gb, (int64_t)p.heads * p.D, i0, q.n, p.D, tid);
      if (tid < ROWS) {
        lse_tile[tid] = i0 + tid < q.n ? lse[i0 + tid] : INFINITY;
        delta_tile[tid] = i0 + tid < q.n ? delta[i0 + tid] : 0.f;
      }
      __syncthreads();
      f32x16 s = zeros(), g = zeros();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = M::mma(M::along(q_tile, LD, 0, ks, lane), kf[ks], s);
        g = M::mma(M::along(g_tile, LD, 0, ks, lane), vf[ks], g);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = acc_row(r, lane);
        s[r] = there && i0 + i >= first && i0 + i < q.n ? __builtin_amdgcn_exp2f(s[r] * c - lse_tile[i]) : 0.f;
        g[r] = s[r] * (g[r] + delta_tile[i]);
      }
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int t = 0; t < 32 / M::STEP; ++t) {
          dv[d] = M::mma(M::across(g_tile, LD, 0, t, d * 32, lane), M::of_acc(s, t), dv[d]);
          dk[d] = M::mma(M::across(q_tile, LD, 0, t, d * 32, lane), M::of_acc(g, t), dk[d]);
        }
    }
  }
  const int64_t at = (((int64_t)b * p.k_len + j) * p.kv_heads + hk) * p.D;
  zeros_unless(there, dk);
  zeros_unless(there, dv);
  if (p.parts > 1) {
    const int64_t values = (int64_t)p.batch * p.k_len * p.kv_heads * p.D;
    float* const to = p.partial + part * 2 * values + at;
    store_row<DP>(j < p.k_len ? to : nullptr, dk, 1.f, p.D, lane);
    store_row<DP>(j < p.k_len ? to + values : nullptr, dv, 1.f, p.D, lane);
    return;
  }
  store_row<DP>(j < p.k_len ? static_cast<float*>(p.dk) + at : nullptr, dk, p.scale, p.D, lane);
  store_row<DP>(j < p.k_len ? static_cast<float*>(p.dv) + at : nullptr, dv, 1.f, p.D, lane);
}

double pairs(const AttentionArgs& a) { return (double)a.batch * a.q_len * a.heads * a.k_len * a.D; }

template <int DP>
hipError_t fwd(const AttentionArgs& a, hipStream_t s) {
  const int tiles = ((int64_t)a.q_len * a.group + 127) / 128;
  note_attention_fwd(a, 4);
  return launch_kernel(SK_LABEL_BY_WIDTH("attention_fwd_f32_kernel", DP),
                       Work{4 * pairs(a), 0.0}, attention_fwd_f32_kernel<DP>, dim3(a.batch * a.kv_heads * tiles), dim3(256), s, a, tiles);
}

template <int DP>
hipError_t bwd(const AttentionArgs& a, hipStream_t s) {
  const int tiles = ((int64_t)a.q_len * a.group + 127) / 128, k_tiles = (a.k_len + 127) / 128;
  note_attention_dq(a, 4);
  hipError_t e = launch_kernel(SK_LABEL_BY_WIDTH("attention_dq_f32_kernel", DP), Work{6 * pairs(a), 0.0},
                               attention_dq_f32_kernel<DP>, dim3(a.batch * a.kv_heads * tiles), dim3(256), s, a, tiles);
  if (e != hipSuccess) return e;
  note_attention_dkv(a, 4);
  e = launch_kernel(SK_LABEL_BY_WIDTH("attention_dkv_f32_kernel", DP), Work{8 * pairs(a), 0.0},
                       attention_dkv_f32_kernel<DP>, dim3(a.batch * a.kv_heads * k_tiles * a.parts), dim3(256), s, a, k_tiles);
  return e != hipSuccess ? e : launch_attention_sum_parts(a, true, s);
}

}  // namespace

hipError_t launch_attention_fwd(const AttentionArgs& a, bool f32, hipStream_t s) {
  if (!f32) return launch_attention_fwd_bf16(a, s);
  return by_width(a.D, [&](auto dp) { return fwd<decltype(dp)::value>(a, s); });
}

hipError_t launch_attention_bwd(const AttentionArgs& a, bool f32, hipStream_t s) {
  if (!f32) return launch_attention_bwd_bf16(a, s);
  return by_width(a.D, [&](auto dp) { return bwd<decltype(dp)::value>(a, s); });
}

}  // namespace sk
