// Attention and its gradients in bf16 (see sk_attention.h and sk_attention_tiles.h for the operands' layouts).
#include "sk_attention_tiles.h"
#include "sk_rows.h"

namespace sk {
namespace {

constexpr int WAVES = 4;   // of 32 rows (queries, or keys) each, to a work-group or half of one

// How the keys are cut where rows alone do not fill the chip, and where the ranges' results are.
struct RangePlan {
  int row_tiles, splits, chunk;   // few rows: tiles of 32 rows, ranges of `chunk` keys; 0: each tile of rows has its keys in `splits` even shares
  int xcds;                       // few rows: that sequences' ranges are dealt over
  float *sums, *stats;            // [heads][splits][rows][D], [heads][splits][rows][2]
};

// Work-group -> (sequence and key head, tile): consecutive work-groups go to the eight XCDs in turn, so with a multiple of
// eight heads each one's tiles, which share keys and values, stay on one XCD's L2; and the tiles with most keys come first.
__device__ __forceinline__ void locate(const AttentionArgs& p, int& b, int& hk, int& tile) {
  const int heads = p.batch * p.kv_heads;
  tile = blockIdx.x / heads;
  const int bh = blockIdx.x - tile * heads;
  b = bh / p.kv_heads;
  hk = bh - b * p.kv_heads;
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

// Share `share` of `shares` of a tile of rows' keys, by whole tiles (none where there are fewer tiles than shares).
template <int HALVES>
struct Keys {
  int begin, end, steps;   // steps: tiles of it; of halves, which wait for each other, of the longer one
  __device__ __forceinline__ Keys(int keys, int share, int shares) {
    const int tiles = (keys + TILE_ROWS - 1) / TILE_ROWS;
    begin = tiles * share / shares * TILE_ROWS;
    end = tiles * (share + 1) / shares * TILE_ROWS;
    end = end < keys ? end : keys;
    steps = HALVES > 1 ? (tiles + shares - 1) / shares : tiles * (share + 1) / shares - tiles * share / shares;
  }
};

// A lane's row as fragments of a product's second operand: zeros past D and where the row is not there (`array`, any row that is, is read
// instead: no branch keeps a load waiting for another).
template <int DP>
__device__ __forceinline__ void load_row(bf16x8 (&f)[DP / 16], const void* array, int64_t row, bool there, int D, int lane) {
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const int c = ks * 16 + (lane >> 5) * 8;
    const bool ok = there && c < D;
    uint4 v = *reinterpret_cast<const uint4*>(static_cast<const bf16*>(array) + (ok ? row + c : 0));
    f[ks] = __builtin_bit_cast(bf16x8, ok ? v : make_uint4(0, 0, 0, 0));
  }
}

// Waits for what has been loaded into them here, ahead of a loop whose own loads go on meanwhile: the compiler, which does not see
// those, would wait for all that is on its way wherever the loop first uses a fragment.
template <int N>
__device__ __forceinline__ void settle(bf16x8 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 u = __builtin_bit_cast(u32x4, f[i]);
    asm volatile("" : "+v"(u));
    f[i] = __builtin_bit_cast(bf16x8, u);
  }
}

// Scores are taken times |scale| log2(e) behind the product, where the maximum has been found; a negative scale is the row's sign, and one
// of zero a row of zeros.
__device__ __forceinline__ float score_factor(float scale) { return scale == 0.f ? 1.f : fabsf(scale) * LOG2E; }
template <int N>
__device__ __forceinline__ void take_sign(bf16x8 (&f)[N], float scale) {
  if (scale > 0.f) return;
  const unsigned flip = scale < 0.f ? 0x80008000u : 0u, keep = scale < 0.f ? 0xffffffffu : 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint4 u = __builtin_bit_cast(uint4, f[i]);
    u = make_uint4((u.x ^ flip) & keep, (u.y ^ flip) & keep, (u.z ^ flip) & keep, (u.w ^ flip) & keep);
    f[i] = __builtin_bit_cast(bf16x8, u);
  }
}

// [DP x 32] with a row of the result to a lane, as rows of D values: the halves of the wave swap four values so that a lane stores eight.
template <int DP>
__device__ __forceinline__ void store_row(bf16* row, bool there, const f32x16 (&acc)[DP / 32], float scale, int D, int lane) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int pr = 0; pr < 2; ++pr) {
      unsigned x[2], y[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = (2 * pr + h) * 4;
        x[h] = pack_bf16x2(acc[d][r] * scale, acc[d][r + 1] * scale);
        y[h] = pack_bf16x2(acc[d][r + 2] * scale, acc[d][r + 3] * scale);
      }
      const auto s0 = __builtin_amdgcn_permlane32_swap(x[0], x[1], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(y[0], y[1], false, false);
      const int c = d * 32 + pr * 16 + (lane >> 5) * 8;
      if (there && c < D) *reinterpret_cast<uint4*>(row + c) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
    }
}

// The same, and in `rest` what rounding leaves off (rounded itself): the backward pass's sum of dO o takes both, since o's rounding alone
// is a third as large an error in dq and dk as their own.
template <int DP>
__device__ __forceinline__ void store_row_and_rest(bf16* row, bf16* rest, bool there, const f32x16 (&acc)[DP / 32], float scale, int D, int lane) {
  store_row<DP>(row, there, acc, scale, D, lane);
  if (rest == nullptr) return;
  f32x16 left[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) left[d][r] = acc[d][r] * scale - (float)(bf16)(acc[d][r] * scale);
  store_row<DP>(rest, there, left, 1.f, D, lane);
}

// The same as fp32 sums, not scaled.
template <int DP>
__device__ __forceinline__ void store_sums(float* row, const f32x16 (&acc)[DP / 32], int D, int lane) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = d * 32 + 8 * g + 4 * (lane >> 5);
      if (c < D) *reinterpret_cast<f32x4*>(row + c) = f32x4{acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]};
    }
}

// Sums of one half of a work-group's waves through LDS to the other half's waves of the same rows: 16 bytes a lane side by side.
template <int ND>
__device__ __forceinline__ void sums_to_lds(unsigned char* lds, const f32x16 (&acc)[ND], int lane) {
#pragma unroll
  for (int i = 0; i < 4 * ND; ++i)
    *reinterpret_cast<f32x4*>(lds + i * 1024 + lane * 16) = f32x4{acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2], acc[i / 4][4 * (i % 4) + 3]};
}
template <int ND>
__device__ __forceinline__ void add_from_lds(f32x16 (&acc)[ND], float keep, const unsigned char* lds, float factor, int lane) {
#pragma unroll
  for (int i = 0; i < 4 * ND; ++i) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(lds + i * 1024 + lane * 16);
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[i / 4][4 * (i % 4) + u] = acc[i / 4][4 * (i % 4) + u] * keep + v[u] * factor;
  }
}

// Running softmax of a lane's row (the lane 32 further has the row's other keys): the maximum and its own keys' sum.
struct Softmax {
  float top = -INFINITY, sum = 0.f, base = 0.f;
  // Takes in a block's scores (before the factor).  What is summed so far, o, is brought down only when a row's maximum has
  // risen by more than 2^8 since it last was: until then the weights are up to 2^8 instead of 1, which neither an fp32 sum nor a
  // bf16's relative rounding minds.
  template <int NB, int ND>
  __device__ __forceinline__ void raise(const f32x16 (&s)[NB], f32x16 (&o)[ND], float factor) {
    float m = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, s[b][r]);
    m = max_halves(m) * factor;
    if (__any(m > top + 8.f)) {
      const float now = fmaxf(top, m), keep = __builtin_amdgcn_exp2f(top - (now == -INFINITY ? 0.f : now));
      top = now;
      sum *= keep;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= keep;
    }
    base = top == -INFINITY ? 0.f : top;   // (nothing seen yet: weights of exp2(-inf))
  }
  // A score's weight
  __device__ __forceinline__ float weigh(float s, float factor) {
    const float w = __builtin_amdgcn_exp2f(s * factor - base);
    sum += w;
    return w;
  }
};

// N products whose first operands are read AHEAD of them: read(i) gives operand i, mma(i, operand) multiplies it, beside(i) is what
// else goes under product i.  In that order: left to itself the compiler reads an operand right before it is used, and waits.
template <int N, int AHEAD, typename Read, typename Multiply, typename Beside>
__device__ __forceinline__ void pipelined(bf16x8 (&f)[AHEAD], Read&& read, Multiply&& mma, Beside&& beside) {
  __builtin_amdgcn_sched_barrier(0);
  static_for<0, N>([&](auto ic) {
    constexpr int i = decltype(ic)::value;
    mma(ic, f[i % AHEAD]);
    if constexpr (i + AHEAD < N) f[i % AHEAD] = read(IntC<i + AHEAD>{});
    beside(ic);
    __builtin_amdgcn_sched_barrier(0);
  });
}
template <int AHEAD, typename Read>
__device__ __forceinline__ void read_first(bf16x8 (&f)[AHEAD], Read&& read) {
  static_for<0, AHEAD>([&](auto ic) { f[decltype(ic)::value] = read(ic); });
  __builtin_amdgcn_sched_barrier(0);
}

// Forward: WAVES x 32 rows a work-group, or with two HALVES twice the waves, each half of which takes half of the keys (with SHARES: a share of their keys, whose
// sums attention_join_kernel puts together), tiles of 64 keys and values through a ring of two slots in LDS, asked for a tile
// ahead; one barrier a tile.  s^T = K q^T, p = exp2(s c - m), o^T = o^T exp2(m' - m) + V^T p^T, in the end o / sum p; a key tile is read by all
// four waves.  At 128 features two waves a SIMD, one's exponentials under the other's products: 16384 tokens in sequences of 4096, 32 heads on 8,
// causal, 543 us = 1010 TFLOP/s of the 4 flops a pair that is seen and feature, the matrix unit 58 % busy at the clock that the power limit
// leaves (zeros for inputs take two thirds as long).  At 64 features four waves a SIMD and the vector unit is the bound (65 % busy, the matrix unit 32 %:
// a score costs it a maximum, a multiplication, an exponential at a quarter of the rate, an addition and half a rounding, and only two products of 64):
// 16 sequences of 512, 16 heads, 29 us, of which the rows' way out, 33 MB behind one round of work-groups, is about 7.
template <int DP, int HALVES, bool SHARES>
__global__ __launch_bounds__(HALVES * WAVES * 64, 2) void attention_fwd_kernel(const AttentionArgs p, RangePlan plan) {
  typedef Tile<DP> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, SLOT = 2 * L::BYTES, K_AHEAD = 2 * KS < 6 ? 2 * KS : 6, V_AHEAD = 4;
  __shared__ __align__(1024) unsigned char smem[HALVES * 2 * SLOT];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = HALVES > 1 ? wave_id / WAVES : 0, wave = wave_id % WAVES;
  int b, hk, tile;
  locate(p, b, hk, tile);
  const int share = SHARES ? tile % plan.splits : 0;
  if (SHARES) tile /= plan.splits;
  if (p.causal) tile = (p.q_len * p.group + WAVES * 32 - 1) / (WAVES * 32) - 1 - tile;
  const Sequence q(p, b);
  const int r0 = tile * WAVES * 32;
  const Row row(p, r0 + wave * 32 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  // the work-group's keys, and the wave's: all rows see those before `common`, none those from `most` on
  const int keys = q.seen(r0 / p.group, (r0 + WAVES * 32 - 1) / p.group);
  const Keys<HALVES> range(keys, share * HALVES + half, HALVES * (SHARES ? plan.splits : 1));
  const int first_i = (r0 + wave * 32) / p.group, last_i = (r0 + wave * 32 + 31) / p.group;
  const int most = __builtin_amdgcn_readfirstlane(first_i < p.q_len ? q.seen(first_i, last_i) : 0);
  const int common = __builtin_amdgcn_readfirstlane(last_i < q.n ? q.limit(first_i) : 0);

  bf16x8 qf[KS];
  load_row<DP>(qf, p.q, b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], row.there && row.i < q.n, p.D, lane);
  take_sign(qf, p.scale);
  settle(qf);
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros();
  Softmax sm;
  const float factor = score_factor(p.scale);

  const bf16* const kb = static_cast<const bf16*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const bf16* const vb = static_cast<const bf16*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  const typename L::template Loader<WAVES> load_k(wave, lane, p.ks[1], p.D), load_v(wave, lane, p.vs[1], p.D);
  const unsigned k_at = L::along_address(lane), v_at = L::across_address(lane);
  Walk<TILE_ROWS> walk_k(kb, p.ks[1], range.begin, p.D), walk_v(vb, p.vs[1], range.begin, p.D);
  if (range.begin < range.end) {
    load_k.load(walk_k.window(q.m - range.begin), half * 2 * SLOT, wave);
    load_v.load(walk_v.window(q.m - range.begin), half * 2 * SLOT + L::BYTES, wave);
  }

  unsigned slot = half * 2 * SLOT;
  int j0 = range.begin;
  for (int step = 0; step < range.steps; ++step, j0 += TILE_ROWS, slot ^= SLOT) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // this tile is there, and nobody reads the other slot
    walk_k.skip(TILE_ROWS);
    walk_v.skip(TILE_ROWS);
    const int left = j0 + TILE_ROWS < range.end ? q.m - j0 - TILE_ROWS : 0;   // (behind the last tile nothing is fetched)
    const u32x4 next_k = walk_k.window(left), next_v = walk_v.window(left);
    // The next tile is asked for an instruction at a time under the scores' products: its 32 KB are half a thousand cycles of the CU's path
    // from memory, in which a wave that asked for all of its own at once would do nothing else.
    constexpr int EACH = L::template Loader<WAVES>::EACH;
    auto ask = [&](auto ic) {
      constexpr int i = decltype(ic)::value, n = 2 * EACH * (i + 1) / (2 * KS) - 1;   // (of K's and V's EACH, at most one a product)
      if constexpr (2 * EACH * i / (2 * KS) <= n) {
        if constexpr (n < EACH) load_k.template load_one<n>(next_k, slot ^ SLOT, wave);
        else load_v.template load_one<n - EACH>(next_v, (slot ^ SLOT) + L::BYTES, wave);
      }
    };
    if (j0 >= most || (HALVES > 1 && j0 >= range.end)) {
      static_for<0, 2 * KS>(ask);
      continue;
    }
    f32x16 s[2] = {zeros(), zeros()};
    {
      bf16x8 f[K_AHEAD];
      auto read = [&](auto ic) { return L::along(slot + k_at, decltype(ic)::value & 1, decltype(ic)::value >> 1); };
      read_first(f, read);
      pipelined<2 * KS>(f, read, [&](auto ic, bf16x8 a) { constexpr int i = decltype(ic)::value; s[i & 1] = M::mma(a, qf[i >> 1], s[i & 1]); }, ask);
    }
    // values 16 step .. + 15 (step i / ND), features 32 (i % ND) .. + 31; the first on their way under the softmax
    bf16x8 f[V_AHEAD];
    auto read = [&](auto ic) { return L::across(slot + L::BYTES + v_at, decltype(ic)::value % ND, decltype(ic)::value / ND); };
    read_first(f, read);
    if (j0 + TILE_ROWS > common)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (j0 + t * 32 + acc_row(r, lane) >= limit) s[t][r] = -INFINITY;
    sm.raise(s, o, factor);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = sm.weigh(s[0][r], factor);
    bf16x8 w[4] = {M::of_acc(s[0], 0), M::of_acc(s[0], 1)};
    pipelined<4 * ND>(f, read, [&](auto ic, bf16x8 a) { constexpr int i = decltype(ic)::value; o[i % ND] = M::mma(a, w[i / ND], o[i % ND]); },
                      [&](auto ic) {   // the second block's weights under the first one's products
                        constexpr int i = decltype(ic)::value;
                        if constexpr (i < 2 * ND) {
#pragma unroll
                          for (int r = 16 * i / (2 * ND); r < 16 * (i + 1) / (2 * ND); ++r) s[1][r] = sm.weigh(s[1][r], factor);
                          if constexpr (i == ND - 1) w[2] = M::of_acc(s[1], 0);
                          if constexpr (i == 2 * ND - 1) w[3] = M::of_acc(s[1], 1);
                        }
                      });
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing may land in LDS any more)
  if (HALVES > 1) {
    __syncthreads();
    float2* const stats = reinterpret_cast<float2*>(smem + WAVES * ND * 4096);
    if (half > 0) {
      sums_to_lds(smem + wave * ND * 4096, o, lane);
      stats[wave * 64 + lane] = make_float2(sm.top, sm.sum);
    }
    __syncthreads();
    if (half > 0) return;
    const float2 other = stats[wave * 64 + lane];
    const float top = fmaxf(sm.top, other.x), base = top == -INFINITY ? 0.f : top;
    const float keep = __builtin_amdgcn_exp2f(sm.top - base), factor = __builtin_amdgcn_exp2f(other.x - base);
    add_from_lds(o, keep, smem + wave * ND * 4096, factor, lane);
    sm.sum = sm.sum * keep + other.y * factor;
    sm.top = top;
  }
  const float sum = sm.sum + other_half(sm.sum);
  if (SHARES) {
    if (!row.there) return;
    const int64_t slot = ((int64_t)(b * p.kv_heads + hk) * plan.splits + share) * p.q_len * p.group + r0 + wave * 32 + (lane & 31);
    store_sums<DP>(plan.sums + slot * p.D, o, p.D, lane);
    if (lane < 32) *reinterpret_cast<float2*>(plan.stats + slot * 2) = make_float2(sm.top, sum);
    return;
  }
  const int64_t at = (((int64_t)b * p.q_len + row.i) * p.heads + row.h) * p.D;
  if (__any(sum == 0.f)) zeros_unless(sum != 0.f, o);   // (selects in every wave would be 1 % of 16 sequences of 512)
  store_row_and_rest<DP>(static_cast<bf16*>(p.o) + at, p.o_rest != nullptr ? static_cast<bf16*>(p.o_rest) + at : nullptr, row.there, o, sum == 0.f ? 0.f : 1.f / sum, p.D,
                         lane);
  if (p.lse != nullptr && row.there && lane < 32)
    p.lse[((int64_t)b * p.heads + row.h) * p.q_len + row.i] = sum == 0.f ? -INFINITY : (sm.top + __builtin_amdgcn_logf(sum)) * LN2;
}

// Forward for few rows: 32 rows a work-group, a range of the keys, of which every wave takes every fourth tile of 32
// by itself (no barrier; 64 KB of LDS, so that eight waves a CU have 8 to 16 KB each on their way), joined through LDS.  Bound by reading: eight
// sequences of 0 to 16384 keys, one query, 64 heads on 8 of 128, 268 MB: 67 us = 4.0 TB/s, where a plain read of 2 GB by stretches reaches 6.3 (51 where the Infinity Cache
// has half of it), and 5 of the join.  Ranges twice and half as long, and grids of three and four work-groups a CU, were level or slower.  With several
// ranges the sums, their maxima and the weights' sums go to the workspace and attention_join_kernel puts them together.
template <int DP>
__global__ __launch_bounds__(256, 2) void attention_few_kernel(const AttentionArgs p, RangePlan plan) {
  typedef Tile<DP, 32> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, LD = DP + 4, EACH = L::INSTRUCTIONS;
  constexpr int ROOM = 2 * L::BYTES > 32 * LD * 4 ? 2 * L::BYTES : 32 * LD * 4;   // of a wave: K and V, at the end its sums
  __shared__ __align__(1024) unsigned char smem[4 * ROOM + 4 * 32 * 8];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // A range's heads, whose keys lie in the same stretch of memory, go to one XCD, the sequences' ranges to the XCDs in turn (another turn each
  // range, so that no XCD has one sequence): 68 us where heads dealt over the XCDs took 71, on the keys above.
  const int local = blockIdx.x / plan.xcds, turn = local / p.kv_heads, hk = local - turn * p.kv_heads, unit = turn * plan.xcds + blockIdx.x - local * plan.xcds;
  const int id = unit / p.batch;
  if (id >= plan.row_tiles * plan.splits) return;
  const int b = (unit + id) % p.batch, bh = b * p.kv_heads + hk, split = id / plan.row_tiles, tile = id - split * plan.row_tiles;
  const Sequence q(p, b);
  const int r0 = tile * 32, rows = p.q_len * p.group - r0 < 32 ? p.q_len * p.group - r0 : 32;
  const Row row(p, r0 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  const int keys = q.seen(r0 / p.group, (r0 + rows - 1) / p.group);
  const int begin = split * plan.chunk, end = begin + plan.chunk < keys ? begin + plan.chunk : keys;
  if (begin >= end && split > 0) return;   // (the join knows; without keys at all the first range writes zeros)
  const int common = __builtin_amdgcn_readfirstlane((r0 + rows - 1) / p.group < q.n ? q.limit(r0 / p.group) : 0);

  const bf16* const kb = static_cast<const bf16*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const bf16* const vb = static_cast<const bf16*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  const typename L::template Loader<1> load_k(0, lane, p.ks[1], p.D), load_v(0, lane, p.vs[1], p.D);
  const unsigned room = wave * ROOM, k_at = room + L::along_address(lane), v_at = room + L::BYTES + L::across_address(lane);
  int j0 = begin + wave * 32;
  Walk<32> walk_k(kb, p.ks[1], j0, p.D), walk_v(vb, p.vs[1], j0, p.D);
  if (j0 < end) {
    load_k.load(walk_k.window(q.m - j0), room, 0);
    load_v.load(walk_v.window(q.m - j0), room + L::BYTES, 0);
  }
  bf16x8 qf[KS];
  load_row<DP>(qf, p.q, b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], row.there && row.i < q.n, p.D, lane);
  take_sign(qf, p.scale);
  settle(qf);
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros();
  Softmax sm;
  const float factor = score_factor(p.scale);
  for (; j0 < end; j0 += 128) {
    f32x16 s[1] = {zeros()};
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(EACH) : "memory");   // all but V's loads, the youngest: K is there
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[0] = M::mma(L::along(k_at, 0, ks), qf[ks], s[0]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // K has been read
    const int left = j0 + 128 < end ? q.m - j0 - 128 : 0;         // (past the last: nothing is fetched)
    walk_k.skip(128);
    walk_v.skip(128);
    load_k.load(walk_k.window(left), room, 0);
    if (j0 + 32 > common)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (j0 + acc_row(r, lane) >= limit) s[0][r] = -INFINITY;
    sm.raise(s, o, factor);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = sm.weigh(s[0][r], factor);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(EACH) : "memory");   // V is there
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 w = M::of_acc(s[0], t);
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = M::mma(L::across(v_at, d, t), w, o[d]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load_v.load(walk_v.window(left), room + L::BYTES, 0);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");     // (no load may land on what follows)
  const float sum = sm.sum + other_half(sm.sum);
  float* const sums = reinterpret_cast<float*>(smem + wave * ROOM);
  float* const stats = reinterpret_cast<float*>(smem + 4 * ROOM);   // [wave][row]: maximum, sum
  if (lane < 32) {
    stats[(wave * 32 + lane) * 2] = sm.top;
    stats[(wave * 32 + lane) * 2 + 1] = sum;
  }
  if ((lane & 31) < rows)
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(sums + (lane & 31) * LD + d * 32 + 8 * g + 4 * (lane >> 5)) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
  __syncthreads();
  // eight features a thread, rows in turn
  constexpr int PER = DP / 8;
  for (int at = threadIdx.x; at < rows * PER; at += 256) {
    const int r = at / PER, c = (at - r * PER) * 8;
    if (c >= p.D) continue;
    float top = -INFINITY, total = 0.f, v[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, stats[(w * 32 + r) * 2]);
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float keep = __builtin_amdgcn_exp2f(stats[(w * 32 + r) * 2] - base);
      total += stats[(w * 32 + r) * 2 + 1] * keep;
      const float* const from = reinterpret_cast<const float*>(smem + w * ROOM) + r * LD + c;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += from[i] * keep;
    }
    if (plan.splits > 1) {
      const int64_t slot = ((int64_t)bh * plan.splits + split) * p.q_len * p.group + r0 + r;
      store_values<float, 8>(plan.sums + slot * p.D + c, v);
      if (c == 0) { plan.stats[slot * 2] = top; plan.stats[slot * 2 + 1] = total; }
    } else {
      const Row out(p, r0 + r, hk);
      const float scale = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = total == 0.f ? 0.f : v[i] * scale;   // (as zeros_unless)
      const int64_t to = (((int64_t)b * p.q_len + out.i) * p.heads + out.h) * p.D + c;
      store_values<bf16, 8>(static_cast<bf16*>(p.o) + to, v);
      if (p.o_rest != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= (float)(bf16)v[i];
        store_values<bf16, 8>(static_cast<bf16*>(p.o_rest) + to, v);
      }
      if (p.lse != nullptr && c == 0) p.lse[((int64_t)b * p.heads + out.h) * p.q_len + out.i] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * LN2;
    }
  }
}

// The ranges' sums of a row in order, each brought to the largest maximum: a thread to four features, eight ranges on their way.
__global__ __launch_bounds__(256) void attention_join_kernel(const AttentionArgs p, RangePlan plan) {
  const int rows = p.q_len * p.group, per = p.D / 4, bh = blockIdx.y;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int r = (int)(id / per), c = (int)(id - (int64_t)r * per) * 4;
  if (r >= rows) return;
  const int b = bh / p.kv_heads, hk = bh - b * p.kv_heads;
  int splits = plan.splits;
  if (plan.chunk > 0) {   // only those that the row's tile has
    const Sequence q(p, b);
    const int r0 = r / 32 * 32, last = r0 + 31 < rows ? r0 + 31 : rows - 1;
    const int keys = q.seen(r0 / p.group, last / p.group);
    splits = keys > 0 ? (keys + plan.chunk - 1) / plan.chunk : 1;
  }
  const int64_t first = (int64_t)bh * plan.splits * rows + r;
  const float2* const stats = reinterpret_cast<const float2*>(plan.stats) + first;
  const float* const sums = plan.sums + first * p.D + c;
  float top = -INFINITY, total = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += 8) {
    float2 stat[8];
    f32x4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t at = (int64_t)(s0 + u < splits ? s0 + u : s0) * rows;
      stat[u] = stats[at];
      x[u] = *reinterpret_cast<const f32x4*>(sums + at * p.D);
    }
    float m = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) m = fmaxf(m, stat[u].x);
    const float base = m == -INFINITY ? 0.f : m, before = __builtin_amdgcn_exp2f(top - base);
    total *= before;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= before;
    top = m;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float keep = s0 + u < splits ? __builtin_amdgcn_exp2f(stat[u].x - base) : 0.f;
      total += stat[u].y * keep;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += x[u][i] * keep;
    }
  }
  const Row out(p, r, hk);
  const float scale = total == 0.f ? 0.f : 1.f / total;
  const int64_t to = (((int64_t)b * p.q_len + out.i) * p.heads + out.h) * p.D + c;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = total == 0.f ? 0.f : v[i] * scale;   // (as zeros_unless)
  store_values<bf16, 4>(static_cast<bf16*>(p.o) + to, v);
  if (p.o_rest != nullptr) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] -= (float)(bf16)v[i];
    store_values<bf16, 4>(static_cast<bf16*>(p.o_rest) + to, v);
  }
  if (p.lse != nullptr && c == 0) p.lse[((int64_t)b * p.heads + out.h) * p.q_len + out.i] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * LN2;
}

// dq: the forward pass's walk over the keys, with the probabilities from lse: p = exp2(s c - lse2), dp = dO v, ds = p (dp - D), dq = scale ds k, where
// -D = -sum dO o is what dp's accumulators begin with, so the subtraction is the product's.  726 us on the forward pass's 16384 tokens (1140
// TFLOP/s of what is executed and seen, the matrix unit 67 % busy), 41 on its 16 sequences of 512 (a third of it the 117 MB that go in and out; 32 keys at a time
// within the registers of four waves a SIMD were level there and 10 % slower at 32 features).  Leaves lse log2(e) and minus sum_d dO o of every row for dk and dv.  With SHARES each
// share of the keys leaves fp32 sums, which attention_sum_parts_kernel adds up in order.  FINE: ds goes into the product in two bf16, rounded and what that left off, so
// that dq is rounded once (off by 0.0017 of 64 bits instead of 0.0024 to 0.0025): for up to 128 keys, where it costs 1 us of 14 (32 sentences of 128, 12 heads of 64),
// and for heads of 32, where a wave has products to spare (33 and 38 us of a pass of 93 to 98, 16 sequences of 512, 16 heads).  With more of both the second rounding stays: it
// would be a third more products.
template <int DP, int HALVES, bool SHARES, bool FINE>
__global__ __launch_bounds__(HALVES * WAVES * 64, 2) void attention_dq_kernel(const AttentionArgs p) {
  typedef Tile<DP> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, SLOT = 2 * L::BYTES, AHEAD = 4;
  __shared__ __align__(1024) unsigned char smem[HALVES * 2 * SLOT];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = HALVES > 1 ? wave_id / WAVES : 0, wave = wave_id % WAVES;
  int b, hk, tile;
  locate(p, b, hk, tile);
  const int share = SHARES ? tile % p.q_shares : 0;
  if (SHARES) tile /= p.q_shares;
  if (p.causal) tile = (p.q_len * p.group + WAVES * 32 - 1) / (WAVES * 32) - 1 - tile;
  const Sequence q(p, b);
  const int r0 = tile * WAVES * 32;
  const Row row(p, r0 + wave * 32 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  const int keys = q.seen(r0 / p.group, (r0 + WAVES * 32 - 1) / p.group);
  const Keys<HALVES> range(keys, share * HALVES + half, HALVES * (SHARES ? p.q_shares : 1));
  const int first_i = (r0 + wave * 32) / p.group, last_i = (r0 + wave * 32 + 31) / p.group;
  const int most = __builtin_amdgcn_readfirstlane(first_i < p.q_len ? q.seen(first_i, last_i) : 0);
  const int common = __builtin_amdgcn_readfirstlane(last_i < q.n ? q.limit(first_i) : 0);
  const bool counts = limit > 0;   // (of a row that sees nothing, not what came back for it either)

  const bf16* const kb = static_cast<const bf16*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const bf16* const vb = static_cast<const bf16*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  const typename L::template Loader<WAVES> load_k(wave, lane, p.ks[1], p.D), load_v(wave, lane, p.vs[1], p.D);
  const unsigned k_at = L::along_address(lane), kt_at = L::across_address(lane);
  Walk<TILE_ROWS> walk_k(kb, p.ks[1], range.begin, p.D), walk_v(vb, p.vs[1], range.begin, p.D);
  if (range.begin < range.end) {
    load_k.load(walk_k.window(q.m - range.begin), half * 2 * SLOT, wave);
    load_v.load(walk_v.window(q.m - range.begin), half * 2 * SLOT + L::BYTES, wave);
  }

  bf16x8 qf[KS], gf[KS];
  const int64_t at = (((int64_t)b * p.q_len + row.i) * p.heads + row.h) * p.D;
  const int64_t stat = ((int64_t)b * p.heads + row.h) * p.q_len + row.i;
  load_row<DP>(qf, p.q, b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], counts, p.D, lane);
  take_sign(qf, p.scale);
  load_row<DP>(gf, p.d_o, at, counts, p.D, lane);
  float delta = 0.f;
  {
    bf16x8 of[KS];
    load_row<DP>(of, p.o_in, at, counts, p.D, lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) delta -= M::dot(of[ks], gf[ks]);
    if (p.o_rest != nullptr) {
      load_row<DP>(of, p.o_rest, at, counts, p.D, lane);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) delta -= M::dot(of[ks], gf[ks]);
    }
  }
  delta += other_half(delta);
  settle(qf);
  settle(gf);
  // (a row that sees nothing has no probabilities, whatever its lse says)
  float lse = counts ? p.lse[stat] * LOG2E : INFINITY;
  asm volatile("" : "+v"(lse), "+v"(delta));
  if (row.there && lane < 32 && share == 0 && half == 0) {
    p.lse2[stat] = lse;
    p.delta[stat] = delta;
  }
  f32x16 dq[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dq[d] = zeros();
  const float factor = score_factor(p.scale);
  unsigned slot = half * 2 * SLOT;
  int j0 = range.begin;
  for (int step = 0; step < range.steps; ++step, j0 += TILE_ROWS, slot ^= SLOT) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    walk_k.skip(TILE_ROWS);
    walk_v.skip(TILE_ROWS);
    const int left = j0 + TILE_ROWS < range.end ? q.m - j0 - TILE_ROWS : 0;
    const u32x4 next_k = walk_k.window(left), next_v = walk_v.window(left);
    constexpr int EACH = L::template Loader<WAVES>::EACH;
    auto ask = [&](auto ic) {   // (as the forward pass's, one to two products)
      constexpr int i = decltype(ic)::value, n = 2 * EACH * (i + 1) / (4 * KS) - 1;
      if constexpr (2 * EACH * i / (4 * KS) <= n) {
        if constexpr (n < EACH) load_k.template load_one<n>(next_k, slot ^ SLOT, wave);
        else load_v.template load_one<n - EACH>(next_v, (slot ^ SLOT) + L::BYTES, wave);
      }
    };
    if (j0 >= most || (HALVES > 1 && j0 >= range.end)) {
      static_for<0, 4 * KS>(ask);
      continue;
    }
    f32x16 s[2], g[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = zeros();
#pragma unroll
      for (int r = 0; r < 16; ++r) g[t][r] = delta;
    }
    if constexpr (DP > 64) {   // operand i: of k and v in turn, two blocks each, 16 features after 16
      bf16x8 f[AHEAD];
      auto read = [&](auto ic) {
        constexpr int i = decltype(ic)::value;
        return L::along(slot + (i & 2 ? L::BYTES : 0) + k_at, i & 1, i >> 2);
      };
      read_first(f, read);
      pipelined<4 * KS>(f, read, [&](auto ic, bf16x8 a) {
        constexpr int i = decltype(ic)::value;
        if constexpr (i & 2) g[i & 1] = M::mma(a, gf[i >> 2], g[i & 1]);
        else s[i & 1] = M::mma(a, qf[i >> 2], s[i & 1]);
      }, ask);
    } else {   // (the compiler's order keeps within the registers of three waves a SIMD, which at 64 features are worth more)
      static_for<0, 4 * KS>(ask);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          s[t] = M::mma(L::along(slot + k_at, t, ks), qf[ks], s[t]);
          g[t] = M::mma(L::along(slot + L::BYTES + k_at, t, ks), gf[ks], g[t]);
        }
    }
    if (j0 + TILE_ROWS > common)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (j0 + t * 32 + acc_row(r, lane) >= limit) s[t][r] = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = __builtin_amdgcn_exp2f(s[t][r] * factor - lse) * g[t][r];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bf16x8 w = M::of_acc(s[t >> 1], t & 1);
      bf16x8 rest;
      if constexpr (FINE) rest = M::rest_of_acc(s[t >> 1], t & 1, w);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const bf16x8 k = L::across(slot + kt_at, d, t);
        dq[d] = M::mma(k, w, dq[d]);
        if constexpr (FINE) dq[d] = M::mma(k, rest, dq[d]);
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (HALVES > 1) {
    __syncthreads();
    if (half > 0) sums_to_lds(smem + wave * ND * 4096, dq, lane_again());
    __syncthreads();
    if (half > 0) return;
    add_from_lds(dq, 1.f, smem + wave * ND * 4096, 1.f, lane_again());
  }
  const int lane_out = lane_again();   // (where the row is need not lie in registers all the way)
  const Row out(p, r0 + wave * 32 + (lane_out & 31), hk);
  const int64_t to = (((int64_t)b * p.q_len + out.i) * p.heads + out.h) * p.D;
  const bool counts_out = out.there && q.limit(out.i) > 0;
  if (__any(!counts_out)) zeros_unless(counts_out, dq);
  if (!SHARES) store_row<DP>(static_cast<bf16*>(p.dq) + to, out.there, dq, p.scale, p.D, lane_out);
  else if (out.there) store_sums<DP>(p.q_partial + share * ((int64_t)p.batch * p.q_len * p.heads * p.D) + to, dq, p.D, lane_out);
}

// dk and dv: 32 keys a wave, their sums in registers over all queries of all heads that share them; tiles of 64 queries and their
// dO through the ring, with what dq's kernel left of their rows.  Two waves a SIMD, so that one's exponentials run under the other's
// products, is what the registers are kept to: one wave of 330 took 1572 us where two take 1081 (16384 tokens in sequences of 4096, 32 heads on 8 of 128,
// causal; the matrix unit 59 % busy).  256 keys a work-group instead of 128 load half as much for 1 % there, and cost 17 to 25 % at 128 to 512 keys of 64.
template <int DP>
__global__ __launch_bounds__(WAVES * 64, 2) void attention_dkv_kernel(const AttentionArgs p) {
  typedef Tile<DP> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, STATS = 2 * L::BYTES, SLOT = STATS + 1024;
  constexpr int APART = DP > 96 ? 1 : 0;   // fragments of v that lie in LDS, a lane's own to read: all of them in registers are four too many
  __shared__ __align__(1024) unsigned char smem[2 * SLOT + WAVES * APART * 1024];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, hk, tile;
  locate(p, b, hk, tile);
  const int part = tile % p.parts;
  tile /= p.parts;
  const Sequence q(p, b);
  const int j0 = tile * WAVES * 32, jw = j0 + wave * 32, j = jw + (lane & 31);
  const bool there = j < q.m;
  // the first query that the work-group and the wave look at: that sees their first key, and no earlier one, whose dO need not be a number if it
  // sees nothing (past the end none does)
  const int i_begin = q.causal && j0 - q.shift + 1 > 0 ? j0 - q.shift + 1 : 0;
  const int i_wave = jw < q.m ? (q.causal ? jw - q.shift + 1 : 0) : INT32_MAX;
  const int i_whole = jw + 31 < q.m ? (q.causal ? jw + 31 - q.shift + 1 : 0) : INT32_MAX;   // from here on queries see all the wave's keys
  const int per_head = j0 < q.m && q.n > i_begin ? (q.n - i_begin + TILE_ROWS - 1) / TILE_ROWS : 0;
  // this part's tiles of all heads' (one head's behind the other's): `first_head`'s from i_first on
  const int all = per_head * p.group, begin = (int)((int64_t)all * part / p.parts), steps = (int)((int64_t)all * (part + 1) / p.parts) - begin;
  const int first_head = hk * p.group + (steps > 0 ? begin / per_head : 0), i_first = i_begin + (steps > 0 ? begin % per_head : 0) * TILE_ROWS;

  // (sums, keys and values take 192 registers of 256, scores 32: a lane's offsets are computed where they are used)
  Walk<TILE_ROWS> walk_q(static_cast<const bf16*>(p.q) + b * p.qs[0] + first_head * p.qs[2], p.qs[1], i_first, p.D);
  Walk<TILE_ROWS> walk_g(static_cast<const bf16*>(p.d_o) + ((int64_t)b * p.q_len * p.heads + first_head) * p.D, (int64_t)p.heads * p.D, i_first, p.D);
  const float* stat = (wave == 0 ? p.lse2 : p.delta) + ((int64_t)b * p.heads + first_head) * p.q_len + i_first;
  const int per_tile = per_head * TILE_ROWS;
  int left = q.n - i_first;
  auto load = [&](unsigned slot) {
    const int lane = lane_again();
    const typename L::template Loader<WAVES> load_q(wave, lane, p.qs[1], p.D), load_g(wave, lane, (int64_t)p.heads * p.D, p.D);
    load_q.load(walk_q.window(left), slot, wave);
    load_g.load(walk_g.window(left), slot + L::BYTES, wave);
    if (wave < 2) {   // 64 rows' statistics: zeros behind the last, where q and dO are zeros too and nothing comes of them
      const uint64_t at = (uint64_t)stat;
      const u32x4 rows = scalar(u32x4{(unsigned)at, (unsigned)(at >> 32), (unsigned)left * 4u, 0x00020000u});
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(slot + STATS + wave * 256), "v"((unsigned)lane * 4u), "s"(rows), "s"(0u) : "m0");
    }
    left -= TILE_ROWS;
    if (left > 0) {
      walk_q.skip(TILE_ROWS);
      walk_g.skip(TILE_ROWS);
      stat += TILE_ROWS;
    } else {   // the group's next head from the first tile on
      const int back = per_tile - TILE_ROWS;
      left = q.n - i_begin;
      walk_q.at += (uint64_t)(p.qs[2] * 2) - (uint64_t)back * walk_q.stride;
      walk_g.at += (uint64_t)(p.D * 2) - (uint64_t)back * walk_g.stride;
      stat += p.q_len - back;
    }
  };
  if (steps > 0) load(0u);

  bf16x8 kf[KS], vf[KS];
  load_row<DP>(kf, p.k, b * p.ks[0] + j * p.ks[1] + hk * p.ks[2], there, p.D, lane);
  take_sign(kf, p.scale);
  load_row<DP>(vf, p.v, b * p.vs[0] + j * p.vs[1] + hk * p.vs[2], there, p.D, lane);
  settle(kf);
  settle(vf);
  const unsigned apart = 2 * SLOT + wave * APART * 1024;
#pragma unroll
  for (int i = 0; i < APART; ++i) *reinterpret_cast<bf16x8*>(smem + apart + i * 1024 + lane * 16) = vf[KS - APART + i];
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dk[d] = dv[d] = zeros();
  const float factor = score_factor(p.scale);
  unsigned slot = 0;
  int i0 = i_first;
  for (int step = 0; step < steps; ++step, slot = SLOT - slot) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int i_now = i0;
    i0 += TILE_ROWS;
    if (i0 >= q.n) i0 = i_begin;
    if (step + 1 < steps) load(SLOT - slot);
    if (i_now + TILE_ROWS <= i_wave) continue;
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
      const int lane = lane_again();
      const unsigned q_at = slot + t * 4096 + L::along_address(lane), g_at = q_at + L::BYTES, stat_at = slot + STATS + t * 128 + (lane >> 5) * 16;
      f32x16 s = zeros(), g;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 d = *(lds_f32x4*)(uintptr_t)(stat_at + 256 + r * 8);
#pragma unroll
        for (int u = 0; u < 4; ++u) g[r + u] = d[u];
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = M::mma(L::along(q_at, 0, ks), kf[ks], s);
        typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
        g = M::mma(L::along(g_at, 0, ks), ks < KS - APART ? vf[ks] : *(lds_bf16x8*)(uintptr_t)(apart + (ks - KS + APART) * 1024 + lane * 16), g);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 lse = *(lds_f32x4*)(uintptr_t)(stat_at + r * 8);
#pragma unroll
        for (int u = 0; u < 4; ++u) s[r + u] = __builtin_amdgcn_exp2f(s[r + u] * factor - lse[u]);
      }
      if (i_now < i_whole) {
        const int j = jw + (lane & 31), first = j < q.m ? (q.causal ? j - q.shift + 1 : 0) : INT32_MAX;   // the first query that sees key j
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (i_now + t * 32 + acc_row(r, lane) < first) s[r] = 0.f;
      }
      // (past the last query the tile has zeros, or where queries overlap in memory that query again: with lse = 0 its weight may be infinite, which
      // the zeros of dO would make NaN)
      if (i_now + TILE_ROWS > q.n) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (i_now + t * 32 + acc_row(r, lane) >= q.n) s[r] = 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) g[r] *= s[r];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 w = M::of_acc(s, u), e = M::of_acc(g, u);
        const unsigned qt_at = slot + L::across_address(lane) + (t * 2 + u) * 2048;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          dv[d] = M::mma(L::across(qt_at + L::BYTES, d, 0), w, dv[d]);
          dk[d] = M::mma(L::across(qt_at, d, 0), e, dk[d]);
        }
      }
    }
  }
  const int j_out = jw + (lane_again() & 31);
  const int64_t row = ((int64_t)b * p.k_len + j_out) * p.kv_heads + hk;
  if (jw + 32 > q.m) {
    zeros_unless(j_out < q.m, dk);
    zeros_unless(j_out < q.m, dv);
  }
  if (p.parts == 1) {
    store_row<DP>(static_cast<bf16*>(p.dk) + row * p.D, j_out < p.k_len, dk, p.scale, p.D, lane_again());
    store_row<DP>(static_cast<bf16*>(p.dv) + row * p.D, j_out < p.k_len, dv, 1.f, p.D, lane_again());
  } else if (j_out < p.k_len) {
    const int64_t values = (int64_t)p.batch * p.k_len * p.kv_heads * p.D;
    float* const to = p.partial + part * 2 * values + row * p.D;
    store_sums<DP>(to, dk, p.D, lane_again());
    store_sums<DP>(to + values, dv, p.D, lane_again());
  }
}

double pairs(const AttentionArgs& a) { return (double)a.batch * a.q_len * a.heads * a.k_len * a.D; }
unsigned groups_of(const AttentionArgs& a, int64_t rows, int per) { return (unsigned)((int64_t)a.batch * a.kv_heads * ((rows + per - 1) / per)); }

// Even shares of each row tile's keys, for the forward pass by attention_fwd_kernel and for dq: where tiles of 128 rows leave CUs empty, so many that they
// do not, of eight tiles of keys at least; under a causal mask, whose walks differ in length, up to two work-groups a CU, whose shorter ones even that out.  Below 24 tiles of
// keys the fp32 sums and the launch that joins them cost more than they save.  Four sequences of 300 queries on 4000 keys, 8 heads on 2 of 128,
// causal: 81 us in one share, 32 + 9 in five; one of 4096, 4 heads on 2 of 64, causal, forward 58 and 23 + 8, dq 63 and 29 + 2; one of 4096, 8 on 4 of 128, the most
// work-groups that are cut, forward 72 and 51 + 15, dq 86 and 71 + 5.  Not cut: two of 1895, 16 heads on 4 of 64, causal: 39 in one share, 31 + 10 in two;
// not causal, one of 2048, 16 heads of 128: 45 and 44 + 10.
int query_shares(const AttentionArgs& a) {
  const int64_t groups = (int64_t)a.batch * a.kv_heads * (((int64_t)a.q_len * a.group + 127) / 128), tiles = (a.k_len + TILE_ROWS - 1) / TILE_ROWS;
  int64_t shares = (a.causal ? 2 : 1) * NUM_CUS / groups;
  if (tiles < 24 || shares < 2) return 1;
  if (shares > tiles / 8) shares = tiles / 8;
  return shares > 16 ? 16 : (int)shares;
}

// Whether a work-group of eight waves, four to each half of the keys, takes a tile of rows (forward, dq), joined through LDS: where a round of work-groups leaves
// SIMDs with one wave, or the walks under a causal mask differ so much that it soon does.  Two sequences of 1800, 8 heads on 4 of 64: forward 36
// and with halves 30 us, dq 42 and 33; two of 1895, 16 on 4 of 64, causal: 39 and 34, 46 and 37; three of up to 3875, 4 on 1 of 128, causal: 79 and 61, 88
// and 72.  At more than 64 features its LDS leaves room for one on a CU: one sequence of 2048, 32 heads on 8 of 128, 512 tiles, causal, 58 and 53, but dq 69 and
// 72; 1001 queries of 64 heads on 8, 504 tiles, 96 and 99; two of 1024, 16 on 8 of 128, 27 and 25, 32 and 33: these stay with four waves.
bool query_halves(const AttentionArgs& a) {
  const int64_t groups = (int64_t)a.batch * a.kv_heads * (((int64_t)a.q_len * a.group + 127) / 128), tiles = a.k_len / TILE_ROWS;
  return a.D <= 64 ? tiles >= 16 && groups <= 2 * NUM_CUS : tiles >= 32 && 2 * groups <= 3 * NUM_CUS;
}

// Whether the forward pass goes by attention_few_kernel, and how: rows that fill one wave's tile at most, or so few that tiles of 32, whose four
// waves share the way through the keys, leave no CU with two (two sequences of 355, eight heads of 64: 8.7 us where tiles of 128 took
// 11.7; 640 queries of 16 heads, 320 tiles of 32: 24.8 and 13.7).
bool few_rows(const AttentionArgs& a, RangePlan& plan) {
  const int64_t heads = (int64_t)a.batch * a.kv_heads, rows = (int64_t)a.q_len * a.group;
  if (rows > 32 && (heads * ((rows + 31) / 32) > NUM_CUS || a.k_len < 128)) return false;
  plan.row_tiles = (int)((rows + 31) / 32);
  // ranges for two rounds of two work-groups a CU, of 512 keys at least: less than four tiles a wave cost less than the join's launch
  const int64_t wanted = (4 * NUM_CUS + heads * plan.row_tiles - 1) / (heads * plan.row_tiles);
  int64_t chunk = (a.k_len + wanted - 1) / wanted;
  chunk = chunk < 512 ? 512 : (chunk + 127) / 128 * 128;
  plan.splits = (int)((a.k_len + chunk - 1) / chunk);
  plan.chunk = (int)chunk;
  return true;
}
size_t range_sums(const AttentionArgs& a, const RangePlan& plan) {
  return plan.splits > 1 ? (size_t)a.batch * a.kv_heads * plan.splits * a.q_len * a.group * a.D * 4 : 0;
}
size_t range_bytes(const AttentionArgs& a, const RangePlan& plan) { return range_sums(a, plan) + range_sums(a, plan) / a.D * 2; }
void place_ranges(const AttentionArgs& a, RangePlan& plan) {
  plan.sums = static_cast<float*>(a.workspace);
  plan.stats = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + range_sums(a, plan));
}
hipError_t join(const AttentionArgs& a, const RangePlan& plan, hipStream_t s) {
  const size_t bytes = range_bytes(a, plan);
  note_matrix(a.workspace, 1, bytes, bytes, 1, false);
  note_attention_fwd(a, 2);
  return launch_kernel("attention_join_kernel", Work{0.0, (double)bytes}, attention_join_kernel,
                       dim3((unsigned)(((int64_t)a.q_len * a.group * (a.D / 4) + 255) / 256), a.batch * a.kv_heads), dim3(256), s, a, plan);
}

template <int DP>
hipError_t few(const AttentionArgs& a, RangePlan plan, hipStream_t s) {
  const size_t bytes = range_bytes(a, plan);
  const int64_t units = (int64_t)a.batch * plan.row_tiles * plan.splits;
  plan.xcds = units < 8 ? (int)units : 8;
  place_ranges(a, plan);
  note_attention_inputs(a, 2);
  if (plan.splits == 1) note_attention_fwd(a, 2);
  else note_matrix(a.workspace, 1, bytes, bytes, 1, true);
  hipError_t e = launch_kernel(SK_LABEL_BY_WIDTH("attention_few_kernel", DP), Work{4 * pairs(a), 0.0}, attention_few_kernel<DP>,
                               dim3((unsigned)((units + plan.xcds - 1) / plan.xcds * plan.xcds * a.kv_heads)), dim3(256), s, a, plan);
  return e != hipSuccess || plan.splits == 1 ? e : join(a, plan, s);
}

template <int DP>
hipError_t fwd(const AttentionArgs& a, hipStream_t s) {
  RangePlan plan{};
  if (few_rows(a, plan)) return few<DP>(a, plan, s);
  plan.splits = query_shares(a);
  if (plan.splits > 1) {
    const size_t bytes = range_bytes(a, plan);
    place_ranges(a, plan);
    note_attention_inputs(a, 2);
    note_matrix(a.workspace, 1, bytes, bytes, 1, true);
    hipError_t e = launch_kernel(SK_LABEL_BY_WIDTH("attention_fwd_shares_kernel", DP), Work{4 * pairs(a), 0.0}, attention_fwd_kernel<DP, 1, true>,
                                 dim3(groups_of(a, (int64_t)a.q_len * a.group, WAVES * 32) * plan.splits), dim3(WAVES * 64), s, a, plan);
    return e != hipSuccess ? e : join(a, plan, s);
  }
  note_attention_fwd(a, 2);
  const dim3 groups(groups_of(a, (int64_t)a.q_len * a.group, WAVES * 32));
  const Work work{4 * pairs(a), 0.0};
  if (query_halves(a)) return launch_kernel(SK_LABEL_BY_WIDTH("attention_fwd_halves_kernel", DP), work, attention_fwd_kernel<DP, 2, false>, groups, dim3(2 * WAVES * 64), s, a, plan);
  return launch_kernel(SK_LABEL_BY_WIDTH("attention_fwd_kernel", DP), work, attention_fwd_kernel<DP, 1, false>, groups, dim3(WAVES * 64), s, a, plan);
}

template <int DP>
hipError_t bwd(const AttentionArgs& a, hipStream_t s) {
  note_attention_dq(a, 2);
  const unsigned groups = groups_of(a, (int64_t)a.q_len * a.group, WAVES * 32);
  const Work work{6 * pairs(a), 0.0};
  constexpr bool FINE = DP == 32;
  hipError_t e = a.q_shares > 1 ? launch_kernel(SK_LABEL_BY_WIDTH("attention_dq_shares_kernel", DP), work, attention_dq_kernel<DP, 1, true, FINE>, dim3(groups * a.q_shares), dim3(WAVES * 64), s, a)
                 : query_halves(a) ? launch_kernel(SK_LABEL_BY_WIDTH("attention_dq_halves_kernel", DP), work, attention_dq_kernel<DP, 2, false, FINE>, dim3(groups), dim3(2 * WAVES * 64), s, a)
                 : a.k_len <= 2 * TILE_ROWS ? launch_kernel(SK_LABEL_BY_WIDTH("attention_dq_fine_kernel", DP), work, attention_dq_kernel<DP, 1, false, true>, dim3(groups), dim3(WAVES * 64), s, a)
                                   : launch_kernel(SK_LABEL_BY_WIDTH("attention_dq_kernel", DP), work, attention_dq_kernel<DP, 1, false, FINE>, dim3(groups), dim3(WAVES * 64), s, a);
  if (e != hipSuccess) return e;
  note_attention_dkv(a, 2);
  e = launch_kernel(SK_LABEL_BY_WIDTH("attention_dkv_kernel", DP), Work{8 * pairs(a), 0.0}, attention_dkv_kernel<DP>, dim3(groups_of(a, a.k_len, WAVES * 32) * a.parts), dim3(WAVES * 64), s, a);
  return e != hipSuccess ? e : launch_attention_sum_parts(a, false, s);
}

}  // namespace

// Results in parts, [part][values] a `step` apart, that are added up in order, scaled and rounded; one to a row of the grid.
struct PartSums {
  struct {
    const float* from;
    void* to;
    int64_t values, step;
    int parts;
    float scale;
  } of[3];
};
template <typename T>
__global__ __launch_bounds__(256) void attention_sum_parts_kernel(const PartSums p) {
  const auto& r = p.of[blockIdx.y];
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= r.values) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int part = 0; part < r.parts; ++part) {
    const float4 x = *reinterpret_cast<const float4*>(r.from + at + part * r.step);
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  const float out[4] = {s.x * r.scale, s.y * r.scale, s.z * r.scale, s.w * r.scale};
  store_values<T, 4>(static_cast<T*>(r.to) + at, out);
}

size_t attention_fwd_bytes_bf16(const AttentionArgs& a) {
  RangePlan plan{};
  if (!few_rows(a, plan)) plan.splits = query_shares(a);
  return range_bytes(a, plan);
}
hipError_t launch_attention_fwd_bf16(const AttentionArgs& a, hipStream_t s) { return by_width(a.D, [&](auto dp) { return fwd<decltype(dp)::value>(a, s); }); }
hipError_t launch_attention_sum_parts(const AttentionArgs& a, bool f32, hipStream_t s) {
  const int64_t keys = (int64_t)a.batch * a.k_len * a.kv_heads * a.D, queries = rows_of(a) * a.D;
  const int esize = f32 ? 4 : 2;
  PartSums p{};
  int n = 0;
  if (a.parts > 1) {
    p.of[n++] = {a.partial, a.dk, keys, 2 * keys, a.parts, a.scale};
    p.of[n++] = {a.partial + keys, a.dv, keys, 2 * keys, a.parts, 1.f};
    note_matrix(a.partial, 2 * a.parts, keys, keys, 4, false);
    note_matrix(a.dk, 1, keys, keys, esize, true);
    note_matrix(a.dv, 1, keys, keys, esize, true);
  }
  if (a.q_shares > 1) {
    p.of[n++] = {a.q_partial, a.dq, queries, queries, a.q_shares, a.scale};
    note_matrix(a.q_partial, a.q_shares, queries, queries, 4, false);
    note_matrix(a.dq, 1, queries, queries, esize, true);
  }
  if (n == 0) return hipSuccess;
  double bytes = 0.0;
  int64_t most = 0;
  for (int i = 0; i < n; ++i) {
    bytes += (4.0 * p.of[i].parts + esize) * p.of[i].values;
    most = p.of[i].values > most ? p.of[i].values : most;
  }
  const dim3 grid((unsigned)((most / 4 + 255) / 256), n);
  return f32 ? launch_kernel("attention_sum_parts_kernel", Work{0.0, bytes}, attention_sum_parts_kernel<float>, grid, dim3(256), s, p)
             : launch_kernel("attention_sum_parts_kernel", Work{0.0, bytes}, attention_sum_parts_kernel<bf16>, grid, dim3(256), s, p);
}

// dk and dv's kernel gets as many work-groups as there are tiles of 128 keys, which with few key heads leaves CUs without one while
// each walks over the queries of a whole group: below two a CU the walk is cut into parts of eight tiles at least (what the sum's launch
// costs), whose fp32 results a second kernel adds up in order: for two a CU, or under a causal mask, whose tiles differ in length,
// three.  One sequence of 2048 tokens, 32 heads on 8 of 128, causal: 317 us in one part, 106 + 14 at two a CU, 92 + 19 at three; of 4096 on 4,
// not causal: 1250, 549 + 15, 583 + 19.  Under a causal mask parts of four tiles up to two a CU still pay: six sequences of 401, 8 heads on 4 of 128: 43 in one,
// 25 + 8 in three; one of 344, 64 on 8: 33 + 6 in six, 25 + 8 in twelve.
int attention_query_shares(const AttentionArgs& a) { return query_shares(a); }
int attention_parts(const AttentionArgs& a, bool f32) {
  const int64_t groups = (int64_t)a.batch * a.kv_heads * ((a.k_len + 127) / 128), tiles = (int64_t)a.group * ((a.q_len + (f32 ? 31 : 63)) / (f32 ? 32 : 64));
  if (groups >= 2 * NUM_CUS) return 1;
  int64_t parts;
  if (f32) {
    // a tile takes 3 to 7 us, so two to a part do; no more parts than one round of the work-groups that the registers leave room for (14 sequences of 512,
    // eight heads of 96, causal: 294 + 21 us in two rounds, 277 in one; one of 55, 4 heads on 1 of 32: 34 in one part, 13 + 6 in four)
    parts = (a.D <= 64 ? 2 : 1) * NUM_CUS / groups;
    parts = parts < tiles / 2 ? parts : tiles / 2;
  } else {
    parts = ((a.causal ? 3 : 2) * NUM_CUS + groups - 1) / groups;
    parts = parts < tiles / 8 ? parts : tiles / 8;
    const int64_t evened = a.causal ? 2 * NUM_CUS / groups : 1;
    if (parts < evened) parts = evened < tiles / 4 ? evened : tiles / 4 > parts ? tiles / 4 : parts;
  }
  return parts < 1 ? 1 : parts > 16 ? 16 : (int)parts;
}

hipError_t launch_attention_bwd_bf16(const AttentionArgs& a, hipStream_t s) { return by_width(a.D, [&](auto dp) { return bwd<decltype(dp)::value>(a, s); }); }

}  // namespace sk
