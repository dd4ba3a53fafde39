// Attention and its gradients in bf16 (see sk_attention.h and sk_attention_tiles.h for the operands' layouts).
#include "sk_attention_tiles.h"

namespace sk {
namespace {

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

// A lane's row as fragments of a product's second operand: zeros past D and where the row is not there.
template <int DP>
__device__ __forceinline__ void load_row(bf16x8 (&f)[DP / 16], const bf16* row, bool there, int D, int lane) {
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const int c = ks * 16 + (lane >> 5) * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (there && c < D) v = *reinterpret_cast<const uint4*>(row + c);
    f[ks] = __builtin_bit_cast(bf16x8, v);
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

// Running softmax of a lane's row (the lane 32 further has the row's other keys): the maximum and its own keys' sum.
struct Softmax {
  float top = -INFINITY, sum = 0.f;
  // s: a block's scores before the factor, on return its weights; o: what the weights so far have summed up.  What is summed is
  // brought down only when a row's maximum has risen by more than 2^8 since it last was: until then the weights are up to
  // 2^8 instead of 1, which neither an fp32 sum nor a bf16's relative rounding minds.
  template <int NB, int ND>
  __device__ __forceinline__ void update(f32x16 (&s)[NB], f32x16 (&o)[ND], float factor) {
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
    const float base = top == -INFINITY ? 0.f : top;   // (nothing seen yet: weights of exp2(-inf))
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(s[b][r] * factor - base);
        sum += s[b][r];
      }
  }
};

// Forward: WAVES x 32 rows a work-group, tiles of 64 keys and values through a ring of two slots in LDS, asked for a tile
// ahead; one barrier a tile.
template <int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void attention_fwd_kernel(const AttentionArgs p) {
  typedef Tile<DP> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, SLOT = 2 * L::BYTES;
  __shared__ __align__(1024) unsigned char smem[2 * SLOT];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, hk, tile;
  locate(p, b, hk, tile);
  if (p.causal) tile = (p.q_len * p.group + WAVES * 32 - 1) / (WAVES * 32) - 1 - tile;
  const Sequence q(p, b);
  const int r0 = tile * WAVES * 32;
  const Row row(p, r0 + wave * 32 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  // the work-group's keys, and the wave's: all rows see those before `common`, none those from `most` on
  const int keys = q.seen(r0 / p.group, (r0 + WAVES * 32 - 1) / p.group);
  const int first_i = (r0 + wave * 32) / p.group, last_i = (r0 + wave * 32 + 31) / p.group;
  const int most = __builtin_amdgcn_readfirstlane(first_i < p.q_len ? q.seen(first_i, last_i) : 0);
  const int common = __builtin_amdgcn_readfirstlane(last_i < q.n ? q.limit(first_i) : 0);

  bf16x8 qf[KS];
  load_row<DP>(qf, static_cast<const bf16*>(p.q) + b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], row.there && row.i < q.n, p.D, lane);
  take_sign(qf, p.scale);
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros();
  Softmax sm;
  const float factor = score_factor(p.scale);

  const bf16* const kb = static_cast<const bf16*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const bf16* const vb = static_cast<const bf16*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  const typename L::template Loader<WAVES> load_k(wave, lane, p.ks[1], p.D), load_v(wave, lane, p.vs[1], p.D);
  const unsigned k_at = L::along_address(lane), v_at = L::across_address(lane);
  auto load = [&](int j0, unsigned slot) {
    load_k.load(rows_from(kb, p.ks[1], j0, q.m, p.D), slot, wave);
    load_v.load(rows_from(vb, p.vs[1], j0, q.m, p.D), slot + L::BYTES, wave);
  };
  if (keys > 0) load(0, 0u);
  unsigned slot = 0;
  for (int j0 = 0; j0 < keys; j0 += TILE_ROWS, slot ^= SLOT) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // this tile is there, and nobody reads the other slot
    if (j0 + TILE_ROWS < keys) load(j0 + TILE_ROWS, slot ^ SLOT);
    if (j0 >= most) continue;
    f32x16 s[2] = {zeros(), zeros()};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t) s[t] = M::mma(L::along(slot + k_at, t, ks), qf[ks], s[t]);
    if (j0 + TILE_ROWS > common)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (j0 + t * 32 + acc_row(r, lane) >= limit) s[t][r] = -INFINITY;
    sm.update(s, o, factor);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bf16x8 w = M::of_acc(s[t >> 1], t & 1);
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] = M::mma(L::across(slot + L::BYTES + v_at, d, t), w, o[d]);
    }
  }
  const float sum = sm.sum + other_half(sm.sum);
  store_row<DP>(static_cast<bf16*>(p.o) + (((int64_t)b * p.q_len + row.i) * p.heads + row.h) * p.D, row.there, o, sum == 0.f ? 0.f : 1.f / sum, p.D, lane);
  if (p.lse != nullptr && row.there && lane < 32)
    p.lse[((int64_t)b * p.heads + row.h) * p.q_len + row.i] = sum == 0.f ? -INFINITY : (sm.top + __builtin_amdgcn_logf(sum)) * LN2;
}

// dq: the forward pass's walk over the keys, with the probabilities from lse.  Leaves lse log2(e) and minus sum_d dO o of every row for dk and dv.
template <int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void attention_dq_kernel(const AttentionArgs p) {
  typedef Tile<DP> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, SLOT = 2 * L::BYTES;
  __shared__ __align__(1024) unsigned char smem[2 * SLOT];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, hk, tile;
  locate(p, b, hk, tile);
  if (p.causal) tile = (p.q_len * p.group + WAVES * 32 - 1) / (WAVES * 32) - 1 - tile;
  const Sequence q(p, b);
  const int r0 = tile * WAVES * 32;
  const Row row(p, r0 + wave * 32 + (lane & 31), hk);
  const int limit = row.there ? q.limit(row.i) : 0;
  const int keys = q.seen(r0 / p.group, (r0 + WAVES * 32 - 1) / p.group);
  const int first_i = (r0 + wave * 32) / p.group, last_i = (r0 + wave * 32 + 31) / p.group;
  const int most = __builtin_amdgcn_readfirstlane(first_i < p.q_len ? q.seen(first_i, last_i) : 0);
  const int common = __builtin_amdgcn_readfirstlane(last_i < q.n ? q.limit(first_i) : 0);
  const bool counts = row.there && row.i < q.n;

  const bf16* const kb = static_cast<const bf16*>(p.k) + b * p.ks[0] + hk * p.ks[2];
  const bf16* const vb = static_cast<const bf16*>(p.v) + b * p.vs[0] + hk * p.vs[2];
  const typename L::template Loader<WAVES> load_k(wave, lane, p.ks[1], p.D), load_v(wave, lane, p.vs[1], p.D);
  const unsigned k_at = L::along_address(lane), kt_at = L::across_address(lane);
  auto load = [&](int j0, unsigned slot) {
    load_k.load(rows_from(kb, p.ks[1], j0, q.m, p.D), slot, wave);
    load_v.load(rows_from(vb, p.vs[1], j0, q.m, p.D), slot + L::BYTES, wave);
  };
  if (keys > 0) load(0, 0u);

  bf16x8 qf[KS], gf[KS];
  const int64_t at = (((int64_t)b * p.q_len + row.i) * p.heads + row.h) * p.D;
  const int64_t stat = ((int64_t)b * p.heads + row.h) * p.q_len + row.i;
  load_row<DP>(qf, static_cast<const bf16*>(p.q) + b * p.qs[0] + row.i * p.qs[1] + row.h * p.qs[2], counts, p.D, lane);
  take_sign(qf, p.scale);
  load_row<DP>(gf, static_cast<const bf16*>(p.d_o) + at, counts, p.D, lane);
  float delta = 0.f;
  {
    bf16x8 of[KS];
    load_row<DP>(of, static_cast<const bf16*>(p.o_in) + at, counts, p.D, lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) delta -= M::dot(of[ks], gf[ks]);
  }
  delta += other_half(delta);
  // (a row that sees nothing has no probabilities, whatever its lse says)
  const float lse = limit > 0 ? p.lse[stat] * LOG2E : INFINITY;
  if (row.there && lane < 32) {
    p.lse2[stat] = lse;
    p.delta[stat] = delta;
  }
  f32x16 dq[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dq[d] = zeros();
  const float factor = score_factor(p.scale);
  unsigned slot = 0;
  for (int j0 = 0; j0 < keys; j0 += TILE_ROWS, slot ^= SLOT) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (j0 + TILE_ROWS < keys) load(j0 + TILE_ROWS, slot ^ SLOT);
    if (j0 >= most) continue;
    f32x16 s[2], g[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = zeros();
#pragma unroll
      for (int r = 0; r < 16; ++r) g[t][r] = delta;
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t] = M::mma(L::along(slot + k_at, t, ks), qf[ks], s[t]);
        g[t] = M::mma(L::along(slot + L::BYTES + k_at, t, ks), gf[ks], g[t]);
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
#pragma unroll
      for (int d = 0; d < ND; ++d) dq[d] = M::mma(L::across(slot + kt_at, d, t), w, dq[d]);
    }
  }
  store_row<DP>(static_cast<bf16*>(p.dq) + at, row.there, dq, p.scale, p.D, lane);
}

// dk and dv: 32 keys a wave, their sums in registers over all queries of all heads that share them; tiles of 64 queries and their
// dO through the ring, with what dq's kernel left of their rows.
template <int DP, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 1) void attention_dkv_kernel(const AttentionArgs p) {
  typedef Tile<DP> L;
  typedef Mma<bf16> M;
  constexpr int KS = DP / 16, ND = DP / 32, STATS = 2 * L::BYTES, SLOT = STATS + 1024;
  __shared__ __align__(1024) unsigned char smem[2 * SLOT];
  asm volatile("" ::"v"((unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem) : "memory");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, hk, tile;
  locate(p, b, hk, tile);
  const Sequence q(p, b);
  const int j0 = tile * WAVES * 32, jw = j0 + wave * 32, j = jw + (lane & 31);
  const bool there = j < q.m;
  // the first query that sees key j (past the end: none does), and the first tile that the work-group and the wave look at
  const int first = there ? (q.causal ? j - q.shift + 1 : 0) : INT32_MAX;
  const int i_begin = q.causal && j0 - q.shift + 1 > 0 ? (j0 - q.shift + 1) / TILE_ROWS * TILE_ROWS : 0;
  const int i_wave = jw < q.m ? (q.causal ? jw - q.shift + 1 : 0) : INT32_MAX;
  const int i_whole = jw + 31 < q.m ? (q.causal ? jw + 31 - q.shift + 1 : 0) : INT32_MAX;   // from here on queries see all the wave's keys
  const int per_head = j0 < q.m && q.n > i_begin ? (q.n - i_begin + TILE_ROWS - 1) / TILE_ROWS : 0, steps = per_head * p.group;

  const typename L::template Loader<WAVES> load_q(wave, lane, p.qs[1], p.D), load_g(wave, lane, (int64_t)p.heads * p.D, p.D);
  const unsigned at_along = L::along_address(lane), at_across = L::across_address(lane);
  auto load = [&](int h, int i0, unsigned slot) {
    const int head = hk * p.group + h;
    load_q.load(rows_from(static_cast<const bf16*>(p.q) + b * p.qs[0] + head * p.qs[2], p.qs[1], i0, q.n, p.D), slot, wave);
    load_g.load(rows_from(static_cast<const bf16*>(p.d_o) + ((int64_t)b * p.q_len * p.heads + head) * p.D, (int64_t)p.heads * p.D, i0, q.n, p.D), slot + L::BYTES, wave);
    if (wave < 2) {   // 64 rows' statistics: zeros behind the last, where q and dO are zeros too and nothing comes of them
      const float* const stat = (wave == 0 ? p.lse2 : p.delta) + ((int64_t)b * p.heads + head) * p.q_len + i0;
      const uint64_t at = (uint64_t)stat;
      const u32x4 left = scalar(u32x4{(unsigned)at, (unsigned)(at >> 32), (unsigned)(q.n - i0) * 4u, 0x00020000u});
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(slot + STATS + wave * 256), "v"((unsigned)lane * 4u), "s"(left), "s"(0u) : "m0");
    }
  };
  if (steps > 0) load(0, i_begin, 0u);

  bf16x8 kf[KS], vf[KS];
  load_row<DP>(kf, static_cast<const bf16*>(p.k) + b * p.ks[0] + j * p.ks[1] + hk * p.ks[2], there, p.D, lane);
  take_sign(kf, p.scale);
  load_row<DP>(vf, static_cast<const bf16*>(p.v) + b * p.vs[0] + j * p.vs[1] + hk * p.vs[2], there, p.D, lane);
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dk[d] = dv[d] = zeros();
  const float factor = score_factor(p.scale);
  unsigned slot = 0;
  int h = 0, i0 = i_begin;
  for (int step = 0; step < steps; ++step, slot = SLOT - slot) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int i_now = i0;
    i0 += TILE_ROWS;
    if (i0 >= q.n) { i0 = i_begin; ++h; }
    if (step + 1 < steps) load(h, i0, SLOT - slot);
    if (i_now + TILE_ROWS <= i_wave) continue;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s = zeros(), g;
      float lse[16];
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
        const unsigned at = slot + STATS + (t * 32 + acc_row(r, lane)) * 4;
        const f32x4 a = *(lds_f32x4*)(uintptr_t)at, d = *(lds_f32x4*)(uintptr_t)(at + 256);
#pragma unroll
        for (int u = 0; u < 4; ++u) { lse[r + u] = a[u]; g[r + u] = d[u]; }
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = M::mma(L::along(slot + at_along, t, ks), kf[ks], s);
        g = M::mma(L::along(slot + L::BYTES + at_along, t, ks), vf[ks], g);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * factor - lse[r]);
      if (i_now < i_whole)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (i_now + t * 32 + acc_row(r, lane) < first) s[r] = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) g[r] *= s[r];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 w = M::of_acc(s, u), e = M::of_acc(g, u);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          dv[d] = M::mma(L::across(slot + L::BYTES + at_across, d, t * 2 + u), w, dv[d]);
          dk[d] = M::mma(L::across(slot + at_across, d, t * 2 + u), e, dk[d]);
        }
      }
    }
  }
  const int64_t at = (((int64_t)b * p.k_len + j) * p.kv_heads + hk) * p.D;
  store_row<DP>(static_cast<bf16*>(p.dk) + at, j < p.k_len, dk, p.scale, p.D, lane);
  store_row<DP>(static_cast<bf16*>(p.dv) + at, j < p.k_len, dv, 1.f, p.D, lane);
}

double pairs(const AttentionArgs& a) { return (double)a.batch * a.q_len * a.heads * a.k_len * a.D; }
unsigned groups_of(const AttentionArgs& a, int64_t rows, int per) { return (unsigned)((int64_t)a.batch * a.kv_heads * ((rows + per - 1) / per)); }

template <int DP>
hipError_t fwd(const AttentionArgs& a, hipStream_t s) {
  constexpr int WAVES = 4;
  note_attention_fwd(a, 2);
  return launch_kernel(kernel_label("attention_fwd_kernel", {lbl(DP), lbl(WAVES)}).c_str(), Work{4 * pairs(a), 0.0}, attention_fwd_kernel<DP, WAVES>,
                       dim3(groups_of(a, (int64_t)a.q_len * a.group, WAVES * 32)), dim3(WAVES * 64), s, a);
}

template <int DP>
hipError_t bwd(const AttentionArgs& a, hipStream_t s) {
  constexpr int WAVES = 4;
  note_attention_dq(a, 2);
  hipError_t e = launch_kernel(kernel_label("attention_dq_kernel", {lbl(DP), lbl(WAVES)}).c_str(), Work{6 * pairs(a), 0.0}, attention_dq_kernel<DP, WAVES>,
                               dim3(groups_of(a, (int64_t)a.q_len * a.group, WAVES * 32)), dim3(WAVES * 64), s, a);
  if (e != hipSuccess) return e;
  note_attention_dkv(a, 2);
  return launch_kernel(kernel_label("attention_dkv_kernel", {lbl(DP), lbl(WAVES)}).c_str(), Work{8 * pairs(a), 0.0}, attention_dkv_kernel<DP, WAVES>,
                       dim3(groups_of(a, a.k_len, WAVES * 32)), dim3(WAVES * 64), s, a);
}

}  // namespace

hipError_t launch_attention_fwd_bf16(const AttentionArgs& a, hipStream_t s) { return a.D <= 64 ? fwd<64>(a, s) : fwd<128>(a, s); }
hipError_t launch_attention_bwd_bf16(const AttentionArgs& a, hipStream_t s) { return a.D <= 64 ? bwd<64>(a, s) : bwd<128>(a, s); }

}  // namespace sk
