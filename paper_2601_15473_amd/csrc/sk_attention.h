// What the attention kernels share: MFMA operands of either type, the rows and keys of a work-group, masks.
//
// Every product of these kernels has its C operand as [32 x 32] with the column in the lane (lane % 32) and rows
// 8 (r / 4) + 4 (lane / 32) + r % 4 in register r.  The probabilities come out of one product with the reduced
// dimension of the next along the registers, and a contraction may run in any order, so they go into the next one as
// they lie, only rounded: register r is element r % 8 of k step r / 8, for which the other operand's rows are read in
// the same order.  No probability passes through LDS or another lane.
//
// Rounded: in bf16 a probability (and ds) is off by up to 2^-9 of itself there, as any bf16 product's operand, and what is summed of it by 0.0022 to
// 0.0024 of 64 bits, where one rounding of an exact result is 0.0017.  In two bf16 parts it would be another product for each that takes it, where products are the
// bound.  The sum that divides, and lse, are of the weights before rounding: of 32 bits throughout.
#pragma once
#include "sk_bf16_tile.h"
#include "sk_block_launch.h"

namespace sk {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

template <typename T>
struct Mma;

template <>
struct Mma<bf16> {
  typedef bf16x8 Frag;                 // of a lane: 16 bytes
  static constexpr int E = 8;          // values in them
  static constexpr int STEP = 16;      // of the contraction, covered by a fragment
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ Frag of_acc(const f32x16& p, int s) {
    uint4 u;
    u.x = pack_bf16x2(p[8 * s + 0], p[8 * s + 1]);
    u.y = pack_bf16x2(p[8 * s + 2], p[8 * s + 3]);
    u.z = pack_bf16x2(p[8 * s + 4], p[8 * s + 5]);
    u.w = pack_bf16x2(p[8 * s + 6], p[8 * s + 7]);
    return __builtin_bit_cast(Frag, u);
  }
  // What rounding left off fragment s of them
  static __device__ __forceinline__ Frag rest_of_acc(const f32x16& p, int s, Frag rounded) {
    uint4 u;
    u.x = pack_bf16x2(p[8 * s + 0] - (float)rounded[0], p[8 * s + 1] - (float)rounded[1]);
    u.y = pack_bf16x2(p[8 * s + 2] - (float)rounded[2], p[8 * s + 3] - (float)rounded[3]);
    u.z = pack_bf16x2(p[8 * s + 4] - (float)rounded[4], p[8 * s + 5] - (float)rounded[5]);
    u.w = pack_bf16x2(p[8 * s + 6] - (float)rounded[6], p[8 * s + 7] - (float)rounded[7]);
    return __builtin_bit_cast(Frag, u);
  }
  static __device__ __forceinline__ float dot(Frag a, Frag b) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (float)a[j] * (float)b[j];
    return s;
  }
};

template <>
struct Mma<float> {
  typedef f32x4 Frag;
  static constexpr int E = 4;
  static constexpr int STEP = 8;
  static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
  // Rows row0 .. + 31 of a row-major tile, contraction along its rows' elements
  static __device__ __forceinline__ Frag along(const float* tile, int ld, int row0, int ks, int lane) {
    return *reinterpret_cast<const Frag*>(tile + (row0 + (lane & 31)) * ld + ks * 8 + (lane >> 5) * 4);
  }
  // Columns col0 .. + 31 of it, contraction along rows row0 .. + 31 in the order of of_acc
  static __device__ __forceinline__ Frag across(const float* tile, int ld, int row0, int s, int col0, int lane) {
    const float* p = tile + (row0 + s * 8 + (lane >> 5) * 4) * ld + col0 + (lane & 31);
    return Frag{p[0], p[ld], p[2 * ld], p[3 * ld]};
  }
  static __device__ __forceinline__ Frag of_acc(const f32x16& p, int s) { return Frag{p[4 * s], p[4 * s + 1], p[4 * s + 2], p[4 * s + 3]}; }
  static __device__ __forceinline__ float dot(Frag a, Frag b) { return a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]; }
};

__device__ __forceinline__ f32x16 zeros() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// Rows (a row of the result to a lane) that do not count are zeros whatever was summed for them: a weight of zero times what is not a number is none.
template <int ND>
__device__ __forceinline__ void zeros_unless(bool counts, f32x16 (&acc)[ND]) {
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = counts ? acc[d][r] : 0.f;
}

// Row of register r in the C operand's lane layout.
__device__ __forceinline__ int acc_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// The other half of the wave's value.
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// What a sequence has: n queries, m keys, and by how much the keys that query i sees end past i (limit(i) keys).
struct Sequence {
  int n, m, shift;
  bool causal;
  __device__ __forceinline__ Sequence(const AttentionArgs& p, int b) {
    n = p.q_len; m = p.k_len;
    if (p.q_lengths != nullptr) n = p.q_lengths[b];
    if (p.k_lengths != nullptr) m = p.k_lengths[b];
    n = n < 0 ? 0 : n > p.q_len ? p.q_len : n;
    m = m < 0 ? 0 : m > p.k_len ? p.k_len : m;
    causal = p.causal != 0;
    shift = m - n + 1;
  }
  // Keys 0 .. limit(i) - 1 are those that query i sees (none where it is not positive).
  __device__ __forceinline__ int limit(int i) const {
    if (i >= n) return 0;
    return !causal ? m : i + shift < m ? i + shift : m;
  }
  // ... that any of queries first .. last sees: the last one's
  __device__ __forceinline__ int seen(int first, int last) const {
    return first >= n ? 0 : limit(last < n ? last : n - 1);
  }
};

// The trace's view of a strided [batch, tokens, heads, D] array.
inline void note_strided(const void* base, int esize, int64_t batch, int64_t tokens, int64_t heads, int64_t D, const int64_t (&st)[3]) {
  note_matrix(base, 1, (batch - 1) * st[0] + (tokens - 1) * st[1] + (heads - 1) * st[2] + D, 0, esize, false);
}
inline void note_attention_inputs(const AttentionArgs& a, int esize) {
  if (!tracing()) return;
  note_strided(a.q, esize, a.batch, a.q_len, a.heads, a.D, a.qs);
  note_strided(a.k, esize, a.batch, a.k_len, a.kv_heads, a.D, a.ks);
  note_strided(a.v, esize, a.batch, a.k_len, a.kv_heads, a.D, a.vs);
  note_matrix(a.q_lengths, 1, a.batch, a.batch, 4, false);
  note_matrix(a.k_lengths, 1, a.batch, a.batch, 4, false);
}

inline int64_t rows_of(const AttentionArgs& a) { return (int64_t)a.batch * a.q_len * a.heads; }

inline void note_attention_fwd(const AttentionArgs& a, int esize) {
  note_attention_inputs(a, esize);
  note_matrix(a.o, rows_of(a), a.D, a.D, esize, true);
  note_matrix(a.lse, 1, rows_of(a), rows_of(a), 4, true);
  note_matrix(a.o_rest, rows_of(a), a.D, a.D, esize, true);
}
inline void note_attention_dq(const AttentionArgs& a, int esize) {
  note_attention_inputs(a, esize);
  note_matrix(a.d_o, rows_of(a), a.D, a.D, esize, false);
  note_matrix(a.o_in, rows_of(a), a.D, a.D, esize, false);
  note_matrix(a.o_rest, rows_of(a), a.D, a.D, esize, false);
  note_matrix(a.lse, 1, rows_of(a), rows_of(a), 4, false);
  note_matrix(a.lse2, 1, rows_of(a), rows_of(a), 4, true);
  note_matrix(a.delta, 1, rows_of(a), rows_of(a), 4, true);
  if (a.q_shares > 1) note_matrix(a.q_partial, a.q_shares * rows_of(a), a.D, a.D, 4, true);
  else note_matrix(a.dq, rows_of(a), a.D, a.D, esize, true);
}
inline void note_attention_dkv(const AttentionArgs& a, int esize) {
  note_attention_inputs(a, esize);
  note_matrix(a.d_o, rows_of(a), a.D, a.D, esize, false);
  note_matrix(a.lse2, 1, rows_of(a), rows_of(a), 4, false);
  note_matrix(a.delta, 1, rows_of(a), rows_of(a), 4, false);
  const int64_t keys = (int64_t)a.batch * a.k_len * a.kv_heads;
  if (a.parts > 1) {
    note_matrix(a.partial, 2 * a.parts * keys, a.D, a.D, 4, true);
  } else {
    note_matrix(a.dk, keys, a.D, a.D, esize, true);
    note_matrix(a.dv, keys, a.D, a.D, esize, true);
  }
}

// Kernels are built for 32, 64, 96 and 128 features; those behind a head's own are zeros.  Forward and backward passes of 16 sequences of 512, 16 heads
// of 32 take 91 us on 32 and 108 on 64, of 80 188 on 96 and 203 on 128; four of 2048, 16 heads on 8 of 96, causal: 308 and 362; in fp32, eight
// of 256, eight heads of 32: 76 and 120, of 80: 178 and 220.
template <typename Run>
hipError_t by_width(int D, Run&& run) {
  if (D <= 32) return run(IntC<32>{});
  if (D <= 64) return run(IntC<64>{});
  if (D <= 96) return run(IntC<96>{});
  return run(IntC<128>{});
}
#define SK_LABEL_BY_WIDTH(name, DP) (DP == 32 ? name "<32>" : DP == 64 ? name "<64>" : DP == 96 ? name "<96>" : name "<128>")

}  // namespace sk
