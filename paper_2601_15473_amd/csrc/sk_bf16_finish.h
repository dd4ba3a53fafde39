// How a bf16 product's tile leaves as a dense layer's result: z = acc + bias, y = act(z) + residual.
//
// Accumulators come with a row and four columns to a lane; the residual has to be read and the results written in whole lines.  So a wave turns its
// block of 32 rows over 64 columns at a time in fp32 through a strip of LDS of its own (no barrier: a wave's LDS operations execute in order): bias, activation and residual are applied to
// eight consecutive columns of a row, and y, and z for a backward pass, are rounded once.  16-byte pieces are XOR-swizzled by row, so that neither the
// column-wise writes nor the row-wise reads collide on banks.
//
// z is kept in bf16, as the operands are: what a backward pass needs of it is a derivative.
//
// Forward, us, with a bias alone (the plain product's epilogue, rounded in registers) : a residual : gelu : gelu with z stored: 4096 tokens, 1024 -> 4096 36 : 42 : 44 : 44; 16384, 512 -> 512
// 15 : 15 : 19 : 20; 4096, 4096 -> 1024 36 : 39 : 39 : 40; 16384, 4096 -> 11008 1090 : 1131 : 1164 : 1217.  Where a CU has one tile, nothing runs under the turn and the activation.  On fp32
// from the product, as a launch of its own, the last was 1835.
#pragma once
#include "sk_activation.h"
#include "sk_bf16_tile.h"

namespace sk {

struct FinishArgs {
  const void* residual;   // rows residual_ld elements apart, or null
  void* z;                // as the result, or null
  int64_t residual_ld;
};

template <int TN>
struct FinishStrip {
  static constexpr int COLS = TN >= 2 ? 64 : 32, BYTES = 32 * COLS * 4;
  static constexpr int LANES = COLS / 8, ROWS = 64 / LANES, PASSES = 32 / ROWS;   // of a row; rows that an instruction covers
  static constexpr int STEPS = TN * 32 / COLS;
  static_assert(TN * 32 % COLS == 0, "whole steps");
  static __device__ __forceinline__ int place(int row, int piece) { return row * (COLS * 4) + ((COLS == 64 ? piece ^ (row & 15) : piece ^ ((row >> 1) & 7)) << 4); }
};

// The bias of a lane's eight columns of every step (zeros without one, or past the last)
template <int TN>
__device__ __forceinline__ void finish_bias(uint4 (&bias)[FinishStrip<TN>::STEPS], const void* p, int col0, int N, int lane) {
  typedef FinishStrip<TN> S;
  const GWindow w = make_window(p, 0, p != nullptr ? N : 0, 2);
#pragma unroll
  for (int s = 0; s < S::STEPS; ++s) bias[s] = window_load16(w, (unsigned)(col0 + s * S::COLS + (lane % S::LANES) * 8) * 2u);
}

// The wave's block of 32 rows from `row` on, its columns from col0 on; acc as the MFMA leaves it, C [M, N] with rows ldc apart.
template <int ACT, int TN>
__device__ __forceinline__ void finish_rows(const f32x16 (&acc)[TN], const FinishArgs& f, const uint4 (&bias)[FinishStrip<TN>::STEPS], void* C, int64_t ldc, int64_t row,
                                            int col0, int M, int N, unsigned char* strip, int lane) {
  typedef FinishStrip<TN> S;
  const GWindow y_w = make_window(C, row * ldc + col0, (int64_t)M * ldc, 2);
  const GWindow z_w = make_window(f.z, row * ldc + col0, f.z != nullptr ? (int64_t)M * ldc : 0, 2);
  const GWindow r_w = make_window(f.residual, row * f.residual_ld + col0, f.residual != nullptr ? (int64_t)M * f.residual_ld : 0, 2);
#pragma unroll
  for (int s = 0; s < S::STEPS; ++s) {
    const int c = s * S::COLS + (lane % S::LANES) * 8, r0 = lane / S::LANES;
    const bool in = col0 + c < N;
    uint4 add[S::PASSES];
    if (f.residual != nullptr) {
#pragma unroll
      for (int u = 0; u < S::PASSES; ++u)
        add[u] = window_load16(r_w, in ? ((unsigned)(u * S::ROWS + r0) * (unsigned)f.residual_ld + (unsigned)c) * 2u : OOB_OFFSET);
    } else {
#pragma unroll
      for (int u = 0; u < S::PASSES; ++u) add[u] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int j = 0; j < S::COLS / 32; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& a = acc[s * (S::COLS / 32) + j];
        *reinterpret_cast<float4*>(strip + S::place(lane & 31, j * 8 + q * 2 + (lane >> 5))) = make_float4(a[q * 4 + 0], a[q * 4 + 1], a[q * 4 + 2], a[q * 4 + 3]);
      }
    const unsigned b[4] = {bias[s].x, bias[s].y, bias[s].z, bias[s].w};
#pragma unroll
    for (int u = 0; u < S::PASSES; ++u) {
      const int r = u * S::ROWS + r0, piece = (lane % S::LANES) * 2;
      const float4 lo = *reinterpret_cast<const float4*>(strip + S::place(r, piece)), hi = *reinterpret_cast<const float4*>(strip + S::place(r, piece + 1));
      const unsigned d[4] = {add[u].x, add[u].y, add[u].z, add[u].w};
      float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      const unsigned at = in ? ((unsigned)r * (unsigned)ldc + (unsigned)c) * 2u : OOB_OFFSET;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] += bf16_bits_to_float(b[e] & 0xffffu);
        v[2 * e + 1] += __builtin_bit_cast(float, b[e] & 0xffff0000u);
      }
      if (ACT != ACT_NONE && f.z != nullptr) window_store16(z_w, at, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = activation<ACT, false>(v[2 * e]) + bf16_bits_to_float(d[e] & 0xffffu);
        v[2 * e + 1] = activation<ACT, false>(v[2 * e + 1]) + __builtin_bit_cast(float, d[e] & 0xffff0000u);
      }
      window_store16(y_w, at, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
    }
  }
}

}  // namespace sk
