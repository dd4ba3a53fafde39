// Tiles of 64 rows (keys, or queries; 32 where a wave has one to itself) in LDS that both kinds of MFMA operand are read from: along the features
// (scores) and across the rows (what is summed over them).
//
// A tile of DP features is DP / 64 panels (rounded up) of [64 rows][64 features], 128 bytes a row.  It goes from global memory straight
// into LDS, eight rows an instruction, and its 16-byte pieces are XOR-swizzled by row so that neither read conflicts: along the
// features 16 lanes read one piece of 16 consecutive rows (rows 2 i and 2 i + 1 share the 64 banks: the eight pairs
// need eight different pieces), across them 32 lanes read four pieces of four consecutive rows (rows i and i + 2
// need the two different halves of a row).  swizzle(row) = bit 1 of the row, then bits 3 and 2: a bijection of the pairs with their lowest bit on top.
#pragma once
#include "sk_attention.h"
#include "sk_bf16_lds.h"

namespace sk {

constexpr int TILE_ROWS = 64;

template <int DP, int ROWS = TILE_ROWS>
struct Tile {
  static constexpr int PANELS = (DP + 63) / 64, PANEL_BYTES = ROWS * 128, BYTES = PANELS * PANEL_BYTES;
  static constexpr int INSTRUCTIONS = BYTES / 1024;   // a wave's load fills eight rows of a panel
  static __device__ __forceinline__ int swizzle(int row) {
    const int t = (row >> 1) & 7;
    return ((t & 1) << 2) | (t >> 1);
  }

  // A wave's share of a tile's loads: instruction i of WAVES * i + wave.
  template <int WAVES>
  struct Loader {
    static constexpr int EACH = INSTRUCTIONS / WAVES, PER_PANEL = ROWS / 8 / WAVES;
    // (the swizzle has a period of 16 rows: a lone wave's odd instructions have another piece of it)
    static constexpr int KINDS = WAVES == 1 ? 2 : 1;
    static_assert(WAVES == 1 || WAVES == 4 || WAVES == 8, "a wave's instructions in a panel are a multiple of 16 rows apart, or turn by turn");
    unsigned at[PANELS][KINDS];   // byte offset of this lane's piece in its first rows; out of bounds past D
    unsigned step;                // bytes between instructions of a kind in a panel
    __device__ __forceinline__ Loader(int wave, int lane, int64_t stride, int D) {
      step = (unsigned)stride * 2u * (WAVES * KINDS * 8);
#pragma unroll
      for (int p = 0; p < PANELS; ++p)
#pragma unroll
        for (int k = 0; k < KINDS; ++k) {   // (an offset out of bounds stays so, a tile being at most 1 GB)
          const int row = (wave + k) * 8 + (lane >> 3), piece = p * 8 + ((lane & 7) ^ swizzle(row));
          at[p][k] = piece * 8 < D ? (unsigned)row * (unsigned)stride * 2u + (unsigned)piece * 16u : OOB_OFFSET;
        }
    }
    // Rows from the descriptor's start on to LDS byte `lds` on: instruction i of EACH, or all of them.
    template <int I>
    __device__ __forceinline__ void load_one(u32x4 rows, unsigned lds, int wave) const {
      constexpr int P = I / PER_PANEL, K = I % PER_PANEL;
      load_to_lds(lds + P * PANEL_BYTES + (K * WAVES + wave) * 1024, at[P][K % KINDS] + K / KINDS * step, rows, 0u);
    }
    __device__ __forceinline__ void load(u32x4 rows, unsigned lds, int wave) const {
      static_for<0, EACH>([&](auto ic) { load_one<decltype(ic)::value>(rows, lds, wave); });
    }
  };

  // LDS offsets of a lane's reads
  static __device__ __forceinline__ unsigned along_address(int lane) {
    const int row = lane & 31;
    return row * 128 + (((lane >> 5) ^ swizzle(row)) << 4);
  }
  static __device__ __forceinline__ unsigned across_address(int lane) {
    const int row = (lane >> 5) * 4 + ((lane & 15) >> 2), piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    return row * 128 + ((piece ^ swizzle(row)) << 4) + (lane & 1) * 8;
  }
  // Rows 32 block .. + 31, features 16 ks .. + 15
  static __device__ __forceinline__ bf16x8 along(unsigned address, int block, int ks) {
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
    return *(lds_bf16x8*)(uintptr_t)((address ^ ((ks & 3) << 5)) + (ks >> 2) * PANEL_BYTES + block * 4096);
  }
  // Features 32 d .. + 31, rows 16 step .. + 15 in the order of Mma::of_acc (rows 8 further: the swizzle's bit 1 the other way)
  static __device__ __forceinline__ bf16x8 across(unsigned address, int d, int step) {
    const unsigned lo_at = (address ^ ((d & 1) << 6)) + (d >> 1) * PANEL_BYTES + step * 2048;
    const unsigned hi_at = (address ^ 32u ^ ((d & 1) << 6)) + (d >> 1) * PANEL_BYTES + step * 2048 + 1024;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)lo_at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)hi_at);
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
  }
};

// A walk over an array's rows (D values each, `stride` elements apart), ROWS at a time, as buffers that read as zeros behind the last: a
// scalar's few additions a tile.
template <int ROWS>
struct Walk {
  uint64_t at;                     // of the tile's first row
  unsigned stride, row, whole;     // bytes from row to row, of a row, and of ROWS of them
  __device__ __forceinline__ Walk(const bf16* base, int64_t stride_, int first, int D) {
    const uint64_t a = (uint64_t)(base + first * stride_);
    at = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)a);
    stride = __builtin_amdgcn_readfirstlane((int)stride_ * 2);
    row = D * 2;
    whole = (ROWS - 1) * stride + row;
  }
  // The tile's rows, `left` of which there are from its first on (none where that is not positive)
  __device__ __forceinline__ u32x4 window(int left) const {
    const unsigned bytes = left >= ROWS ? whole : left > 0 ? (unsigned)(left - 1) * stride + row : 0u;
    return u32x4{(unsigned)at, (unsigned)(at >> 32), (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
  }
  __device__ __forceinline__ void skip(int rows) { at += (uint64_t)rows * stride; }
};

// The larger of a value and the other half-wave's.
__device__ __forceinline__ float max_halves(float x) {
  const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)s[0]), __builtin_bit_cast(float, (unsigned)s[1]));
}

}  // namespace sk
