// The kernels of the 256 x 256 tile (sk_bf16_gemm256.h) and the column sums of dY that go with it.
#include "sk_bf16_gemm256.h"
#include "sk_launch.h"

namespace sk {

// One work-group per CU (the tile takes all of its LDS) walks the tiles index, index + grid, ...
template <int BM, int BN, int CHUNKS, int STEPS, bool A_KC, bool B_KC, typename OutT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void gemm_bf16_crew_kernel(const GemmArgs, const int total) {
  static_assert(BM == 256 && BN == 256 && CHUNKS == 2 && STEPS == 4, "256 x 256, two chunks of four k steps in LDS");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[GEMM256_LDS];
  gemm256_tiles<A_KC, B_KC, OutT, false>(smem, blockIdx.x, gridDim.x, total);
}
template <bool A_KC, bool B_KC, typename OutT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void gemm_bf16_far_kernel(const GemmArgs, const int total) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[GEMM256_LDS];
  gemm256_tiles<A_KC, B_KC, OutT, true>(smem, blockIdx.x, gridDim.x, total);
}

// ---- column sums ----
// Column sums of a dense row-major bf16 matrix [rows, cols] in fp32, the row range cut
// into `splits` runs of rows_per_split (out[s][c] = sum of rows of run s; fixed order).
// One work-group owns 512 columns of one run: a wave reads one whole 1 KB row segment
// per instruction (lane = 8 columns), sixteen of them in flight, the four waves stride over the
// rows, and their four partial sums meet in LDS and are added in wave order.
// (As a loop unrolled sixteen times by the compiler the last rows of a run, up to fifteen a wave, were one trip each: backward pass of 8192 tokens,
// 3072 -> 8192, R = 2048, 648 us, now 640; 9001, 4096 -> 8192 915 : 909; level where the sums ride beside a round of tiles.)
constexpr int COLSUM_COLS = 512;
__device__ __forceinline__ void colsum_body(const unsigned short* __restrict__ in, float* __restrict__ out,
                                            int rows, int cols, int rows_per_split, int bx, int by, float* part) {
  constexpr int NW = 4, AHEAD = 16, PLD = COLSUM_COLS + 8;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = bx * COLSUM_COLS + lane * 8;
  const int r_begin = by * rows_per_split;
  const int r_end = (r_begin + rows_per_split < rows) ? r_begin + rows_per_split : rows;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < cols) {
    for (int r = r_begin + wave; r < r_end; r += AHEAD * NW) {
      uint4 v[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {   // (past the run: its last row again, not added)
        const int at = r + u * NW < r_end ? r + u * NW : r_end - 1;
        v[u] = *reinterpret_cast<const uint4*>(in + (int64_t)at * cols + c);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const bool in_run = r + u * NW < r_end;
        const unsigned w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[2 * e] += in_run ? __builtin_bit_cast(float, w[e] << 16) : 0.f;
          acc[2 * e + 1] += in_run ? __builtin_bit_cast(float, w[e] & 0xffff0000u) : 0.f;
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[wave * PLD + lane * 8 + e] = acc[e];
  __syncthreads();
  for (int i = tid; i < COLSUM_COLS; i += 64 * NW) {
    const int gc = bx * COLSUM_COLS + i;
    if (gc < cols) {
      float s = part[i];
#pragma unroll
      for (int w = 1; w < NW; ++w) s += part[w * PLD + i];   // in wave order
      out[(int64_t)by * cols + gc] = s;
    }
  }
}

__global__ __launch_bounds__(256) void colsum_bf16_kernel(const unsigned short* __restrict__ in,
                                                          float* __restrict__ out, int rows,
                                                          int cols, int rows_per_split) {
  __shared__ float part[4 * (COLSUM_COLS + 8)];
  colsum_body(in, out, rows, cols, rows_per_split, blockIdx.x, blockIdx.y, part);
}

// A launch of the GEMM that does not fill the chip, with the column sums riding along:
// work-groups past the GEMM's own run the column-sum body on the CUs the GEMM leaves free --
// one streams from HBM while the other multiplies.
template <bool A_KC, bool B_KC, typename OutT, bool FAR>
__device__ __forceinline__ void gemm256_with_colsum(const int gemm_groups, const ColsumArgs& c) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[GEMM256_LDS];
  if ((int)blockIdx.x < gemm_groups) {
    gemm256_tiles<A_KC, B_KC, OutT, FAR>(smem, blockIdx.x, gemm_groups, gemm_groups);
  } else {
    const int w = blockIdx.x - gemm_groups;
    colsum_body(static_cast<const unsigned short*>(c.in), c.out, c.rows, c.cols, c.rows_per_split,
                w % c.col_groups, w / c.col_groups, reinterpret_cast<float*>(smem));
  }
}
template <int BM, int BN, int CHUNKS, int STEPS, bool A_KC, bool B_KC, typename OutT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void gemm_bf16_with_colsum_kernel(
    const GemmArgs, const int gemm_groups, const ColsumArgs c) {
  static_assert(BM == 256 && BN == 256 && CHUNKS == 2 && STEPS == 4, "256 x 256, two chunks of four k steps in LDS");
  gemm256_with_colsum<A_KC, B_KC, OutT, false>(gemm_groups, c);
}
template <bool A_KC, bool B_KC, typename OutT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void gemm_bf16_far_with_colsum_kernel(
    const GemmArgs, const int gemm_groups, const ColsumArgs c) {
  gemm256_with_colsum<A_KC, B_KC, OutT, true>(gemm_groups, c);
}

bool gemm256_supported(GemmKind kind, const GemmArgs& a) {
  bool a_kc, b_kc, f32;
  gemm_kind_traits(kind, a_kc, b_kc, f32);
  if (kind == GEMM_NN_F32_COLSUM || kind == GEMM_TN_F32) return false;   // no registers for the sums
  if (kind == GEMM_NT_F32 || kind == GEMM_TT_F32) return false;          // (no plan splits these on this tile)
  // ranges but the last: whole pairs of chunks (their zero chunks would be the next range's rows)
  if (a.splits > 1 && (a.k_per_split % 128 != 0 || a.k_per_split < 256)) return false;
  // byte offsets from a tile's origin are 32-bit: 256 rows of a k-contiguous operand, over the whole
  // k range, a few chunks of the other kind (is_far)
  const int64_t range = (int64_t)(a.splits > 1 ? a.k_per_split : a.K) + 512;
  if (!(a_kc ? within_window(256, a.lda, range, 2) : a.lda <= 1 << 20)) return false;
  if (!(b_kc ? within_window(256, a.ldb, range, 2) : a.ldb <= 1 << 20)) return false;
  // ... and rows of the result: all 256, or 32 where there is a variant for far ones
  return within_window(f32 || (a_kc && b_kc) ? 256 : 32, a.ldc, a.n_store > 0 ? a.n_store : a.N, f32 ? 4 : 2);
}

// Whether an operand that is not k-contiguous spans more over a tile's k range than offsets reach, or the
// result over its rows.
static bool is_far(bool a_kc, bool b_kc, const GemmArgs& a, int osize) {
  const int64_t range = (int64_t)(a.splits > 1 ? a.k_per_split : a.K) + 512;
  return (!a_kc && range * a.lda * 2 > 0x7fffffffLL) || (!b_kc && range * a.ldb * 2 > 0x7fffffffLL) ||
         !within_window(256, a.ldc, a.n_store > 0 ? a.n_store : a.N, osize);
}

template <bool A_KC, bool B_KC, typename OutT>
static hipError_t launch_crew(GemmArgs a, hipStream_t s) {
  a.tiles_m = (a.M + 255) / 256;
  a.tiles_n = (a.N + 255) / 256;
  if (a.n_store <= 0) a.n_store = a.N;
  const long long total = (long long)a.tiles_m * a.tiles_n * a.splits;
  if (total <= 0 || total > 0x7fffffffLL - NUM_CUS) return hipErrorInvalidValue;
  constexpr bool F32 = sizeof(OutT) == 4;
  note_gemm(a, A_KC, B_KC, 2, sizeof(OutT), F32);
  const dim3 grid((unsigned)(total < NUM_CUS ? total : NUM_CUS));
  const Work work = gemm_work(a, 2, sizeof(OutT), F32);
  if constexpr (!A_KC || !B_KC) {
    if (is_far(A_KC, B_KC, a, sizeof(OutT))) {
      static const std::string far = kernel_label("gemm_bf16_far_kernel", {lbl(A_KC), lbl(B_KC), F32 ? "float" : "bf16"});
      return launch_kernel(far.c_str(), work, gemm_bf16_far_kernel<A_KC, B_KC, OutT>, grid, dim3(256), s, a, (int)total);
    }
  }
  static const std::string name = kernel_label("gemm_bf16_crew_kernel", {lbl(256), lbl(256), lbl(2), lbl(4), lbl(A_KC), lbl(B_KC), F32 ? "float" : "bf16"});
  return launch_kernel(name.c_str(), work, gemm_bf16_crew_kernel<256, 256, 2, 4, A_KC, B_KC, OutT>, grid, dim3(256), s, a, (int)total);
}

hipError_t launch_gemm256_bf16(GemmKind kind, const GemmArgs& a, hipStream_t s) {
  if (!gemm256_supported(kind, a)) return hipErrorInvalidValue;
  switch (kind) {
    case GEMM_NN: return launch_crew<true, false, bf16>(a, s);
    case GEMM_NT: return launch_crew<true, true, bf16>(a, s);
    case GEMM_TT: return launch_crew<false, true, bf16>(a, s);
    case GEMM_NN_F32: return launch_crew<true, false, float>(a, s);
    case GEMM_TN_F32_PLAIN: return launch_crew<false, false, float>(a, s);
    case GEMM_TN: return launch_crew<false, false, bf16>(a, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_gemm256_with_colsum(GemmArgs a, const void* in, float* out, int rows, int cols, int splits,
                                      int rows_per_split, hipStream_t s) {
  if (!gemm256_supported(GEMM_NN_F32, a)) return hipErrorInvalidValue;
  a.tiles_m = (a.M + 255) / 256;
  a.tiles_n = (a.N + 255) / 256;
  if (a.n_store <= 0) a.n_store = a.N;
  ColsumArgs c;
  c.in = in; c.out = out; c.rows = rows; c.cols = cols; c.rows_per_split = rows_per_split;
  c.col_groups = (cols + COLSUM_COLS - 1) / COLSUM_COLS;
  const long long gg = (long long)a.tiles_m * a.tiles_n * a.splits;
  const long long grid = gg + (long long)c.col_groups * splits;
  if (gg <= 0 || grid > 0x7fffffffLL) return hipErrorInvalidValue;
  note_gemm(a, true, false, 2, 4, true);
  note_matrix(in, rows, cols, cols, 2, false);
  note_matrix(out, splits, cols, cols, 4, true);
  Work work = gemm_work(a, 2, 4, true);
  work.bytes += (double)rows * cols * 2 + (double)splits * cols * 4;
  return is_far(true, false, a, 4)
             ? launch_kernel("gemm_bf16_far_with_colsum_kernel<true, false, float>", work,
                             gemm_bf16_far_with_colsum_kernel<true, false, float>, dim3((unsigned)grid), dim3(256), s, a, (int)gg, c)
             : launch_kernel("gemm_bf16_with_colsum_kernel<256, 256, 2, 4, true, false, float>", work,
                             gemm_bf16_with_colsum_kernel<256, 256, 2, 4, true, false, float>,
                             dim3((unsigned)grid), dim3(256), s, a, (int)gg, c);
}

hipError_t launch_colsum_bf16(const void* in, float* out, int rows, int cols, int splits,
                              int rows_per_split, hipStream_t s) {
  const dim3 grid((unsigned)((cols + COLSUM_COLS - 1) / COLSUM_COLS), (unsigned)splits);
  note_matrix(in, rows, cols, cols, 2, false);
  note_matrix(out, splits, cols, cols, 4, true);
  return launch_kernel("colsum_bf16_kernel", Work{0.0, (double)rows * cols * 2 + (double)splits * cols * 4},
                       colsum_bf16_kernel, grid, dim3(256), s,
                       static_cast<const unsigned short*>(in), out, rows, cols, rows_per_split);
}

}  // namespace sk
