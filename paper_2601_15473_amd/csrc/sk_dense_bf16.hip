// A dense layer's product in bf16 with all that follows it in its epilogue (sk_bf16_finish.h): the GEMM's tiles, one kernel an activation.
// The tile is dense_tile's: of 26 layers of 512 to 16384 tokens, 256 to 4096 wide, with gelu and z or with a residual, all but one were on the best of the five or within 5 % of it
// (3000 tokens of 1536 -> 1536 with gelu, 31 : 28 us).
#include "sk_bf16_ring.h"
#include "sk_bf16_staged.h"
#include "sk_dense_launch.h"
#include "sk_launch.h"

namespace sk {

template <int BM, int BN, int ACT, bool RING>
__global__ __launch_bounds__(256) void dense_bf16_kernel(const GemmArgs p, const FinishArgs f) {
  typedef typename std::conditional<RING, RingTile<BM, BN, true, true, bf16, false, ACT>, GemmTile<BM, BN, true, true, bf16, false, ACT>>::type G;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[G::LDS_BYTES];
  G::run(p, blockIdx.x, smem, f);
}

void note_dense(const GemmArgs& a, const FinishArgs& f, int esize) {
  note_gemm(a, true, true, esize, esize, false);
  if (f.residual) note_matrix(f.residual, a.M, a.N, f.residual_ld, esize, false);
  note_matrix(f.z, a.M, a.N, a.ldc, esize, true);
}
Work dense_work(const GemmArgs& a, const FinishArgs& f, int esize) {
  Work w = gemm_work(a, esize, esize, false);
  w.bytes += (double)esize * a.M * a.N * ((f.residual != nullptr) + (f.z != nullptr));
  return w;
}

template <int BM, int BN, int ACT, bool RING>
static hipError_t launch_tile(GemmArgs a, const FinishArgs& f, hipStream_t s) {
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + BN - 1) / BN;
  const long long total = (long long)a.tiles_m * a.tiles_n;
  if (a.splits != 1 || total <= 0 || total > 0x7fffffffLL || !within_window(BM, a.lda, BK, 2) || !within_window(BN, a.ldb, BK, 2) || !within_window(32, a.ldc, a.N, 2) ||
      !within_window(32, f.residual_ld, a.N, 2))
    return hipErrorInvalidValue;
  note_dense(a, f);
  static const std::string name = kernel_label("dense_bf16_kernel", {lbl(BM), lbl(BN), lbl(ACT), lbl(RING)});
  return launch_kernel(name.c_str(), dense_work(a, f), dense_bf16_kernel<BM, BN, ACT, RING>, dim3((unsigned)total), dim3(256), s, a, f);
}

template <int ACT>
static hipError_t launch_by_tile(int tile, const GemmArgs& a, const FinishArgs& f, hipStream_t s) {
  auto groups = [&](int bm, int bn) { return (long long)((a.M + bm - 1) / bm) * ((a.N + bn - 1) / bn); };
  switch (tile) {
    case TILE_256x256: return launch_dense_crew(ACT, a, f, s);
    case TILE_256x128: return launch_tile<256, 128, ACT, true>(a, f, s);
    // (on a ring while they make one round, as the product by itself)
    case TILE_128x128: return groups(128, 128) <= NUM_CUS ? launch_tile<128, 128, ACT, true>(a, f, s) : launch_tile<128, 128, ACT, false>(a, f, s);
    case TILE_128x64: return launch_tile<128, 64, ACT, false>(a, f, s);
    case TILE_64x128: return launch_tile<64, 128, ACT, false>(a, f, s);
    case TILE_64x64: return groups(64, 64) <= 2 * NUM_CUS ? launch_tile<64, 64, ACT, true>(a, f, s) : launch_tile<64, 64, ACT, false>(a, f, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_dense_bf16(int tile, int act, const GemmArgs& a, const FinishArgs& f, hipStream_t s) {
  switch (act) {
    case ACT_NONE: return launch_by_tile<ACT_NONE>(tile, a, f, s);
    case ACT_RELU: return launch_by_tile<ACT_RELU>(tile, a, f, s);
    case ACT_GELU: return launch_by_tile<ACT_GELU>(tile, a, f, s);
    case ACT_GELU_TANH: return launch_by_tile<ACT_GELU_TANH>(tile, a, f, s);
    case ACT_SILU: return launch_by_tile<ACT_SILU>(tile, a, f, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sk
