// The dense layers' product on the 256 x 256 tile (sk_bf16_gemm256.h), one kernel an activation.  Bound as the product: 16384 tokens, 4096 -> 11008, silu, 1204 to 1237 us (1.23 to 1.19 PFLOP/s; the
// library's 8192^3 product 1.23).
#include "sk_bf16_gemm256.h"
#include "sk_dense_launch.h"

namespace sk {

template <int ACT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void dense_crew_kernel(const CrewFinishArgs, const int total) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[GEMM256_LDS];
  gemm256_tiles<true, true, bf16, false, ACT>(smem, blockIdx.x, gridDim.x, total);
}

template <int ACT>
static hipError_t launch(const CrewFinishArgs& c, int total, hipStream_t s) {
  static const std::string name = kernel_label("dense_crew_kernel", {lbl(ACT)});
  return launch_kernel(name.c_str(), dense_work(c.g, c.f), dense_crew_kernel<ACT>, dim3((unsigned)(total < NUM_CUS ? total : NUM_CUS)), dim3(256), s, c, total);
}

hipError_t launch_dense_crew(int act, const GemmArgs& a, const FinishArgs& f, hipStream_t s) {
  if (!gemm256_supported(GEMM_NT, a) || a.splits != 1 || !within_window(32, f.residual_ld, a.N, 2)) return hipErrorInvalidValue;
  CrewFinishArgs c{a, f};
  c.g.tiles_m = (a.M + 255) / 256;
  c.g.tiles_n = (a.N + 255) / 256;
  c.g.n_store = a.N;
  const long long total = (long long)c.g.tiles_m * c.g.tiles_n;
  if (total <= 0 || total > 0x7fffffffLL - NUM_CUS) return hipErrorInvalidValue;
  note_dense(c.g, f);
  switch (act) {
    case ACT_NONE: return launch<ACT_NONE>(c, (int)total, s);
    case ACT_RELU: return launch<ACT_RELU>(c, (int)total, s);
    case ACT_GELU: return launch<ACT_GELU>(c, (int)total, s);
    case ACT_GELU_TANH: return launch<ACT_GELU_TANH>(c, (int)total, s);
    case ACT_SILU: return launch<ACT_SILU>(c, (int)total, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sk
