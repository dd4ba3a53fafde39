// Launchers of the dense layers' fused products (internal).
#pragma once
#include "sk_bf16_finish.h"
#include "sk_launch.h"

namespace sk {

// y = act(A . B^T + bias) + residual, A [M, K], B [N, K], y = a.C [M, N] rows a.ldc apart, z as y
hipError_t launch_dense_bf16(int tile, int act, const GemmArgs& a, const FinishArgs& f, hipStream_t s);
hipError_t launch_dense_crew(int act, const GemmArgs& a, const FinishArgs& f, hipStream_t s);              // TILE_256x256 of the above
hipError_t launch_dense_f32(int tile, int act, const GemmArgs& a, const FinishArgs& f, hipStream_t s);      // in fp32, TILE_64x64 or TILE_128x128
hipError_t launch_dense_few_rows(int act, const GemmArgs& a, const FinishArgs& f, hipStream_t s);          // one range of few rows of A
void note_dense(const GemmArgs& a, const FinishArgs& f, int esize = 2);
Work dense_work(const GemmArgs& a, const FinishArgs& f, int esize = 2);

}  // namespace sk
