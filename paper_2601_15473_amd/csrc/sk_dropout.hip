// Dropout by a counter-based generator, with a residual added in the same pass: y = residual + x keep / (1 - p'), where p' = drop / 65536 and keep
// is whether the value's 16 bits are not below drop.  Nothing is stored for the gradient, which is the same call on dY without a residual.
//
// Bound by memory: 16383 tokens of 4096 in bf16, 403 MB, 77 us = 5.2 TB/s, without a residual 44 us = 6.1 (what was just written is read
// out of the Infinity Cache in part).
//
// Eight values a lane, one counter: Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as
// 1, 2, 3, 2011) makes four 32-bit words of (counter, key), used as eight of 16 bits, since a drop rate needs no more than that and the generator's
// multiplications, at a quarter of the VALU's rate, are half of the memory's time at eight values a counter and as much as it at four.
#include "sk_block_launch.h"
#include "sk_rows.h"

namespace sk {
namespace {

__device__ __forceinline__ uint4 philox(uint4 c, unsigned k0, unsigned k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((unsigned)(b >> 32) ^ c.y ^ k0, (unsigned)b, (unsigned)(a >> 32) ^ c.w ^ k1, (unsigned)a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

template <typename T, bool RESIDUAL>
__device__ __forceinline__ void drop8(const DropoutArgs& p, int64_t piece) {
  const int64_t at = piece * 8;
  const T *x = static_cast<const T*>(p.x) + at, *res = static_cast<const T*>(p.residual) + at;
  T* const y = static_cast<T*>(p.y) + at;
  const uint4 r = philox(make_uint4((unsigned)piece, (unsigned)(piece >> 32), p.offset[0], p.offset[1]), p.key[0], p.key[1]);
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
  auto kept = [&](float v, int i) {   // (dropped whatever it is)
    return ((i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu) >= p.drop ? v * p.scale : 0.f;
  };
  if (at + 8 <= p.n) {
    float v[8], u[8];
    load_values<T, 8>(v, x);
    if constexpr (RESIDUAL) load_values<T, 8>(u, res);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = kept(v[i], i);
      if constexpr (RESIDUAL) v[i] += u[i];
    }
    store_values<T, 8>(y, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < p.n) {
        float v = kept(load_one(x + i), i);
        if constexpr (RESIDUAL) v += load_one(res + i);
        store_one(y + i, v);
      }
  }
}

template <typename T, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs p) {
  const int64_t pieces = (p.n + 7) / 8, stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += stride) drop8<T, RESIDUAL>(p, i);
}

template <typename T>
hipError_t run(const DropoutArgs& a, hipStream_t s) {
  const int64_t pieces = (a.n + 7) / 8, groups = (pieces + 255) / 256;
  const unsigned grid = (unsigned)(groups < 8 * NUM_CUS * 4 ? groups : 8 * NUM_CUS * 4);
  const int esize = sizeof(T);
  note_matrix(a.x, 1, a.n, a.n, esize, false);
  note_matrix(a.residual, 1, a.n, a.n, esize, false);
  note_matrix(a.y, 1, a.n, a.n, esize, true);
  const Work work{2.0 * a.n, (a.residual != nullptr ? 3.0 : 2.0) * a.n * esize};
  if (a.residual != nullptr) return launch_kernel("dropout_kernel", work, dropout_kernel<T, true>, dim3(grid), dim3(256), s, a);
  return launch_kernel("dropout_kernel", work, dropout_kernel<T, false>, dim3(grid), dim3(256), s, a);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, bool f32, hipStream_t s) { return f32 ? run<float>(a, s) : run<bf16>(a, s); }

}  // namespace sk
