// Pieces of rows that a lane holds: 4 or 8 consecutive values of the storage type as fp32.
#pragma once
#include "sk_bf16_tile.h"

namespace sk {

template <typename T, int N>
__device__ __forceinline__ void load_values(float (&v)[N], const T* p) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 f = *reinterpret_cast<const float4*>(p + i);
      v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
    }
  } else {
    unsigned u[N / 2];
    if constexpr (N == 8) {
      const uint4 w = *reinterpret_cast<const uint4*>(p);
      u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
    } else {
      static_assert(N == 4, "4 or 8 values");
      const uint2 w = *reinterpret_cast<const uint2*>(p);
      u[0] = w.x; u[1] = w.y;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      v[2 * i] = __builtin_bit_cast(float, u[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
    }
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_values(T* p, const float (&v)[N]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else if constexpr (N == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

template <typename T>
__device__ __forceinline__ float load_one(const T* p) { return (float)*p; }
template <typename T>
__device__ __forceinline__ void store_one(T* p, float v) { *p = (T)v; }

}  // namespace sk
