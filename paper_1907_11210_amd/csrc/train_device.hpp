// train_device.hpp -- device helpers of the operators around the convolutions.
#pragma once

#include <hip/hip_runtime.h>

#include "device.hpp"

namespace huge2 {

// VW consecutive elements, moved with one load or store (bf16 as uint16_t, fp32
// as uint32_t).
template <typename T, int VW>
struct alignas(sizeof(T) * VW) Pack {
  T v[VW];
};

template <typename T>
__device__ __forceinline__ T from_f32(float f) {
  if constexpr (sizeof(T) == 2)
    return f32_to_bf16_rne(f);
  else
    return __float_as_uint(f);
}

template <typename T, int VW>
__device__ __forceinline__ Pack<T, VW> load_pack(const T* p) {
  return *(const Pack<T, VW>*)p;
}
template <typename T, int VW>
__device__ __forceinline__ void unpack(const Pack<T, VW>& p, float (&f)[VW]) {
#pragma unroll
  for (int e = 0; e < VW; ++e) f[e] = to_f32<T>(p.v[e]);
}
template <typename T, int VW>
__device__ __forceinline__ Pack<T, VW> pack(const float (&f)[VW]) {
  Pack<T, VW> p;
  if constexpr (sizeof(T) == 2 && VW % 2 == 0) {
#pragma unroll
    for (int e = 0; e < VW; e += 2) {
      const uint32_t w = pack_bf16x2_rne(f[e], f[e + 1]);
      p.v[e] = (T)w;
      p.v[e + 1] = (T)(w >> 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < VW; ++e) p.v[e] = from_f32<T>(f[e]);
  }
  return p;
}

// Sum over the lanes that differ in the bits from `lo` (a power of two) up to a
// whole wave, in every one of them; the order is the same in each.
__device__ __forceinline__ float lanes_sum(float v, int lo) {
  for (int m = 32; m >= lo; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

}  // namespace huge2
