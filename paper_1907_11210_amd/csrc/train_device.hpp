// train_device.hpp -- device helpers of the operators around the convolutions.
#pragma once

#include <hip/hip_runtime.h>

#include "device.hpp"

namespace huge2 {

// VW consecutive elements as they lie in memory (bf16 as T = uint16_t, fp32 as
// uint32_t), moved with one load or store of 2, 4, 8 or 16 bytes.
template <typename T, int VW>
struct Pack {
  static constexpr int kBytes = (int)sizeof(T) * VW;
  uint32_t w[(kBytes + 3) / 4];
};

template <typename T, int VW>
__device__ __forceinline__ Pack<T, VW> load_pack(const T* p) {
  Pack<T, VW> r;
  if constexpr (sizeof(T) * VW == 16) {
    const u32x4 v = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = v[i];
  } else if constexpr (sizeof(T) * VW == 8) {
    const uint2 v = *(const uint2*)p;
    r.w[0] = v.x, r.w[1] = v.y;
  } else if constexpr (sizeof(T) * VW == 4) {
    r.w[0] = *(const uint32_t*)p;
  } else {
    r.w[0] = *(const uint16_t*)p;
  }
  return r;
}
// The same past the caches (16 bytes only).
template <typename T, int VW>
__device__ __forceinline__ Pack<T, VW> load_stream(const T* p) {
  Pack<T, VW> r;
  const u32x4 v = __builtin_nontemporal_load((const u32x4*)p);
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = v[i];
  return r;
}
template <typename T, int VW>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, VW>& r) {
  if constexpr (sizeof(T) * VW == 16)
    *(u32x4*)p = u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
  else if constexpr (sizeof(T) * VW == 8)
    *(uint2*)p = make_uint2(r.w[0], r.w[1]);
  else if constexpr (sizeof(T) * VW == 4)
    *(uint32_t*)p = r.w[0];
  else
    *(uint16_t*)p = (uint16_t)r.w[0];
}
// The same past the caches (uniform; 4 bytes and more).
template <typename T, int VW>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, VW>& r, int stream) {
  if constexpr (sizeof(T) * VW >= 4) {
    if (stream) {
      // (between two empty statements: the compiler would else make the two stores one
      // ahead of or behind the branch, and that an ordinary one)
      asm volatile("");
      if constexpr (sizeof(T) * VW == 16)
        __builtin_nontemporal_store(u32x4{r.w[0], r.w[1], r.w[2], r.w[3]}, (u32x4*)p);
      else if constexpr (sizeof(T) * VW == 8)
        __builtin_nontemporal_store((uint64_t)r.w[1] << 32 | r.w[0], (uint64_t*)p);
      else
        __builtin_nontemporal_store(r.w[0], (uint32_t*)p);
      asm volatile("");
      return;
    }
  }
  store_pack<T, VW>(p, r);
}
template <typename T, int VW>
__device__ __forceinline__ void unpack(const Pack<T, VW>& p, float (&f)[VW]) {
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    if constexpr (sizeof(T) == 4)
      f[e] = __uint_as_float(p.w[e]);
    else
      f[e] = __uint_as_float(e & 1 ? p.w[e / 2] & 0xffff0000u : p.w[e / 2] << 16);
  }
}
template <typename T, int VW>
__device__ __forceinline__ Pack<T, VW> pack(const float (&f)[VW]) {
  Pack<T, VW> p;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < VW; ++e) p.w[e] = __float_as_uint(f[e]);
  } else if constexpr (VW == 1) {
    p.w[0] = f32_to_bf16_rne(f[0]);
  } else {
#pragma unroll
    for (int e = 0; e < VW; e += 2) p.w[e / 2] = pack_bf16x2_rne(f[e], f[e + 1]);
  }
  return p;
}
// Makes the compiler take the registers for new values: what it unpacked of them
// before is unpacked again and not held beside them (twice the registers of bf16).
template <typename T, int VW>
__device__ __forceinline__ void forget(Pack<T, VW>& p) {
#pragma unroll
  for (auto& w : p.w) asm volatile("" : "+v"(w));
}

// Sum over the lanes that differ in the bits from `lo` (a power of two) up to a
// whole wave, in every one of them; the order is the same in each.
__device__ __forceinline__ float lanes_sum(float v, int lo) {
  for (int m = 32; m >= lo; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

}  // namespace huge2
