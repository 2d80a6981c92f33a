// layer_device.hpp -- device helpers of the layer norm kernels.
#pragma once

#include "norm_device.hpp"

namespace huge2 {

// Vectors of a run whose length the vector's does not divide lie on any element: the
// hardware's loads and stores of global memory need no more than the element's alignment.
// The last vector of such a run ends with it and repeats elements of the one before.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <typename T, int VW>
__device__ __forceinline__ Pack<T, VW> load_run(const T* p) {
  if constexpr (VW == 1) return load_pack<T, 1>(p);
  Pack<T, VW> r;
  const u32x4 v = *(const u32x4_any*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = v[i];
  return r;
}
template <typename T, int VW>
__device__ __forceinline__ void store_run(T* p, const Pack<T, VW>& r, int stream) {
  if constexpr (VW == 1) return store_pack<T, 1>(p, r);
  const u32x4 v = {r.w[0], r.w[1], r.w[2], r.w[3]};
  if (stream) {
    asm volatile("");  // (as in store_pack)
    __builtin_nontemporal_store(v, (u32x4_any*)p);
    asm volatile("");
  } else {
    *(u32x4_any*)p = v;
  }
}

// A vector's place in a run of `len` elements: its first element, and how many of its
// own the vector before it has already (those count once).
struct Piece {
  int at, skip;
  bool in;
};
template <int VW, bool RAGGED>
__device__ __forceinline__ Piece piece(long long first, int len) {
  Piece p;
  p.in = first < len;
  p.at = p.in ? (int)first : 0;
  p.skip = 0;
  if (RAGGED && p.in && p.at + VW > len) {
    p.skip = p.at + VW - len;
    p.at = len - VW;
  }
  return p;
}

// xh and dz of one value.
template <int ACT, typename T>
__device__ __forceinline__ void layer_dz(float x, float dy, const Channel& k, float& xh,
                                         float& dz) {
  constexpr bool kSmooth = ACT == HUGE2_NORM_TANH || ACT == HUGE2_NORM_SILU;
  xh = (x - k.mean) * k.rstd;
  const float z = kSmooth ? fmaf(xh, k.gamma, k.beta) : norm_z(xh, k.gamma, k.beta);
  dz = norm_act_grad<ACT, T>(dy, z);
}

}  // namespace huge2
