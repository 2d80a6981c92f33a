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

// Sums over lanes without LDS.  v of the lane that DPP's control gives.
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
  return __uint_as_float(
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int kPairs = 0xb1, kQuads = 0x4e;  // lane ^ 1, lane ^ 2
constexpr int kMirror4 = 0x1b, kMirror8 = 0x141, kMirror16 = 0x140, kRotate8 = 0x128;
__device__ __forceinline__ float from_xor4(float v) {
  return from_lane<kMirror4>(from_lane<kMirror8>(v));
}
// The upper halves of pairs of 16 (32) lanes of a, and the lower ones of b, change places: the
// sum of the two is a's of both halves in the lower, b's in the upper.
__device__ __forceinline__ float swap_sum16(float a, float b) {
  const auto r =
      __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float swap_sum32(float a, float b) {
  const auto r =
      __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum over 2^log2 lanes side by side (of a wave), the same bits in each of them: every step
// adds two sums of as many lanes.
__device__ __forceinline__ float wave_sum(float v) {
  v += from_lane<kPairs>(v);
  v += from_lane<kQuads>(v);
  v += from_lane<kMirror8>(v);
  v += from_lane<kMirror16>(v);
  v = swap_sum16(v, v);
  return swap_sum32(v, v);
}
__device__ __forceinline__ float side_sum(float v, int log2) {
  if (log2 >= 6) return wave_sum(v);  // (one branch)
  if (log2 > 0) v += from_lane<kPairs>(v);
  if (log2 > 1) v += from_lane<kQuads>(v);
  if (log2 > 2) v += from_lane<kMirror8>(v);
  if (log2 > 3) v += from_lane<kMirror16>(v);
  if (log2 > 4) v = swap_sum16(v, v);
  return v;
}
// Sums of N values (a power of two up to 16) over the lanes that differ in the bits from 2^log2
// (at most 8) up.  Half of the values change places with half of the lanes at each of the three
// upper bits, so that a lane ends with the sums of N / 8 values (at least one), from scatter_at.
template <int N>
__device__ __forceinline__ int scatter_at() {
  const int lane = threadIdx.x & 63;
  return (lane >> 5) * (N / 2) + (lane >> 4 & 1) * (N / 4) + (lane >> 3 & 1) * (N / 8);
}
template <int N>
__device__ __forceinline__ void scatter_sum(float (&v)[N], int log2) {
  constexpr int kHalf = N > 1 ? N / 2 : 1, kQuarter = N > 3 ? N / 4 : 1;
  constexpr int kEighth = N > 7 ? N / 8 : 1;
#pragma unroll
  for (int e = 0; e < kHalf; ++e) v[e] = swap_sum32(v[e], v[N > 1 ? e + kHalf : e]);
#pragma unroll
  for (int e = 0; e < kQuarter; ++e) v[e] = swap_sum16(v[e], v[N > 3 ? e + kQuarter : e]);
  const bool up = threadIdx.x & 8;
#pragma unroll
  for (int e = 0; e < kEighth; ++e) {
    const float other = v[N > 7 ? e + kEighth : e];
    v[e] = (up ? other : v[e]) + from_lane<kRotate8>(up ? v[e] : other);
  }
#pragma unroll
  for (int e = 0; e < kEighth; ++e) {
    if (log2 < 3) v[e] += from_xor4(v[e]);
    if (log2 < 2) v[e] += from_lane<kQuads>(v[e]);
    if (log2 < 1) v[e] += from_lane<kPairs>(v[e]);
  }
}

// y of a value less its mean.  A ReLU's z is rounded as the gradient rounds it.
template <int ACT, typename T>
__device__ __forceinline__ float layer_value(float d, float rstd, float gamma, float beta) {
  const float z =
      ACT == HUGE2_NORM_RELU ? norm_z(d * rstd, gamma, beta) : fmaf(d, rstd * gamma, beta);
  return norm_act<ACT, T>(z);
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
