// norm_device.hpp -- device helpers of the group norm kernels.
#pragma once

#include <cmath>
#include <type_traits>

#include "huge2_train.h"
#include "train.hpp"
#include "train_device.hpp"

namespace huge2 {

// z of a normalised value where its sign counts.  Rounded after the product, here and
// in the gradient, so that both see the same sign (and the same as a framework without
// fused multiply-adds).
__device__ __forceinline__ float norm_z(float xh, float gamma, float beta) {
#pragma clang fp contract(off)
  return xh * gamma + beta;
}

// f(integral_constant) of a huge2_norm_activation: one branch around a whole loop
// (one for each value took half of the gradient's instructions).
template <typename F>
__device__ __forceinline__ void by_act(int act, F&& f) {
  switch (act) {
    case HUGE2_NORM_RELU: return f(std::integral_constant<int, HUGE2_NORM_RELU>());
    case HUGE2_NORM_TANH: return f(std::integral_constant<int, HUGE2_NORM_TANH>());
    case HUGE2_NORM_SILU: return f(std::integral_constant<int, HUGE2_NORM_SILU>());
    default: return f(std::integral_constant<int, HUGE2_NORM_NONE>());
  }
}

// For bf16 tensors on the hardware's exponential and reciprocal, each within 1 unit in the
// last place: with them the activations stay below the memory's time (with the library's
// expf and a division the gradient of SiLU took 1.8 times as long).  The exponent's
// rounding makes exp(z) off by |z| 2^-24 of itself, which 1 / (1 + exp(-z)) keeps
// only where it is itself small.  fp32 results would show these errors (tanh 10 units of 2^-24
// of the value, SiLU 16): there the library's functions and a division (64 images of 128x32x32
// in NCHW: tanh 15.4 -> 17.6 us, its gradient 28.1 -> 30.6, SiLU 14.2 -> 17.7 and 26.0 -> 31.3).
template <typename T>
constexpr bool kFastAct = sizeof(T) == 2;
template <typename T>
__device__ __forceinline__ float sigmoid(float z) {
  if constexpr (kFastAct<T>)
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
  else
    return 1.f / (1.f + expf(-z));
}
// 1 - 2 / (exp(2z) + 1), and its series near 0, where that cancels: the term left out
// is 62/2835 z^8 of the value, 6e-8 at 0.2.
template <typename T>
__device__ __forceinline__ float tanh_of(float z) {
  if constexpr (!kFastAct<T>) return tanhf(z);
  const float far =
      1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * 2.88539008177792681f) + 1.f);
  const float q = z * z;
  const float near = z + z * q * (-1.f / 3 + q * (2.f / 15 - q * (17.f / 315)));
  return fabsf(z) < 0.2f ? near : far;
}

template <int ACT, typename T>
__device__ __forceinline__ float norm_act(float z) {
  if constexpr (ACT == HUGE2_NORM_RELU) return z < 0.f ? 0.f : z;
  if constexpr (ACT == HUGE2_NORM_TANH) return tanh_of<T>(z);
  if constexpr (ACT == HUGE2_NORM_SILU)
    return kFastAct<T> ? z * sigmoid<T>(z) : z / (1.f + expf(-z));
  return z;
}
// dy * activation'(z)
template <int ACT, typename T>
__device__ __forceinline__ float norm_act_grad(float dy, float z) {
  if constexpr (ACT == HUGE2_NORM_RELU) return z > 0.f ? dy : 0.f;
  if constexpr (ACT == HUGE2_NORM_TANH) {
    const float th = tanh_of<T>(z);
    return dy * (1.f - th * th);
  }
  if constexpr (ACT == HUGE2_NORM_SILU) {
    const float s = sigmoid<T>(z);
    return dy * (s * (1.f + z * (1.f - s)));
  }
  return dy;
}

// Sum of one value a thread over a workgroup (whole waves, at most 16), in every
// thread; lds: a float for each wave.
__device__ __forceinline__ float block_sum(float v, float* lds) {
  v = lanes_sum(v, 1);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = lds[0];
  for (int w = 1; w < waves; ++w) s += lds[w];
  return s;
}

// A thread's vectors: their mean and the squares around it, per channel where a
// vector may span groups, else over all in s[0], m2[0].
template <typename T, int VW, int R, bool SPAN>
__device__ __forceinline__ void own_stats(Pack<T, VW> (&f)[R], int mine, float (&s)[VW],
                                          float (&m2)[VW]) {
#pragma unroll
  for (int e = 0; e < VW; ++e) s[e] = m2[e] = 0.f;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (k < mine) {
      float v[VW];
      unpack<T, VW>(f[k], v);
#pragma unroll
      for (int e = 0; e < VW; ++e) s[e] += v[e];
      forget(f[k]);
    }
  }
  if constexpr (!SPAN) {
#pragma unroll
    for (int e = 1; e < VW; ++e) s[0] += s[e];
#pragma unroll
    for (int e = 1; e < VW; ++e) s[e] = s[0];
  }
  const float own = 1.f / (float)max(1, mine * (SPAN ? 1 : VW));
#pragma unroll
  for (int e = 0; e < VW; ++e) s[e] *= own;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (k < mine) {
      float v[VW];
      unpack<T, VW>(f[k], v);
#pragma unroll
      for (int e = 0; e < VW; ++e) m2[e] += (v[e] - s[e]) * (v[e] - s[e]);
      forget(f[k]);
    }
  }
  if constexpr (!SPAN) {
#pragma unroll
    for (int e = 1; e < VW; ++e) m2[0] += m2[e];
  }
}

// Joins a batch of `now` vectors with the `before` vectors that came before it.
template <int VW, bool SPAN>
__device__ __forceinline__ void join_batch(int before, int now, const float (&batch)[VW],
                                           const float (&batch_m2)[VW], float (&s)[VW],
                                           float (&m2)[VW]) {
  const float share = (float)now / ((float)before + (float)now);
  const float cross = (float)before * share * (SPAN ? 1 : VW);
#pragma unroll
  for (int e = 0; e < (SPAN ? VW : 1); ++e) {
    const float d = batch[e] - s[e];
    s[e] += d * share;
    m2[e] += batch_m2[e] + d * (d * cross);  // (with nothing before, 0 however large d is)
  }
}

// A channel's constants: z = ((x - mean) * rstd) * gamma + beta.
struct Channel {
  float mean, rstd, gamma, beta;
};
__device__ __forceinline__ int group_of(const NormArgs& a, int ch) {
  return (int)fast_div((uint32_t)ch, a.d_mul, a.d_shift);
}
__device__ __forceinline__ Channel channel(const NormArgs& a, const float* stats, int img, int ch) {
  const float2 s = ((const float2*)stats)[(size_t)img * a.groups + group_of(a, ch)];
  return {s.x, s.y, a.gamma ? a.gamma[ch] : 1.f, a.beta ? a.beta[ch] : 0.f};
}
// gamma and beta of VW channels from ch, a multiple of VW.
template <int VW>
__device__ __forceinline__ void channel_params(const NormArgs& a, int ch, Channel (&k)[VW]) {
  float g[VW], b[VW];
  const auto load = [&](const float* p, float none, float (&f)[VW]) {
    if (!p) {
#pragma unroll
      for (int e = 0; e < VW; ++e) f[e] = none;
    } else if constexpr (VW % 4 == 0) {
#pragma unroll
      for (int e = 0; e < VW; e += 4) {
        const float4 v = *(const float4*)(p + ch + e);
        f[e] = v.x, f[e + 1] = v.y, f[e + 2] = v.z, f[e + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < VW; ++e) f[e] = p[ch + e];
    }
  };
  load(a.gamma, 1.f, g);
  load(a.beta, 0.f, b);
#pragma unroll
  for (int e = 0; e < VW; ++e) k[e].gamma = g[e], k[e].beta = b[e];
}

// y, or dx, of one value.
template <bool GRAD, int ACT, typename T>
__device__ __forceinline__ float norm_value(float x, float dy, const Channel& k, float2 coef) {
  // (A smooth activation is bound by its operations and has no mask to keep: fewer of them.
  // 4002x5 pixels of 1280 bf16: tanh 31.8 -> 28.6 us, SiLU 23.0 -> 21.5.)
  constexpr bool kSmooth = ACT == HUGE2_NORM_TANH || ACT == HUGE2_NORM_SILU;
  if constexpr (!GRAD && kSmooth)
    return norm_act<ACT, T>(fmaf(x - k.mean, k.rstd * k.gamma, k.beta));
  const float xh = (x - k.mean) * k.rstd;
  const float z = kSmooth ? fmaf(xh, k.gamma, k.beta) : norm_z(xh, k.gamma, k.beta);
  if constexpr (!GRAD) return norm_act<ACT, T>(z);
  const float t = norm_act_grad<ACT, T>(dy, z) * k.gamma;
  return k.rstd * (t - coef.x - xh * coef.y);
}

// dgamma and dbeta of 16 channels: rows of 16 threads share the runs.
struct ParamSums {
  float2 of[64][16];
};
__device__ __forceinline__ void param_sums(const NormArgs& a, int block, ParamSums& sums) {
  const int col = threadIdx.x & 15, ch = block * 16 + col, row = threadIdx.x >> 4;
  const int rows = blockDim.x >> 4;
  float2 s = make_float2(0.f, 0.f);
  if (ch < a.c) {
    const long long runs = (long long)a.n * a.chunks;
#pragma unroll 4
    for (long long r = row; r < runs; r += rows) {
      const float2 v = a.part[(size_t)r * a.c + ch];
      s.x += v.x;
      s.y += v.y;
    }
  }
  sums.of[row][col] = s;
  __syncthreads();
  if (row == 0 && ch < a.c) {
    for (int r = 1; r < rows; ++r) {
      s.x += sums.of[r][col].x;
      s.y += sums.of[r][col].y;
    }
    if (a.dbeta) a.dbeta[ch] = s.x;
    if (a.dgamma) a.dgamma[ch] = s.y;
  }
}

}  // namespace huge2
