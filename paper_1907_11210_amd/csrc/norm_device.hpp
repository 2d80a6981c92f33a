// norm_device.hpp -- device helpers of the group norm kernels.
#pragma once

#include <cmath>

#include "train.hpp"
#include "train_device.hpp"

namespace huge2 {

// z of a normalised value.  Rounded after the product, here and in the gradient,
// so that both see the same sign (and the same as a framework without fused
// multiply-adds).
__device__ __forceinline__ float norm_z(float xh, float gamma, float beta) {
#pragma clang fp contract(off)
  return xh * gamma + beta;
}

// huge2_norm_activation; act is uniform over the launch.
__device__ __forceinline__ float norm_act(float z, int act) {
  switch (act) {
    case 1: return z < 0.f ? 0.f : z;
    case 2: return tanhf(z);
    case 3: return z / (1.f + expf(-z));
  }
  return z;
}
// dy * activation'(z)
__device__ __forceinline__ float norm_act_grad(float dy, float z, int act) {
  switch (act) {
    case 1: return z > 0.f ? dy : 0.f;
    case 2: {
      const float th = tanhf(z);
      return dy * (1.f - th * th);
    }
    case 3: {
      const float s = 1.f / (1.f + expf(-z));
      return dy * (s * (1.f + z * (1.f - s)));
    }
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

// A channel's constants: z = ((x - mean) * rstd) * gamma + beta.
struct Channel {
  float mean, rstd, gamma, beta;
};
__device__ __forceinline__ Channel channel(const NormArgs& a, const float* stats, int img, int ch) {
  const float2 s = ((const float2*)stats)[(size_t)img * a.groups + ch / a.d];
  return {s.x, s.y, a.gamma ? a.gamma[ch] : 1.f, a.beta ? a.beta[ch] : 0.f};
}

// y, or dx, of one value.
template <bool GRAD>
__device__ __forceinline__ float norm_value(float x, float dy, const Channel& k, float2 coef,
                                            int act) {
  const float xh = (x - k.mean) * k.rstd, z = norm_z(xh, k.gamma, k.beta);
  if constexpr (!GRAD) return norm_act(z, act);
  const float t = norm_act_grad(dy, z, act) * k.gamma;
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
