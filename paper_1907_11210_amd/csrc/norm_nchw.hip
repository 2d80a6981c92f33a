// norm_nchw.hip -- group norm in NCHW where a workgroup holds a group of an image in
// registers: x, and dy for the gradient, are read once.
//
// Bound by the bytes, or for the small by latency: 16x16x256, 64 images, 32 groups,
// bf16, forward: 6.7 us for 17 MB.
#include "norm_device.hpp"

namespace huge2 {

namespace {

// dgamma and dbeta of a channel for each row of 2^direct_log2 lanes, from all images' x
// and dy.
template <typename T, int VW>
__device__ __forceinline__ void direct_params(const NormArgs& a, int block) {
  constexpr int kDeep = 4;
  const int lanes = 1 << a.direct_log2, lane = threadIdx.x & (lanes - 1);
  const int mine = block * (blockDim.x >> a.direct_log2) + (threadIdx.x >> a.direct_log2);
  const int ch = min(mine, a.c - 1);  // (rows behind the last: of that, and not written)
  const int vecs = a.hw / VW, all = a.n * vecs;
  const float gamma = a.gamma ? a.gamma[ch] : 1.f, beta = a.beta ? a.beta[ch] : 0.f;
  const float2* stats = (const float2*)a.stats + group_of(a, ch);
  float s1 = 0.f, s2 = 0.f;
  by_act(a.act, [&](auto act) {
    for (int i = lane; i < all; i += lanes * kDeep) {
      Pack<T, VW> f[kDeep], g[kDeep];
      float2 st[kDeep];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        const int p = min(i + j * lanes, all - 1);
        const int img = (int)fast_div((uint32_t)p, a.px_mul, a.px_shift);
        const size_t at = ((size_t)img * a.c + ch) * a.hw + (size_t)(p - img * vecs) * VW;
        f[j] = load_pack<T, VW>((const T*)a.x + at);
        g[j] = load_pack<T, VW>((const T*)a.dy + at);
        st[j] = stats[(size_t)img * a.groups];
      }
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        if (i + j * lanes < all) {
          float v[VW], w[VW];
          unpack<T, VW>(f[j], v);
          unpack<T, VW>(g[j], w);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            const float xh = (v[e] - st[j].x) * st[j].y;
            const float dz = norm_act_grad<act.value, T>(w[e], norm_z(xh, gamma, beta));
            s1 += dz;
            s2 += dz * xh;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  });
  for (int m = lanes >> 1; m; m >>= 1) {
    s1 += __shfl_xor(s1, m);
    s2 += __shfl_xor(s2, m);
  }
  if (lane == 0 && mine < a.c) {
    if (a.dbeta) a.dbeta[ch] = s1;
    if (a.dgamma) a.dgamma[ch] = s2;
  }
}

}  // namespace

// NCHW: a slab is a group of an image, d planes one behind the other.  Rows of
// lanes lie side by side on a plane; a thread has every `lanes`-th vector of every
// `planes`-th plane, `along` vectors of a plane, R in all.
template <typename T, int VW, int R, bool GRAD, bool DIRECT>
__global__ __launch_bounds__(1024) void norm_slab_nchw_kernel(NormArgs a) {
  __shared__ float lds[16];
  if constexpr (DIRECT) {  // (a kernel of its own: these take more registers)
    if ((int)blockIdx.x >= a.slabs) {
      direct_params<T, VW>(a, blockIdx.x - a.slabs);
      return;
    }
  }
  const int slab = xcd_remap(blockIdx.x, a.slabs);
  const int img = slab / a.groups, c0 = slab % a.groups * a.d;
  const int lanes = 1 << a.lanes_log2, planes = blockDim.x >> a.lanes_log2;
  const int lane = threadIdx.x & (lanes - 1), plane = threadIdx.x >> a.lanes_log2;
  const size_t at = ((size_t)img * a.c + c0) * a.hw;
  const T* x = (const T*)a.x + at;
  const T* dy = (const T*)a.dy + at;
  const int vecs = a.hw / VW;
  Pack<T, VW> f[R], g[R];
  int place[R];  // element of the slab, negative where there is none
  {
    int pl = plane, v = lane, j = 0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      place[k] = pl < a.d && v < vecs ? pl * a.hw + v * VW : -1;
      v += lanes;
      if (++j == a.along) j = 0, v = lane, pl += planes;
    }
  }
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (place[k] < 0) continue;
    f[k] = load_pack<T, VW>(x + place[k]);
    if constexpr (GRAD) g[k] = load_pack<T, VW>(dy + place[k]);
  }
  const float total = (float)a.d * (float)a.hw;
  float2 stats, coef = make_float2(0.f, 0.f);
  if constexpr (!GRAD) {
    float s = 0.f, sq = 0.f;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (place[k] < 0) continue;
      float v[VW];
      unpack<T, VW>(f[k], v);
#pragma unroll
      for (int e = 0; e < VW; ++e) s += v[e];
      forget(f[k]);
    }
    const float mean = block_sum(s, lds) / total;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (place[k] < 0) continue;
      float v[VW];
      unpack<T, VW>(f[k], v);
#pragma unroll
      for (int e = 0; e < VW; ++e) sq += (v[e] - mean) * (v[e] - mean);
      forget(f[k]);
    }
    const float var = block_sum(sq, lds) / total;
    stats = make_float2(mean, 1.f / sqrtf(var + a.eps));
    if (threadIdx.x == 0) ((float2*)a.stats_out)[(size_t)img * a.groups + c0 / a.d] = stats;
  } else {
    stats = ((const float2*)a.stats)[(size_t)img * a.groups + c0 / a.d];
    float g1 = 0.f, g2 = 0.f, s1 = 0.f, s2 = 0.f;
    by_act(a.act, [&](auto act) {
      int pl = plane, j = 0;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int ch = c0 + min(pl, a.d - 1);
        const float gamma = a.gamma ? a.gamma[ch] : 1.f;
        if (place[k] >= 0) {
          const float beta = a.beta ? a.beta[ch] : 0.f;
          float v[VW], w[VW];
          unpack<T, VW>(f[k], v);
          unpack<T, VW>(g[k], w);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            const float xh = (v[e] - stats.x) * stats.y;
            const float dz = norm_act_grad<act.value, T>(w[e], norm_z(xh, gamma, beta));
            s1 += dz;
            s2 += dz * xh;
          }
        }
        __builtin_amdgcn_sched_barrier(0);  // vector by vector: all at once would spill
        if (++j == a.along) {  // the plane is done: its sums over the row of lanes
          for (int m = lanes >> 1; m; m >>= 1) {
            s1 += __shfl_xor(s1, m);
            s2 += __shfl_xor(s2, m);
          }
          if (lane == 0 && pl < a.d) {
            if (a.n > 1) {
              if (!a.direct) a.part[(size_t)img * a.c + ch] = make_float2(s1, s2);
            } else {  // nothing to add up
              if (a.dbeta) a.dbeta[ch] = s1;
              if (a.dgamma) a.dgamma[ch] = s2;
            }
            g1 += gamma * s1;
            g2 += gamma * s2;
          }
          s1 = s2 = 0.f;
          j = 0;
          pl += planes;
        }
      }
    });
#pragma unroll
    for (int k = 0; k < R; ++k) {
      forget(f[k]);
      forget(g[k]);
    }
    coef.x = block_sum(g1, lds) / total;
    coef.y = block_sum(g2, lds) / total;
  }
  T* out = (T*)a.out + at;
  by_act(a.act, [&](auto act) {
    int pl = plane, j = 0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (place[k] >= 0) {
        const int ch = c0 + pl;
        const Channel c = {stats.x, stats.y, a.gamma ? a.gamma[ch] : 1.f,
                           a.beta ? a.beta[ch] : 0.f};
        float v[VW], w[VW];
        unpack<T, VW>(f[k], v);
        if constexpr (GRAD) unpack<T, VW>(g[k], w);
#pragma unroll
        for (int e = 0; e < VW; ++e) v[e] = norm_value<GRAD, act.value, T>(v[e], w[e], c, coef);
        store_pack<T, VW>(out + place[k], pack<T, VW>(v), a.stream);
      }
      if (GRAD) __builtin_amdgcn_sched_barrier(0);
      if (++j == a.along) j = 0, pl += planes;
    }
  });
}

namespace {

template <typename T, int VW, bool GRAD>
void launch_t(const NormArgs& a, hipStream_t stream) {
  constexpr int kMost = slab_most(VW, GRAD, false);
  const int direct = GRAD && (a.dgamma || a.dbeta) ? a.direct : 0;
  const auto launch = [&](auto slots) {
    constexpr int R = slots.value;
    const auto kernel = direct ? norm_slab_nchw_kernel<T, VW, R, GRAD, GRAD>
                               : norm_slab_nchw_kernel<T, VW, R, GRAD, false>;
    hipLaunchKernelGGL(kernel, dim3(a.slabs + direct), dim3(a.threads), 0, stream, a);
  };
  if (a.slots == 1)
    launch(std::integral_constant<int, 1>());
  else if (a.slots <= 4)
    launch(std::integral_constant<int, 4>());
  else
    launch(std::integral_constant<int, kMost>());
  // (its error is the last one, read by the caller)
  if (GRAD && a.n > 1 && !a.direct && (a.dgamma || a.dbeta)) (void)launch_norm_params(a, stream);
}

template <bool GRAD>
hipError_t launch_any(const NormArgs& a, int dtype, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16) {
    if (vec == 8)
      launch_t<uint16_t, 8, GRAD>(a, stream);
    else if (vec == 2)
      launch_t<uint16_t, 2, GRAD>(a, stream);
    else
      launch_t<uint16_t, 1, GRAD>(a, stream);
  } else if (vec == 4) {
    launch_t<uint32_t, 4, GRAD>(a, stream);
  } else {
    launch_t<uint32_t, 1, GRAD>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_nchw(const NormArgs& a, int dtype, int vec, hipStream_t stream) {
  return launch_any<false>(a, dtype, vec, stream);
}
hipError_t launch_norm_grad_nchw(const NormArgs& a, int dtype, int vec, hipStream_t stream) {
  return launch_any<true>(a, dtype, vec, stream);
}

}  // namespace huge2
