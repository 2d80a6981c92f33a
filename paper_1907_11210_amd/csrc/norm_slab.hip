// norm_slab.hip -- group norm where a workgroup holds all pixels of some groups of
// an image (a slab) in registers: x, and dy for the gradient, are read once.
#include "norm_device.hpp"

namespace huge2 {

// NHWC: a slab is slab_c channels (whole groups, whole vectors) of an image.  Rows
// of 2^lanes_log2 lanes lie side by side on a pixel's channels; a thread has one
// vector of channels at every `rows`-th pixel, R of them.
//
// Statistics: a thread's own mean and squares around it, joined per group by as
// many lanes as the workgroup has for a group; in LDS, an entry a thread, or one
// a channel where a vector spans groups (a.span).
template <typename T, int VW, int R, bool SPAN>
__global__ __launch_bounds__(1024) void norm_slab_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  const int slab = xcd_remap(blockIdx.x, gridDim.x);
  const int img = slab / a.cblocks, c0 = slab % a.cblocks * a.slab_c;
  const int channels = min(a.slab_c, a.c - c0), groups = channels / a.d;
  const int lanes = 1 << a.lanes_log2, rows = blockDim.x >> a.lanes_log2;
  const int lane = threadIdx.x & (lanes - 1), row = threadIdx.x >> a.lanes_log2;
  const bool in = lane * VW < channels;
  const size_t at = (size_t)img * a.hw * a.c + c0 + lane * VW;
  const T* x = (const T*)a.x + at;
  Pack<T, VW> f[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int p = row + k * rows;
    if (in && p < a.hw) f[k] = load_pack<T, VW>(x + (size_t)p * a.c);
  }
  const int mine = in ? (a.hw - row + rows - 1) / rows : 0;  // pixels of this thread
  float s[VW], m2[VW];
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
  constexpr int kPer = SPAN ? VW : 1;  // entries a thread
  const int width = lanes * kPer, dl = SPAN ? a.d : a.d / VW;
  if constexpr (!SPAN) {
#pragma unroll
    for (int e = 1; e < VW; ++e) s[0] += s[e];
#pragma unroll
    for (int e = 1; e < VW; ++e) s[e] = s[0];
  }
  const float own = 1.f / (float)max(1, mine * (VW / kPer));
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
  if constexpr (SPAN) {
#pragma unroll
    for (int e = 0; e < VW; ++e) lds[row * width + lane * VW + e] = make_float2(s[e], m2[e]);
  } else {
#pragma unroll
    for (int e = 1; e < VW; ++e) m2[0] += m2[e];
    lds[row * width + lane] = make_float2(s[0], m2[0]);
  }
  __syncthreads();
  float2* const result = lds + rows * width;
  const int gl = 1 << a.join_log2;  // lanes that join a group
  for (int g = threadIdx.x >> a.join_log2; g < groups; g += blockDim.x >> a.join_log2) {
    const int terms = min(rows, a.hw) * dl, l = threadIdx.x & (gl - 1);
    const float2* e = lds + g * dl;
    float sum = 0.f;
    for (int t = l; t < terms; t += gl) {
      const int r = (int)fast_div(t, a.dl_mul, a.dl_shift), j = t - r * dl;
      sum += (float)((a.hw - r + rows - 1) / rows) * e[r * width + j].x;
    }
    for (int m = gl >> 1; m; m >>= 1) sum += __shfl_xor(sum, m);
    const float each = (float)(VW / kPer), total = (float)a.d * (float)a.hw;
    const float mean = sum * each / total;
    float sq = 0.f;
    for (int t = l; t < terms; t += gl) {
      const int r = (int)fast_div(t, a.dl_mul, a.dl_shift), j = t - r * dl;
      const float2 v = e[r * width + j];
      const float count = (float)((a.hw - r + rows - 1) / rows) * each;
      sq += v.y + count * (v.x - mean) * (v.x - mean);
    }
    for (int m = gl >> 1; m; m >>= 1) sq += __shfl_xor(sq, m);
    if (l == 0) {
      const float2 st = make_float2(mean, 1.f / sqrtf(sq / total + a.eps));
      result[g] = st;
      ((float2*)a.stats_out)[(size_t)img * a.groups + c0 / a.d + g] = st;
    }
  }
  __syncthreads();
  if (!in) return;
  T* out = (T*)a.out + at;
  Channel k[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    const int ch = lane * VW + e;
    const float2 st = result[(SPAN ? ch : lane * VW) / a.d];
    k[e] = {st.x, st.y, a.gamma ? a.gamma[c0 + ch] : 1.f, a.beta ? a.beta[c0 + ch] : 0.f};
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < mine) {
      float v[VW];
      unpack<T, VW>(f[i], v);
#pragma unroll
      for (int e = 0; e < VW; ++e)
        v[e] = norm_value<false>(v[e], 0.f, k[e], make_float2(0.f, 0.f), a.act);
      store_pack<T, VW>(out + (size_t)(row + i * rows) * a.c, pack<T, VW>(v));
    }
  }
}

// The gradient on the same slabs: a thread's sums of dz and dz * xh per channel,
// joined over the rows through LDS (consecutive lanes on consecutive channels),
// then per group.
template <typename T, int VW, int R, bool SPAN>
__global__ __launch_bounds__(1024) void norm_slab_grad_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  const int slab = xcd_remap(blockIdx.x, gridDim.x);
  const int img = slab / a.cblocks, c0 = slab % a.cblocks * a.slab_c;
  const int channels = min(a.slab_c, a.c - c0), groups = channels / a.d;
  const int lanes = 1 << a.lanes_log2, rows = blockDim.x >> a.lanes_log2;
  const int lane = threadIdx.x & (lanes - 1), row = threadIdx.x >> a.lanes_log2;
  const bool in = lane * VW < channels;
  const size_t at = (size_t)img * a.hw * a.c + c0 + lane * VW;
  const T* x = (const T*)a.x + at;
  const T* dy = (const T*)a.dy + at;
  Pack<T, VW> f[R], g[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int p = row + k * rows;
    if (in && p < a.hw) {
      f[k] = load_pack<T, VW>(x + (size_t)p * a.c);
      g[k] = load_pack<T, VW>(dy + (size_t)p * a.c);
    }
  }
  const int mine = in ? (a.hw - row + rows - 1) / rows : 0;
  Channel k[VW];
  float s1[VW], s2[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    s1[e] = s2[e] = 0.f;
    k[e] = channel(a, a.stats, img, min(c0 + lane * VW + e, a.c - 1));
    if (!SPAN && e) k[e].mean = k[0].mean, k[e].rstd = k[0].rstd;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < mine) {
      float v[VW], w[VW];
      unpack<T, VW>(f[i], v);
      unpack<T, VW>(g[i], w);
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        const float xh = (v[e] - k[e].mean) * k[e].rstd;
        const float dz = norm_act_grad(w[e], norm_z(xh, k[e].gamma, k[e].beta), a.act);
        s1[e] += dz;
        s2[e] += dz * xh;
      }
      forget(f[i]);
      forget(g[i]);
    }
  }
  // rows in LDS: a wave's two halves first where both have the same channels
  const int width = lanes * VW, width_log2 = a.lanes_log2 + (VW == 8 ? 3 : VW == 4 ? 2 : VW == 2 ? 1 : 0);
  int held = rows, slot = row;
  if (lanes <= 32) {
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      s1[e] += __shfl_xor(s1[e], 32);
      s2[e] += __shfl_xor(s2[e], 32);
    }
    const int half = 32 >> a.lanes_log2;  // rows of half a wave
    held = rows >> 1;
    slot = (threadIdx.x >> 6) * half + (row & (half - 1));
  }
  if (lanes > 32 || (threadIdx.x & 32) == 0) {
#pragma unroll
    for (int e = 0; e < VW; ++e) lds[slot * width + lane * VW + e] = make_float2(s1[e], s2[e]);
  }
  __syncthreads();
  float2* const sums = lds + held * width;  // [segments][width]
  int segments;
  if (width >= (int)blockDim.x) {
    segments = 1;
    for (int ch = threadIdx.x; ch < width; ch += blockDim.x) {
      float2 t = lds[ch];
      for (int r = 1; r < held; ++r) {
        t.x += lds[r * width + ch].x;
        t.y += lds[r * width + ch].y;
      }
      sums[ch] = t;
    }
  } else {
    const int ch = threadIdx.x & (width - 1), parts = blockDim.x >> width_log2;
    float2 t = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int r = threadIdx.x >> width_log2; r < held; r += parts) {
      t.x += lds[r * width + ch].x;
      t.y += lds[r * width + ch].y;
    }
    for (int m = 32; m >= width; m >>= 1) {
      t.x += __shfl_xor(t.x, m);
      t.y += __shfl_xor(t.y, m);
    }
    segments = width >= 64 ? parts : (int)(blockDim.x >> 6);
    const int seg = width >= 64 ? (int)(threadIdx.x >> width_log2) : (int)(threadIdx.x >> 6);
    if (width >= 64 || (int)(threadIdx.x & 63) < width) sums[seg * width + ch] = t;
  }
  __syncthreads();
  for (int ch = threadIdx.x; ch < channels; ch += blockDim.x) {
    float2 t = sums[ch];
    for (int q = 1; q < segments; ++q) {
      t.x += sums[q * width + ch].x;
      t.y += sums[q * width + ch].y;
    }
    a.part[(size_t)img * a.c + c0 + ch] = t;
    const float gamma = a.gamma ? a.gamma[c0 + ch] : 1.f;
    sums[ch] = make_float2(gamma * t.x, gamma * t.y);  // read by this thread alone so far
  }
  __syncthreads();
  float2* const result = lds;  // the rows are done with
  const int gl = 1 << a.join_log2;
  for (int q = threadIdx.x >> a.join_log2; q < groups; q += blockDim.x >> a.join_log2) {
    const int l = threadIdx.x & (gl - 1);
    float2 t = make_float2(0.f, 0.f);
    for (int j = l; j < a.d; j += gl) {
      t.x += sums[q * a.d + j].x;
      t.y += sums[q * a.d + j].y;
    }
    for (int m = gl >> 1; m; m >>= 1) {
      t.x += __shfl_xor(t.x, m);
      t.y += __shfl_xor(t.y, m);
    }
    const float total = (float)a.d * (float)a.hw;
    if (l == 0) result[q] = make_float2(t.x / total, t.y / total);
  }
  __syncthreads();
  if (!in) return;
  T* out = (T*)a.out + at;
  float2 coef[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) coef[e] = result[(lane * VW + (SPAN ? e : 0)) / a.d];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < mine) {
      float v[VW], w[VW];
      unpack<T, VW>(f[i], v);
      unpack<T, VW>(g[i], w);
#pragma unroll
      for (int e = 0; e < VW; ++e) v[e] = norm_value<true>(v[e], w[e], k[e], coef[e], a.act);
      store_pack<T, VW>(out + (size_t)(row + i * rows) * a.c, pack<T, VW>(v));
    }
  }
}

// NCHW: a slab is a group of an image, d planes one behind the other.  Rows of
// lanes lie side by side on a plane; a thread has every `lanes`-th vector of every
// `planes`-th plane, `along` vectors of a plane, R in all.
template <typename T, int VW, int R, bool GRAD>
__global__ __launch_bounds__(1024) void norm_slab_nchw_kernel(NormArgs a) {
  __shared__ float lds[16];
  const int slab = xcd_remap(blockIdx.x, gridDim.x);
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
          const float dz = norm_act_grad(w[e], norm_z(xh, gamma, beta), a.act);
          s1 += dz;
          s2 += dz * xh;
        }
        forget(f[k]);
        forget(g[k]);
      }
      if (++j == a.along) {  // the plane is done: its sums over the row of lanes
        for (int m = lanes >> 1; m; m >>= 1) {
          s1 += __shfl_xor(s1, m);
          s2 += __shfl_xor(s2, m);
        }
        if (lane == 0 && pl < a.d) {
          a.part[(size_t)img * a.c + ch] = make_float2(s1, s2);
          g1 += gamma * s1;
          g2 += gamma * s2;
        }
        s1 = s2 = 0.f;
        j = 0;
        pl += planes;
      }
    }
    coef.x = block_sum(g1, lds) / total;
    coef.y = block_sum(g2, lds) / total;
  }
  T* out = (T*)a.out + at;
  int pl = plane, j = 0;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (place[k] >= 0) {
      const int ch = c0 + pl;
      const Channel c = {stats.x, stats.y, a.gamma ? a.gamma[ch] : 1.f, a.beta ? a.beta[ch] : 0.f};
      float v[VW], w[VW];
      unpack<T, VW>(f[k], v);
      if constexpr (GRAD) unpack<T, VW>(g[k], w);
#pragma unroll
      for (int e = 0; e < VW; ++e) v[e] = norm_value<GRAD>(v[e], w[e], c, coef, a.act);
      store_pack<T, VW>(out + place[k], pack<T, VW>(v));
    }
    if (++j == a.along) j = 0, pl += planes;
  }
}

namespace {

template <typename T, int VW, int R, bool GRAD, bool SPAN>
void launch_r(const NormArgs& a, int nhwc, hipStream_t stream) {
  const dim3 grid(nhwc ? (unsigned)a.n * a.cblocks : (unsigned)a.n * a.groups), wg(a.threads);
  if (nhwc) {
    if constexpr (GRAD)
      hipLaunchKernelGGL((norm_slab_grad_nhwc_kernel<T, VW, R, SPAN>), grid, wg, a.lds_bytes,
                         stream, a);
    else
      hipLaunchKernelGGL((norm_slab_nhwc_kernel<T, VW, R, SPAN>), grid, wg, a.lds_bytes, stream, a);
  } else if constexpr (!SPAN) {
    hipLaunchKernelGGL((norm_slab_nchw_kernel<T, VW, R, GRAD>), grid, wg, 0, stream, a);
  }
}

template <typename T, int VW, bool GRAD, bool SPAN>
hipError_t launch_t(const NormArgs& a, int nhwc, hipStream_t stream) {
  if (a.slots == 1)
    launch_r<T, VW, 1, GRAD, SPAN>(a, nhwc, stream);
  else if (a.slots <= 4)
    launch_r<T, VW, 4, GRAD, SPAN>(a, nhwc, stream);
  else if constexpr (slab_most(VW, GRAD, SPAN) > 4)
    launch_r<T, VW, slab_most(VW, GRAD, SPAN), GRAD, SPAN>(a, nhwc, stream);
  return hipGetLastError();
}

template <typename T, int VW, bool GRAD>
hipError_t launch_v(const NormArgs& a, int nhwc, hipStream_t stream) {
  if constexpr (VW > 1)
    if (a.span) return launch_t<T, VW, GRAD, true>(a, nhwc, stream);
  return launch_t<T, VW, GRAD, false>(a, nhwc, stream);
}

template <bool GRAD>
hipError_t launch_any(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    return vec == 8   ? launch_v<uint16_t, 8, GRAD>(a, nhwc, stream)
           : vec == 2 ? launch_v<uint16_t, 2, GRAD>(a, nhwc, stream)
                      : launch_v<uint16_t, 1, GRAD>(a, nhwc, stream);
  return vec == 4 ? launch_v<uint32_t, 4, GRAD>(a, nhwc, stream)
                  : launch_v<uint32_t, 1, GRAD>(a, nhwc, stream);
}

}  // namespace

hipError_t launch_norm_slab(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream) {
  return launch_any<false>(a, dtype, nhwc, vec, stream);
}
hipError_t launch_norm_slab_grad(const NormArgs& a, int dtype, int nhwc, int vec,
                                 hipStream_t stream) {
  const hipError_t e = launch_any<true>(a, dtype, nhwc, vec, stream);
  if (e != hipSuccess || !(a.dgamma || a.dbeta)) return e;
  return launch_norm_params(a, stream);
}

}  // namespace huge2
