// norm.hip -- group norm with an activation and its gradients (huge2_train.h).
//
// The general form, two passes over x: sums per channel and run of pixels, a merge per
// group, and the pass that writes.  In NHWC it takes groups wider than a workgroup; in
// NCHW all that do not fit one or would occupy too few compute units, with the merge in
// the second pass.  Bound by the bytes of the two passes: 32 images of 300x42x123 bf16,
// forward, by 4 bytes 29 and 39 us; 8 of 64x40x40 in 4 groups, gradient, 4.6 and 5.6.
#include "norm_device.hpp"

namespace huge2 {

namespace {

// Where a workgroup of 256 works in NHWC: image, run of pixels, and its threads
// as rows of 2^lanes_log2 lanes side by side on a pixel's channels.
struct PlaceNhwc {
  int img, chunk, len, row, rows, ch;  // len: pixels of the run
  size_t at;                           // element of (img, the run's first pixel, ch)
};
template <int VW>
__device__ __forceinline__ PlaceNhwc place_nhwc(const NormArgs& a) {
  PlaceNhwc q;
  const int b = blockIdx.x, cb = b % a.cblocks, t = b / a.cblocks;
  q.chunk = t % a.chunks;
  q.img = t / a.chunks;
  const int p0 = q.chunk * a.chunk_len;
  q.len = min(a.chunk_len, a.hw - p0);
  q.rows = 256 >> a.lanes_log2;
  q.row = threadIdx.x >> a.lanes_log2;
  q.ch = ((cb << a.lanes_log2) + (threadIdx.x & ((1 << a.lanes_log2) - 1))) * VW;
  q.at = ((size_t)q.img * a.hw + p0) * a.c + q.ch;
  return q;
}

// The same in NCHW: rows of lanes side by side on the pixels of one plane's run.
struct PlaceNchw {
  size_t at;  // element of (img, ch, the run's first pixel)
  int img, ch, chunk, len, lane, lanes;
  bool in;
};
__device__ __forceinline__ PlaceNchw place_nchw(const NormArgs& a) {
  PlaceNchw q;
  const long long unit =
      (long long)blockIdx.x * (256 >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  q.in = unit < (long long)a.n * a.c * a.chunks;
  const long long plane = q.in ? unit / a.chunks : 0;  // img * c + ch
  q.chunk = q.in ? (int)(unit % a.chunks) : 0;
  q.img = (int)(plane / a.c);
  q.ch = (int)(plane % a.c);
  const int p0 = q.chunk * a.chunk_len;
  q.len = q.in ? min(a.chunk_len, a.hw - p0) : 0;
  q.at = (size_t)plane * a.hw + p0;
  q.lanes = 1 << a.lanes_log2;
  q.lane = threadIdx.x & (q.lanes - 1);
  return q;
}

// Vectors of a batch: their loads are in flight together.
template <int VW>
constexpr int kBatch = VW >= 4 ? 4 : 8;

// Joins what the lanes hold (a mean of `own` values and the squares around it), `count`
// values in all, in each of them; sum: over those lanes.
template <typename F>
__device__ __forceinline__ void join_lanes(float own, float count, float& mean, float& m2,
                                           F&& sum) {
  const float all = sum(own * mean) / fmaxf(count, 1.f);
  m2 = sum(m2 + own * ((mean - all) * (mean - all)));
  mean = all;
}

}  // namespace

// Sums of a run of pixels per channel.  Forward: the run's mean and its squares around
// that, from the means of a few vectors at a time, so that no value is measured from
// another one that may lie far from it.  Gradient: the sums of dz and of dz * xh.
template <typename T, int VW, bool GRAD>
__global__ __launch_bounds__(256) void norm_sums_nhwc_kernel(NormArgs a) {
  const PlaceNhwc q = place_nhwc<VW>(a);
  const bool in = q.ch < a.c;
  const T* x = (const T*)a.x + q.at;
  const T* dy = (const T*)a.dy + q.at;
  float s1[VW], s2[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) s1[e] = s2[e] = 0.f;
  // rows of one wave, then the four waves
  __shared__ float2 lds[4][64 * VW];
  __shared__ float pixels[4];
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), wave = threadIdx.x >> 6;
  if constexpr (GRAD) {
    if (in) {
      Channel k[VW];
#pragma unroll
      for (int e = 0; e < VW; ++e) k[e] = channel(a, a.stats, q.img, q.ch + e);
      by_act(a.act, [&](auto act) {
#pragma unroll 4
        for (int p = q.row; p < q.len; p += q.rows) {
          float f[VW], g[VW];
          unpack<T, VW>(load_pack<T, VW>(x + (size_t)p * a.c), f);
          unpack<T, VW>(load_pack<T, VW>(dy + (size_t)p * a.c), g);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            const float xh = (f[e] - k[e].mean) * k[e].rstd;
            const float dz = norm_act_grad<act.value, T>(g[e], norm_z(xh, k[e].gamma, k[e].beta));
            s1[e] += dz;
            s2[e] += dz * xh;
          }
        }
      });
    }
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      s1[e] = lanes_sum(s1[e], lanes);
      s2[e] = lanes_sum(s2[e], lanes);
    }
  } else {
    const int mine = (q.len - q.row + q.rows - 1) >> (8 - a.lanes_log2);
    for (int i = 0; in && i < mine; i += kBatch<VW>) {
      Pack<T, VW> f[kBatch<VW>];
#pragma unroll
      for (int k = 0; k < kBatch<VW>; ++k)
        if (i + k < mine)
          f[k] = load_pack<T, VW>(x + (size_t)(q.row + (i + k) * q.rows) * a.c);
      float mean[VW], m2[VW];
      own_stats<T, VW, kBatch<VW>, true>(f, min(kBatch<VW>, mine - i), mean, m2);
      join_batch<VW, true>(i, min(kBatch<VW>, mine - i), mean, m2, s1, s2);
    }
    const float count = lanes_sum((float)mine, lanes);
#pragma unroll
    for (int e = 0; e < VW; ++e)
      join_lanes((float)mine, count, s1[e], s2[e], [&](float v) { return lanes_sum(v, lanes); });
    if ((threadIdx.x & 63) == 0) pixels[wave] = count;
  }
  if ((threadIdx.x & 63) < lanes) {
#pragma unroll
    for (int e = 0; e < VW; ++e) lds[wave][lane * VW + e] = make_float2(s1[e], s2[e]);
  }
  __syncthreads();
  if (threadIdx.x < lanes && in) {
    float2* part = a.part + ((size_t)q.img * a.chunks + q.chunk) * a.c + q.ch;
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      float2 s = make_float2(0.f, 0.f);
      if constexpr (GRAD) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          s.x += lds[w][lane * VW + e].x;
          s.y += lds[w][lane * VW + e].y;
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) s.x += pixels[w] * lds[w][lane * VW + e].x;
        s.x /= (float)q.len;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 v = lds[w][lane * VW + e];
          s.y += v.y + pixels[w] * ((v.x - s.x) * (v.x - s.x));
        }
      }
      part[e] = s;
    }
  }
}

template <typename T, int VW, bool GRAD>
__global__ __launch_bounds__(256) void norm_sums_nchw_kernel(NormArgs a) {
  const PlaceNchw q = place_nchw(a);
  if (!q.in) return;  // whole rows of lanes: the sums below stay in one
  const T* x = (const T*)a.x + q.at;
  const T* dy = (const T*)a.dy + q.at;
  const auto row_sum = [&](float v) {
    for (int m = q.lanes >> 1; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
  };
  const int vecs = q.len / VW, mine = (vecs - q.lane + q.lanes - 1) >> a.lanes_log2;
  const auto load = [&](const T* from, int i, Pack<T, VW>(&f)[kBatch<VW>]) {
#pragma unroll
    for (int k = 0; k < kBatch<VW>; ++k)
      if (i + k < mine) f[k] = load_pack<T, VW>(from + (q.lane + (i + k) * q.lanes) * VW);
  };
  float2 part;
  if constexpr (GRAD) {
    const Channel c = channel(a, a.stats, q.img, q.ch);
    float s1 = 0.f, s2 = 0.f;
    by_act(a.act, [&](auto act) {
      for (int i = 0; i < mine; i += kBatch<VW>) {
        Pack<T, VW> f[kBatch<VW>], g[kBatch<VW>];
        load(x, i, f);
        load(dy, i, g);
#pragma unroll
        for (int k = 0; k < kBatch<VW>; ++k) {
          if (i + k >= mine) break;
          float v[VW], w[VW];
          unpack<T, VW>(f[k], v);
          unpack<T, VW>(g[k], w);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            const float xh = (v[e] - c.mean) * c.rstd;
            const float dz = norm_act_grad<act.value, T>(w[e], norm_z(xh, c.gamma, c.beta));
            s1 += dz;
            s2 += dz * xh;
          }
        }
      }
    });
    part = make_float2(row_sum(s1), row_sum(s2));
  } else {
    float s[VW], m2[VW];  // (the first of each)
    s[0] = m2[0] = 0.f;
    for (int i = 0; i < mine; i += kBatch<VW>) {
      Pack<T, VW> f[kBatch<VW>];
      load(x, i, f);
      float mean[VW], batch_m2[VW];
      own_stats<T, VW, kBatch<VW>, false>(f, min(kBatch<VW>, mine - i), mean, batch_m2);
      join_batch<VW, false>(i, min(kBatch<VW>, mine - i), mean, batch_m2, s, m2);
    }
    join_lanes((float)(mine * VW), (float)q.len, s[0], m2[0], row_sum);
    part = make_float2(s[0], m2[0]);
  }
  if (q.lane == 0) a.part[((size_t)q.img * a.chunks + q.chunk) * a.c + q.ch] = part;
}

// Joins the runs.  A workgroup to an (image, group): its statistics, or the two
// means of its gradient; behind those, a workgroup to 16 channels: dgamma, dbeta.
template <bool GRAD>
__global__ __launch_bounds__(256) void norm_merge_kernel(NormArgs a) {
  __shared__ float lds[4];
  const long long ng = (long long)a.n * a.groups;
  if ((long long)blockIdx.x < ng) {
    const int img = (int)(blockIdx.x / a.groups), g = (int)(blockIdx.x % a.groups);
    const float2* part = a.part + (size_t)img * a.chunks * a.c + (size_t)g * a.d;
    const int entries = a.chunks * a.d;
    const float m = (float)a.d * (float)a.hw;
    if constexpr (GRAD) {
      float s1 = 0.f, s2 = 0.f;
      for (int e = threadIdx.x; e < entries; e += 256) {
        const int chunk = e / a.d, j = e - chunk * a.d;
        const float2 v = part[(size_t)chunk * a.c + j];
        const float gamma = a.gamma ? a.gamma[g * a.d + j] : 1.f;
        s1 += gamma * v.x;
        s2 += gamma * v.y;
      }
      s1 = block_sum(s1, lds);
      s2 = block_sum(s2, lds);
      if (threadIdx.x == 0) a.coef[blockIdx.x] = make_float2(s1 / m, s2 / m);
    } else {
      float s = 0.f;
      for (int e = threadIdx.x; e < entries; e += 256) {
        const int chunk = e / a.d, j = e - chunk * a.d;
        const int count = min(a.chunk_len, a.hw - chunk * a.chunk_len);
        s += part[(size_t)chunk * a.c + j].x * (float)count;
      }
      const float mean = block_sum(s, lds) / m;
      s = 0.f;
      for (int e = threadIdx.x; e < entries; e += 256) {
        const int chunk = e / a.d, j = e - chunk * a.d;
        const int count = min(a.chunk_len, a.hw - chunk * a.chunk_len);
        const float2 v = part[(size_t)chunk * a.c + j];
        s += v.y + (float)count * (v.x - mean) * (v.x - mean);
      }
      const float var = block_sum(s, lds) / m;
      if (threadIdx.x == 0)
        ((float2*)a.stats_out)[blockIdx.x] = make_float2(mean, 1.f / sqrtf(var + a.eps));
    }
    return;
  }
  if constexpr (GRAD) {
    __shared__ ParamSums sums;
    param_sums(a, (int)(blockIdx.x - ng), sums);
  }
}

__global__ __launch_bounds__(256) void norm_params_kernel(NormArgs a) {
  __shared__ ParamSums sums;
  param_sums(a, blockIdx.x, sums);
}

template <typename T, int VW, bool GRAD>
__global__ __launch_bounds__(256) void norm_apply_nhwc_kernel(NormArgs a) {
  const PlaceNhwc q = place_nhwc<VW>(a);
  if (q.ch >= a.c) return;
  const T* x = (const T*)a.x + q.at;
  const T* dy = (const T*)a.dy + q.at;
  T* out = (T*)a.out + q.at;
  Channel k[VW];
  float2 coef[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    k[e] = channel(a, GRAD ? a.stats : a.stats_out, q.img, q.ch + e);
    if (GRAD) coef[e] = a.coef[(size_t)q.img * a.groups + (q.ch + e) / a.d];
  }
  by_act(a.act, [&](auto act) {
    for (int p = q.row; p < q.len; p += q.rows) {
      float f[VW], g[VW];
      unpack<T, VW>(load_pack<T, VW>(x + (size_t)p * a.c), f);
      if constexpr (GRAD) unpack<T, VW>(load_pack<T, VW>(dy + (size_t)p * a.c), g);
#pragma unroll
      for (int e = 0; e < VW; ++e) f[e] = norm_value<GRAD, act.value, T>(f[e], g[e], k[e], coef[e]);
      store_pack<T, VW>(out + (size_t)p * a.c, pack<T, VW>(f), a.stream);
    }
  });
}

// A workgroup to some runs of a group's planes (a row of lanes each).  Where the
// group has few runs (JOIN, up to kJoined) it joins them itself: no launch between the two passes,
// and dgamma and dbeta come from workgroups behind the others.
constexpr int kJoined = 1024;  // four a thread
template <typename T, int VW, bool GRAD, bool JOIN>
__global__ __launch_bounds__(256) void norm_apply_nchw_kernel(NormArgs a, int parts) {
  __shared__ float lds[4];
  constexpr int kAhead = 4;
  const long long ng = (long long)a.n * a.groups;
  if (GRAD && JOIN && (long long)blockIdx.x >= ng * parts) {
    __shared__ ParamSums sums;
    param_sums(a, (int)(blockIdx.x - ng * parts), sums);
    return;
  }
  const long long ig = blockIdx.x / parts;
  const int img = (int)(ig / a.groups), c0 = (int)(ig % a.groups) * a.d;
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int unit = blockIdx.x % parts * (256 >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  const bool in = unit < a.d * a.chunks;
  const int ch = c0 + (in ? unit / a.chunks : 0), first = in ? unit % a.chunks * a.chunk_len : 0;
  const int end = in ? min(a.chunk_len, a.hw - first) : 0, step = lanes * VW;
  const size_t at = ((size_t)img * a.c + ch) * a.hw + first;
  const T* x = (const T*)a.x + at;
  const T* dy = (const T*)a.dy + at;
  T* out = (T*)a.out + at;
  Pack<T, VW> f[kAhead], g[kAhead];
  const auto load = [&](int p) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (p + j * step < end) {
        f[j] = load_pack<T, VW>(x + p + j * step);
        if constexpr (GRAD) g[j] = load_pack<T, VW>(dy + p + j * step);
      }
    }
  };
  int p = lane * VW;
  load(p);  // in flight meanwhile
  float2 stats, coef = make_float2(0.f, 0.f);
  if constexpr (JOIN) {
    const float2* part = a.part + (size_t)img * a.chunks * a.c + c0;
    const int entries = a.chunks * a.d;
    const float total = (float)a.d * (float)a.hw;
    float2 v[kJoined / 256];
    float weight[kJoined / 256], s1 = 0.f, s2 = 0.f;  // gamma, or the run's pixels
#pragma unroll
    for (int i = 0; i < kJoined / 256; ++i) {
      const int e = threadIdx.x + i * 256, chunk = e / a.d, j = e - chunk * a.d;
      const bool mine = e < entries;
      v[i] = mine ? part[(size_t)chunk * a.c + j] : make_float2(0.f, 0.f);
      if constexpr (GRAD)
        weight[i] = mine && a.gamma ? a.gamma[c0 + j] : 1.f;
      else
        weight[i] = mine ? (float)min(a.chunk_len, a.hw - chunk * a.chunk_len) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kJoined / 256; ++i) s1 += weight[i] * v[i].x;
    s1 = block_sum(s1, lds) / total;
    if constexpr (GRAD) {
#pragma unroll
      for (int i = 0; i < kJoined / 256; ++i) s2 += weight[i] * v[i].y;
      coef = make_float2(s1, block_sum(s2, lds) / total);
      stats = ((const float2*)a.stats)[ig];
    } else {  // the squares around the mean of all
#pragma unroll
      for (int i = 0; i < kJoined / 256; ++i)
        s2 += v[i].y + weight[i] * ((v[i].x - s1) * (v[i].x - s1));
      stats = make_float2(s1, 1.f / sqrtf(block_sum(s2, lds) / total + a.eps));
      if (threadIdx.x == 0 && blockIdx.x % parts == 0) ((float2*)a.stats_out)[ig] = stats;
    }
  } else {
    stats = ((const float2*)(GRAD ? a.stats : a.stats_out))[ig];
    if (GRAD) coef = a.coef[ig];
  }
  const Channel k = {stats.x, stats.y, a.gamma ? a.gamma[ch] : 1.f, a.beta ? a.beta[ch] : 0.f};
  by_act(a.act, [&](auto act) {
    for (;;) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (p + j * step < end) {
          float v[VW], w[VW];
          unpack<T, VW>(f[j], v);
          if constexpr (GRAD) unpack<T, VW>(g[j], w);
#pragma unroll
          for (int e = 0; e < VW; ++e) v[e] = norm_value<GRAD, act.value, T>(v[e], w[e], k, coef);
          store_pack<T, VW>(out + p + j * step, pack<T, VW>(v), a.stream);
        }
      }
      p += kAhead * step;
      if (p >= end) break;
      load(p);
    }
  });
}

namespace {

template <typename T, int VW, bool GRAD>
hipError_t launch_t(const NormArgs& a, int nhwc, hipStream_t stream) {
  const dim3 wg(256);
  const long long units = (long long)a.n * a.chunks * (nhwc ? a.cblocks : a.c);
  const unsigned grid =
      (unsigned)(nhwc ? units : (units + (256 >> a.lanes_log2) - 1) / (256 >> a.lanes_log2));
  const unsigned merge = (unsigned)((long long)a.n * a.groups +
                                    (GRAD && (a.dgamma || a.dbeta) ? (a.c + 15) / 16 : 0));
  if (nhwc) {
    hipLaunchKernelGGL((norm_sums_nhwc_kernel<T, VW, GRAD>), dim3(grid), wg, 0, stream, a);
    hipLaunchKernelGGL((norm_merge_kernel<GRAD>), dim3(merge), wg, 0, stream, a);
    hipLaunchKernelGGL((norm_apply_nhwc_kernel<T, VW, GRAD>), dim3(grid), wg, 0, stream, a);
    return hipGetLastError();
  }
  const int rows = 256 >> a.lanes_log2, parts = (a.d * a.chunks + rows - 1) / rows;
  const unsigned apply = (unsigned)a.n * a.groups * parts;
  hipLaunchKernelGGL((norm_sums_nchw_kernel<T, VW, GRAD>), dim3(grid), wg, 0, stream, a);
  if (a.d * a.chunks <= kJoined) {
    hipLaunchKernelGGL((norm_apply_nchw_kernel<T, VW, GRAD, true>),
                       dim3(apply + merge - a.n * a.groups), wg, 0, stream, a, parts);
  } else {
    hipLaunchKernelGGL((norm_merge_kernel<GRAD>), dim3(merge), wg, 0, stream, a);
    hipLaunchKernelGGL((norm_apply_nchw_kernel<T, VW, GRAD, false>), dim3(apply), wg, 0, stream, a,
                       parts);
  }
  return hipGetLastError();
}

template <bool GRAD>
hipError_t launch_any(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    return vec == 8   ? launch_t<uint16_t, 8, GRAD>(a, nhwc, stream)
           : vec == 2 ? launch_t<uint16_t, 2, GRAD>(a, nhwc, stream)
                      : launch_t<uint16_t, 1, GRAD>(a, nhwc, stream);
  return vec == 4 ? launch_t<uint32_t, 4, GRAD>(a, nhwc, stream)
                  : launch_t<uint32_t, 1, GRAD>(a, nhwc, stream);
}

}  // namespace

hipError_t launch_norm_params(const NormArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(norm_params_kernel, dim3((a.c + 15) / 16), dim3(256), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_norm(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream) {
  return launch_any<false>(a, dtype, nhwc, vec, stream);
}
hipError_t launch_norm_grad(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream) {
  return launch_any<true>(a, dtype, nhwc, vec, stream);
}

}  // namespace huge2
