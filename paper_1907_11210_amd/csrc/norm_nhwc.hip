// norm_nhwc.hip -- group norm in NHWC by slabs: some whole groups of channels of an
// image, all of its pixels or a run of them, to a workgroup.
//
// Where a slab of all pixels fits the registers of a workgroup, and the slabs are enough,
// x (and dy for the gradient) are read once.  Else a first pass leaves each run's sums
// and a second one joins them and reads x again: 1.5 times the bytes for the forward, 5/3
// for the gradient, of which what the Infinity Cache still holds costs less.
//
// Bound by those bytes.  32x32x128, 64 images, bf16, gradient in one pass: 15.8 us for
// 50 MB and 3.8 for the launch that adds up dgamma and dbeta.  64x64x2048, 8 images,
// bf16, forward in two: 26.8 us for the first read of 134 MB and 42.2 for the second
// and the result.
#include "norm_device.hpp"

namespace huge2 {

namespace {

// Rows of 2^lanes_log2 lanes lie side by side on a pixel's channels; a thread has one
// vector of channels at every `rows`-th pixel of the run.
struct Slab {
  int img, chunk, p0, len;    // the run of pixels
  int c0, channels, groups;   // of the slab
  int lane, row, rows, ch;    // ch: the thread's first channel in the slab
  bool in;
  size_t at;                  // element of (img, p0, c0 + ch)
};
template <int VW>
__device__ __forceinline__ Slab slab_of(const NormArgs& a) {
  Slab q;
  int s = xcd_remap(blockIdx.x, a.slabs);
  q.c0 = s % a.cblocks * a.slab_c;
  s /= a.cblocks;
  q.chunk = s % a.chunks;
  q.img = s / a.chunks;
  q.p0 = q.chunk * a.chunk_len;
  q.len = min(a.chunk_len, a.hw - q.p0);
  q.channels = min(a.slab_c, a.c - q.c0);
  q.groups = q.channels / a.d;
  q.rows = 1 << a.rows_log2;
  q.lane = threadIdx.x & ((1 << a.lanes_log2) - 1);
  q.row = threadIdx.x >> a.lanes_log2;
  q.ch = q.lane * VW;
  q.in = q.ch < q.channels;
  q.at = ((size_t)q.img * a.hw + q.p0) * a.c + q.c0 + q.ch;
  return q;
}
// Pixels of row r.
__device__ __forceinline__ int pixels_of(const NormArgs& a, const Slab& q, int r) {
  return (q.len - r + q.rows - 1) >> a.rows_log2;
}

// Joins the threads' entries: f(group of the slab, mean, squares around it) by one
// lane of those that join the group.
template <int VW, bool SPAN, typename F>
__device__ __forceinline__ void join_stats(const NormArgs& a, const Slab& q, float2* lds,
                                           const float (&s)[VW], const float (&m2)[VW], F&& f) {
  constexpr int kPer = SPAN ? VW : 1;  // entries a thread
  const int width = kPer << a.lanes_log2, dl = SPAN ? a.d : a.d / VW;
#pragma unroll
  for (int e = 0; e < kPer; ++e) lds[q.row * width + q.lane * kPer + e] = make_float2(s[e], m2[e]);
  __syncthreads();
  const int gl = 1 << a.join_log2, l = threadIdx.x & (gl - 1);
  const int terms = min(q.rows, q.len) * dl;
  constexpr float kEach = (float)(VW / kPer);
  for (int g = threadIdx.x >> a.join_log2; g < q.groups; g += blockDim.x >> a.join_log2) {
    const float2* e = lds + g * dl;
    float sum = 0.f, sq = 0.f;
    for (int t = l; t < terms; t += gl) {
      const int r = (int)fast_div(t, a.dl_mul, a.dl_shift), j = t - r * dl;
      sum += (float)pixels_of(a, q, r) * e[r * width + j].x;
    }
    for (int m = gl >> 1; m; m >>= 1) sum += __shfl_xor(sum, m);
    const float mean = sum * kEach / ((float)a.d * (float)q.len);
    for (int t = l; t < terms; t += gl) {
      const int r = (int)fast_div(t, a.dl_mul, a.dl_shift), j = t - r * dl;
      const float2 v = e[r * width + j];
      sq += v.y + (float)pixels_of(a, q, r) * kEach * (v.x - mean) * (v.x - mean);
    }
    for (int m = gl >> 1; m; m >>= 1) sq += __shfl_xor(sq, m);
    if (l == 0) f(g, mean, sq);
  }
}

// The channels' constants of a thread whose groups' (mean, rstd) are in LDS.
template <int VW, bool SPAN>
__device__ __forceinline__ void channels_of(const NormArgs& a, const Slab& q, const float2* result,
                                            Channel (&k)[VW]) {
  channel_params<VW>(a, q.c0 + q.ch, k);
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    const float2 st = result[group_of(a, q.ch + (SPAN ? e : 0))];
    k[e].mean = st.x, k[e].rstd = st.y;
  }
}

template <typename T, int VW, int R>
__device__ __forceinline__ void load_rows(const NormArgs& a, const Slab& q, const T* x, int first,
                                          int mine, Pack<T, VW> (&f)[R]) {
#pragma unroll
  for (int k = 0; k < R; ++k)
    if (first + k < mine) f[k] = load_pack<T, VW>(x + (size_t)(q.row + (first + k) * q.rows) * a.c);
}

template <int ACT, typename T, int VW, int R>
__device__ __forceinline__ void write_rows(const NormArgs& a, const Slab& q, T* out, int first,
                                           int mine, const Pack<T, VW> (&f)[R],
                                           const Channel (&k)[VW]) {
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (first + i < mine) {
      float v[VW];
      unpack<T, VW>(f[i], v);
#pragma unroll
      for (int e = 0; e < VW; ++e)
        v[e] = norm_value<false, ACT, T>(v[e], 0.f, k[e], make_float2(0.f, 0.f));
      store_pack<T, VW>(out + (size_t)(q.row + (first + i) * q.rows) * a.c, pack<T, VW>(v),
                        a.stream);
    }
  }
}

// A thread's sums of dz and dz * xh over some of its vectors.
template <int ACT, typename T, int VW, int R>
__device__ __forceinline__ void add_grad_sums(const NormArgs& a, int first, int mine,
                                              const Pack<T, VW> (&f)[R],
                                              const Pack<T, VW> (&g)[R],
                                              const Channel (&k)[VW], float (&s1)[VW],
                                              float (&s2)[VW]) {
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (first + i < mine) {
      float v[VW], w[VW];
      unpack<T, VW>(f[i], v);
      unpack<T, VW>(g[i], w);
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        const float xh = (v[e] - k[e].mean) * k[e].rstd;
        const float dz = norm_act_grad<ACT, T>(w[e], norm_z(xh, k[e].gamma, k[e].beta));
        s1[e] += dz;
        s2[e] += dz * xh;
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // row by row: all at once would spill
  }
}

// The same from the caller's statistics (lanes behind the last channel: of that).
template <int VW, bool SPAN>
__device__ __forceinline__ void grad_channels(const NormArgs& a, const Slab& q, Channel (&k)[VW]) {
  const int ch = min(q.c0 + q.ch, a.c - VW);
  channel_params<VW>(a, ch, k);
  const float2* stats = (const float2*)a.stats + (size_t)q.img * a.groups;
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    const float2 st = stats[group_of(a, ch + (SPAN ? e : 0))];
    k[e].mean = st.x, k[e].rstd = st.y;
  }
}

// The rows' sums added up through LDS with consecutive lanes on consecutive channels:
// behind a barrier, [segments][width] of them at `sums`.  Returns the segments.
template <int VW>
__device__ __forceinline__ int add_rows(const NormArgs& a, const Slab& q, float2* lds,
                                        float (&s1)[VW], float (&s2)[VW], float2*& sums) {
  const int lanes = 1 << a.lanes_log2, width = lanes * VW;
  const int width_log2 = a.lanes_log2 + (VW == 8 ? 3 : VW == 4 ? 2 : VW == 2 ? 1 : 0);
  // a wave's two halves first where both have the same channels
  int held = q.rows, slot = q.row;
  if (lanes <= 32) {
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      s1[e] += __shfl_xor(s1[e], 32);
      s2[e] += __shfl_xor(s2[e], 32);
    }
    const int half = 32 >> a.lanes_log2;  // rows of half a wave
    held = q.rows >> 1;
    slot = (threadIdx.x >> 6) * half + (q.row & (half - 1));
  }
  if (lanes > 32 || (threadIdx.x & 32) == 0) {
#pragma unroll
    for (int e = 0; e < VW; ++e) lds[slot * width + q.ch + e] = make_float2(s1[e], s2[e]);
  }
  __syncthreads();
  sums = lds + held * width;
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
  return segments;
}
__device__ __forceinline__ float2 add_segments(const float2* sums, int segments, int width,
                                               int ch) {
  float2 t = sums[ch];
  for (int p = 1; p < segments; ++p) {
    t.x += sums[p * width + ch].x;
    t.y += sums[p * width + ch].y;
  }
  return t;
}

// The slab's sums per channel, to part; then f(group, sum of gamma * dz, sum of
// gamma * dz * xh) by one lane of those that join the group.
template <int VW, typename F>
__device__ __forceinline__ void join_grad_sums(const NormArgs& a, const Slab& q, float2* lds,
                                               float (&s1)[VW], float (&s2)[VW], F&& f) {
  float2* sums;
  const int segments = add_rows<VW>(a, q, lds, s1, s2, sums), width = VW << a.lanes_log2;
  float2* part = a.part + ((size_t)q.img * a.chunks + q.chunk) * a.c + q.c0;
  for (int ch = threadIdx.x; ch < q.channels; ch += blockDim.x) {
    const float2 t = add_segments(sums, segments, width, ch);
    if (a.n * a.chunks == 1) {  // nothing to add up
      if (a.dbeta) a.dbeta[q.c0 + ch] = t.x;
      if (a.dgamma) a.dgamma[q.c0 + ch] = t.y;
    } else if (!a.direct) {
      part[ch] = t;
    }
    const float gamma = a.gamma ? a.gamma[q.c0 + ch] : 1.f;
    sums[ch] = make_float2(gamma * t.x, gamma * t.y);  // read by this thread alone so far
  }
  __syncthreads();
  const int gl = 1 << a.join_log2, l = threadIdx.x & (gl - 1);
  for (int g = threadIdx.x >> a.join_log2; g < q.groups; g += blockDim.x >> a.join_log2) {
    float2 t = make_float2(0.f, 0.f);
    for (int j = l; j < a.d; j += gl) {
      t.x += sums[g * a.d + j].x;
      t.y += sums[g * a.d + j].y;
    }
    for (int m = gl >> 1; m; m >>= 1) {
      t.x += __shfl_xor(t.x, m);
      t.y += __shfl_xor(t.y, m);
    }
    if (l == 0) f(g, t.x, t.y);
  }
}

template <int ACT, typename T, int VW, int R>
__device__ __forceinline__ void write_grad_rows(const NormArgs& a, const Slab& q, T* out,
                                                int first, int mine, const Pack<T, VW> (&f)[R],
                                                const Pack<T, VW> (&g)[R], const Channel (&k)[VW],
                                                const float2 (&coef)[VW]) {
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (first + i < mine) {
      float v[VW], w[VW];
      unpack<T, VW>(f[i], v);
      unpack<T, VW>(g[i], w);
#pragma unroll
      for (int e = 0; e < VW; ++e) v[e] = norm_value<true, ACT, T>(v[e], w[e], k[e], coef[e]);
      store_pack<T, VW>(out + (size_t)(q.row + (first + i) * q.rows) * a.c, pack<T, VW>(v),
                        a.stream);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace

namespace {

// dgamma and dbeta of a slab's channels from all images' x and dy.
template <typename T, int VW, bool SPAN>
__device__ __forceinline__ void direct_params(const NormArgs& a, int block, float2* lds) {
  constexpr int kDeep = SPAN && VW == 8 ? 2 : 4;
  Slab q;
  q.c0 = block * a.slab_c;
  q.channels = min(a.slab_c, a.c - q.c0);
  q.rows = 1 << a.rows_log2;
  q.row = threadIdx.x >> a.lanes_log2;
  q.ch = (threadIdx.x & ((1 << a.lanes_log2) - 1)) * VW;
  const int ch = min(q.c0 + q.ch, a.c - VW), pixels = a.n * a.hw;
  const float2* stats = (const float2*)a.stats;
  Channel k[VW];
  channel_params<VW>(a, ch, k);
  float s1[VW], s2[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) s1[e] = s2[e] = 0.f;
  by_act(a.act, [&](auto act) {
    for (int i = q.row; i < pixels; i += q.rows * kDeep) {
      Pack<T, VW> f[kDeep], g[kDeep];
      float2 st[kDeep][SPAN ? VW : 1];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        const int p = min(i + j * q.rows, pixels - 1);
        const int img = (int)fast_div((uint32_t)p, a.px_mul, a.px_shift);
        f[j] = load_pack<T, VW>((const T*)a.x + (size_t)p * a.c + ch);
        g[j] = load_pack<T, VW>((const T*)a.dy + (size_t)p * a.c + ch);
#pragma unroll
        for (int e = 0; e < (SPAN ? VW : 1); ++e)
          st[j][e] = stats[(size_t)img * a.groups + group_of(a, ch + e)];
      }
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        if (i + j * q.rows < pixels) {
          float v[VW], w[VW];
          unpack<T, VW>(f[j], v);
          unpack<T, VW>(g[j], w);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            const float2 s = st[j][SPAN ? e : 0];
            const float xh = (v[e] - s.x) * s.y;
            const float dz = norm_act_grad<act.value, T>(w[e], norm_z(xh, k[e].gamma, k[e].beta));
            s1[e] += dz;
            s2[e] += dz * xh;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  });
  float2* sums;
  const int segments = add_rows<VW>(a, q, lds, s1, s2, sums), width = VW << a.lanes_log2;
  for (int i = threadIdx.x; i < q.channels; i += blockDim.x) {
    const float2 t = add_segments(sums, segments, width, i);
    if (a.dbeta) a.dbeta[q.c0 + i] = t.x;
    if (a.dgamma) a.dgamma[q.c0 + i] = t.y;
  }
}

}  // namespace

// ---- all pixels in registers ----------------------------------------------------

// Mean, then the squares around it: two passes, but over registers.  Between loads
// and stores there is one join through LDS; several workgroups a compute unit cover
// it for each other.

template <typename T, int VW, int R, bool SPAN>
__global__ __launch_bounds__(1024) void norm_slab_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  const Slab q = slab_of<VW>(a);
  const int mine = q.in ? pixels_of(a, q, q.row) : 0;
  Pack<T, VW> f[R];
  load_rows<T, VW, R>(a, q, (const T*)a.x + q.at, 0, mine, f);
  float s[VW], m2[VW];
  own_stats<T, VW, R, SPAN>(f, mine, s, m2);
  float2* const result = lds + ((SPAN ? VW : 1) << a.lanes_log2) * q.rows;
  join_stats<VW, SPAN>(a, q, lds, s, m2, [&](int g, float mean, float sq) {
    const float2 st = make_float2(mean, 1.f / sqrtf(sq / ((float)a.d * (float)a.hw) + a.eps));
    result[g] = st;
    ((float2*)a.stats_out)[(size_t)q.img * a.groups + q.c0 / a.d + g] = st;
  });
  __syncthreads();
  if (!q.in) return;
  Channel k[VW];
  channels_of<VW, SPAN>(a, q, result, k);
  by_act(a.act, [&](auto act) {
    write_rows<act.value, T, VW, R>(a, q, (T*)a.out + q.at, 0, mine, f, k);
  });
}

template <typename T, int VW, int R, bool SPAN, bool DIRECT>
__global__ __launch_bounds__(1024) void norm_slab_grad_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  if constexpr (DIRECT) {  // (a kernel of its own: these take more registers)
    if ((int)blockIdx.x >= a.slabs) {
      direct_params<T, VW, SPAN>(a, blockIdx.x - a.slabs, lds);
      return;
    }
  }
  const Slab q = slab_of<VW>(a);
  const int mine = q.in ? pixels_of(a, q, q.row) : 0;
  Pack<T, VW> f[R], g[R];
  load_rows<T, VW, R>(a, q, (const T*)a.x + q.at, 0, mine, f);
  load_rows<T, VW, R>(a, q, (const T*)a.dy + q.at, 0, mine, g);
  Channel k[VW];
  grad_channels<VW, SPAN>(a, q, k);
  float s1[VW], s2[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) s1[e] = s2[e] = 0.f;
  by_act(a.act, [&](auto act) {
    add_grad_sums<act.value, T, VW, R>(a, 0, mine, f, g, k, s1, s2);
  });
#pragma unroll
  for (int i = 0; i < R; ++i) {
    forget(f[i]);
    forget(g[i]);
  }
  const float total = (float)a.d * (float)a.hw;
  float2* const result = lds;  // the rows are done with by then
  join_grad_sums<VW>(a, q, lds, s1, s2, [&](int grp, float t1, float t2) {
    result[grp] = make_float2(t1 / total, t2 / total);
  });
  __syncthreads();
  if (!q.in) return;
  float2 coef[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) coef[e] = result[group_of(a, q.ch + (SPAN ? e : 0))];
  by_act(a.act, [&](auto act) {
    write_grad_rows<act.value, T, VW, R>(a, q, (T*)a.out + q.at, 0, mine, f, g, k, coef);
  });
}

// ---- runs of pixels, two passes ---------------------------------------------------

constexpr int kRun = 4;  // vectors of a thread in flight (8: no faster, more registers)

// First pass: a run's (mean, squares around it) per group.
template <typename T, int VW, bool SPAN>
__global__ __launch_bounds__(1024) void norm_run_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  const Slab q = slab_of<VW>(a);
  const int mine = q.in ? pixels_of(a, q, q.row) : 0;
  float s[VW], m2[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) s[e] = m2[e] = 0.f;
  for (int i = 0; i < mine; i += kRun) {
    Pack<T, VW> f[kRun];
    load_rows<T, VW, kRun>(a, q, (const T*)a.x + q.at, i, mine, f);
    float bs[VW], bm2[VW];
    own_stats<T, VW, kRun, SPAN>(f, min(kRun, mine - i), bs, bm2);
    join_batch<VW, SPAN>(i, min(kRun, mine - i), bs, bm2, s, m2);
  }
  join_stats<VW, SPAN>(a, q, lds, s, m2, [&](int g, float mean, float sq) {
    a.gpart[((size_t)q.img * a.chunks + q.chunk) * a.groups + q.c0 / a.d + g] =
        make_float2(mean, sq);
  });
}

// Second pass: the runs' sums joined by every workgroup for its own groups, and y.
template <typename T, int VW, bool SPAN>
__global__ __launch_bounds__(1024) void norm_run_apply_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  const Slab q = slab_of<VW>(a);
  const int mine = q.in ? pixels_of(a, q, q.row) : 0;
  const T* x = (const T*)a.x + q.at;
  Pack<T, VW> f[kRun];
  load_rows<T, VW, kRun>(a, q, x, 0, mine, f);  // in flight meanwhile
  const int gl = 1 << a.join_log2, l = threadIdx.x & (gl - 1);
  for (int g = threadIdx.x >> a.join_log2; g < q.groups; g += blockDim.x >> a.join_log2) {
    const float2* part = a.gpart + (size_t)q.img * a.chunks * a.groups + q.c0 / a.d + g;
    const float per = (float)a.d, total = per * (float)a.hw;
    // The mean and the squares around it, of the runs of a lane eight by eight (all loads of
    // eight in flight: their latency is what this takes), then of the lanes; not around one
    // run's mean, which may lie far from the others.  n: pixels.
    constexpr int kHeld = 8;
    float n = 0.f, mean = 0.f, sq = 0.f;
    for (int c0 = l; c0 < a.chunks; c0 += gl * kHeld) {
      float2 v[kHeld];
      float w[kHeld], now = 0.f, s = 0.f, m2 = 0.f;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int c = c0 + i * gl;
        v[i] = c < a.chunks ? part[(size_t)c * a.groups] : make_float2(0.f, 0.f);
        w[i] = c < a.chunks ? (float)min(a.chunk_len, a.hw - c * a.chunk_len) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kHeld; ++i) now += w[i], s += w[i] * v[i].x;
      s *= __builtin_amdgcn_rcpf(now);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) m2 += v[i].y + w[i] * per * ((v[i].x - s) * (v[i].x - s));
      const float share = now * __builtin_amdgcn_rcpf(n + now), d = s - mean;
      sq += m2 + d * (d * (n * share * per));
      mean += d * share;
      n += now;
    }
    float all = n * mean;
    for (int m = gl >> 1; m; m >>= 1) all += __shfl_xor(all, m);
    all /= (float)a.hw;
    sq += n * per * ((mean - all) * (mean - all));
    for (int m = gl >> 1; m; m >>= 1) sq += __shfl_xor(sq, m);
    if (l == 0) {
      const float2 st = make_float2(all, 1.f / sqrtf(sq / total + a.eps));
      lds[g] = st;
      if (q.chunk == 0) ((float2*)a.stats_out)[(size_t)q.img * a.groups + q.c0 / a.d + g] = st;
    }
  }
  __syncthreads();
  if (!q.in) return;
  Channel k[VW];
  channels_of<VW, SPAN>(a, q, lds, k);
  T* out = (T*)a.out + q.at;
  by_act(a.act, [&](auto act) {
    write_rows<act.value, T, VW, kRun>(a, q, out, 0, mine, f, k);
    for (int i = kRun; i < mine; i += kRun) {
      load_rows<T, VW, kRun>(a, q, x, i, mine, f);
      write_rows<act.value, T, VW, kRun>(a, q, out, i, mine, f, k);
    }
  });
}

template <typename T, int VW, bool SPAN>
__global__ __launch_bounds__(1024) void norm_run_grad_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  const Slab q = slab_of<VW>(a);
  const int mine = q.in ? pixels_of(a, q, q.row) : 0;
  Channel k[VW];
  grad_channels<VW, SPAN>(a, q, k);
  float s1[VW], s2[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) s1[e] = s2[e] = 0.f;
  by_act(a.act, [&](auto act) {
    for (int i = 0; i < mine; i += kRun) {
      Pack<T, VW> f[kRun], g[kRun];
      load_rows<T, VW, kRun>(a, q, (const T*)a.x + q.at, i, mine, f);
      load_rows<T, VW, kRun>(a, q, (const T*)a.dy + q.at, i, mine, g);
      add_grad_sums<act.value, T, VW, kRun>(a, i, mine, f, g, k, s1, s2);
    }
  });
  join_grad_sums<VW>(a, q, lds, s1, s2, [&](int grp, float t1, float t2) {
    a.gpart[((size_t)q.img * a.chunks + q.chunk) * a.groups + q.c0 / a.d + grp] =
        make_float2(t1, t2);
  });
}

// ... and dx; workgroups behind the slabs': dgamma and dbeta.
template <typename T, int VW, bool SPAN>
__global__ __launch_bounds__(1024) void norm_run_grad_apply_nhwc_kernel(NormArgs a) {
  extern __shared__ float2 lds[];
  constexpr int kDeep = SPAN && VW == 8 ? kRun / 2 : kRun;  // 128 registers
  if ((int)blockIdx.x >= a.slabs) {
    __shared__ ParamSums sums;
    param_sums(a, blockIdx.x - a.slabs, sums);
    return;
  }
  const Slab q = slab_of<VW>(a);
  const int mine = q.in ? pixels_of(a, q, q.row) : 0;
  const T* x = (const T*)a.x + q.at;
  const T* dy = (const T*)a.dy + q.at;
  Pack<T, VW> f[kDeep], w[kDeep];
  load_rows<T, VW, kDeep>(a, q, x, 0, mine, f);
  load_rows<T, VW, kDeep>(a, q, dy, 0, mine, w);
  const int gl = 1 << a.join_log2, l = threadIdx.x & (gl - 1);
  for (int g = threadIdx.x >> a.join_log2; g < q.groups; g += blockDim.x >> a.join_log2) {
    const float2* part = a.gpart + (size_t)q.img * a.chunks * a.groups + q.c0 / a.d + g;
    float2 t = make_float2(0.f, 0.f);
#pragma unroll 8
    for (int c = l; c < a.chunks; c += gl) {
      const float2 v = part[(size_t)c * a.groups];
      t.x += v.x;
      t.y += v.y;
    }
    for (int m = gl >> 1; m; m >>= 1) {
      t.x += __shfl_xor(t.x, m);
      t.y += __shfl_xor(t.y, m);
    }
    const float total = (float)a.d * (float)a.hw;
    if (l == 0) lds[g] = make_float2(t.x / total, t.y / total);
  }
  __syncthreads();
  if (!q.in) return;
  Channel k[VW];
  grad_channels<VW, SPAN>(a, q, k);
  float2 coef[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) coef[e] = lds[group_of(a, q.ch + (SPAN ? e : 0))];
  T* out = (T*)a.out + q.at;
  by_act(a.act, [&](auto act) {
    write_grad_rows<act.value, T, VW, kDeep>(a, q, out, 0, mine, f, w, k, coef);
    for (int i = kDeep; i < mine; i += kDeep) {
      load_rows<T, VW, kDeep>(a, q, x, i, mine, f);
      load_rows<T, VW, kDeep>(a, q, dy, i, mine, w);
      write_grad_rows<act.value, T, VW, kDeep>(a, q, out, i, mine, f, w, k, coef);
    }
  });
}

namespace {

template <typename T, int VW, int R, bool GRAD, bool SPAN>
void launch_slab(const NormArgs& a, hipStream_t stream) {
  if constexpr (GRAD) {
    const int direct = a.dgamma || a.dbeta ? a.direct : 0;
    const auto kernel = direct ? norm_slab_grad_nhwc_kernel<T, VW, R, SPAN, true>
                               : norm_slab_grad_nhwc_kernel<T, VW, R, SPAN, false>;
    hipLaunchKernelGGL(kernel, dim3(a.slabs + direct), dim3(a.threads), a.lds_bytes, stream, a);
  } else
    hipLaunchKernelGGL((norm_slab_nhwc_kernel<T, VW, R, SPAN>), dim3(a.slabs), dim3(a.threads),
                       a.lds_bytes, stream, a);
}

template <typename T, int VW, bool GRAD, bool SPAN>
void launch_t(const NormArgs& a, hipStream_t stream) {
  if (a.slots == 0) {
    const dim3 grid(a.slabs), wg(a.threads);
    const int group_bytes = a.slab_c / a.d * (int)sizeof(float2);
    if constexpr (GRAD) {
      const unsigned params = (a.dgamma || a.dbeta) && a.n * a.chunks > 1 ? (a.c + 15) / 16 : 0;
      hipLaunchKernelGGL((norm_run_grad_nhwc_kernel<T, VW, SPAN>), grid, wg, a.lds_bytes, stream,
                         a);
      hipLaunchKernelGGL((norm_run_grad_apply_nhwc_kernel<T, VW, SPAN>), dim3(a.slabs + params), wg,
                         group_bytes, stream, a);
    } else {
      hipLaunchKernelGGL((norm_run_nhwc_kernel<T, VW, SPAN>), grid, wg, a.lds_bytes, stream, a);
      hipLaunchKernelGGL((norm_run_apply_nhwc_kernel<T, VW, SPAN>), grid, wg, group_bytes, stream,
                         a);
    }
    return;
  }
  if (a.slots == 1)
    launch_slab<T, VW, 1, GRAD, SPAN>(a, stream);
  else if (a.slots <= 4)
    launch_slab<T, VW, 4, GRAD, SPAN>(a, stream);
  else if constexpr (slab_most(VW, GRAD, SPAN) > 4)
    launch_slab<T, VW, slab_most(VW, GRAD, SPAN), GRAD, SPAN>(a, stream);
  // (its error is the last one, read by the caller)
  if (GRAD && a.n > 1 && !a.direct && (a.dgamma || a.dbeta)) (void)launch_norm_params(a, stream);
}

template <typename T, int VW, bool GRAD>
void launch_v(const NormArgs& a, hipStream_t stream) {
  if constexpr (VW > 1)
    if (a.span) return launch_t<T, VW, GRAD, true>(a, stream);
  launch_t<T, VW, GRAD, false>(a, stream);
}

template <bool GRAD>
hipError_t launch_any(const NormArgs& a, int dtype, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16) {
    if (vec == 8)
      launch_v<uint16_t, 8, GRAD>(a, stream);
    else if (vec == 2)
      launch_v<uint16_t, 2, GRAD>(a, stream);
    else
      launch_v<uint16_t, 1, GRAD>(a, stream);
  } else if (vec == 4) {
    launch_v<uint32_t, 4, GRAD>(a, stream);
  } else {
    launch_v<uint32_t, 1, GRAD>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_nhwc(const NormArgs& a, int dtype, int vec, hipStream_t stream) {
  return launch_any<false>(a, dtype, vec, stream);
}
hipError_t launch_norm_grad_nhwc(const NormArgs& a, int dtype, int vec, hipStream_t stream) {
  return launch_any<true>(a, dtype, vec, stream);
}

}  // namespace huge2
