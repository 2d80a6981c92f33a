// layer_planes.hip -- layer norm over the channels of each pixel in NCHW, where a pixel's
// channels lie a plane apart.
#include <algorithm>

#include "layer_device.hpp"

namespace huge2 {

namespace {

// A tile: lanes side by side on an image's pixels, a vector of them each; rows of lanes
// have every `rows`-th channel.
struct Tile {
  int img;
  Piece q;       // of the image's plane
  size_t first;  // element of (img, channel 0, pixel 0)
};
template <int VW, bool RAGGED>
__device__ __forceinline__ Tile tile_of(const LayerArgs& a, uint32_t t, int lane) {
  Tile i;
  i.img = (int)fast_div(t, a.tile_mul, a.tile_shift);
  const int p = (int)(t - (uint32_t)i.img * (uint32_t)a.tiles_per_image);
  i.q = piece<VW, RAGGED>((((long long)p << a.lanes_log2) + lane) * VW, a.hw);
  i.first = (size_t)i.img * a.c * a.hw;
  return i;
}

// The place of a thread's k-th vector: a base of the workgroup's (k * rows channels behind
// the image) and an offset in 32 bits, which all k share (images that are held take less than
// 2^32 bytes).  The compiler would else keep a sum of them, two registers, for each k.
template <typename T>
__device__ __forceinline__ T* slot_at(T* image, size_t rows_b, int k, uint32_t offset) {
  const uint64_t base = (uint64_t)image + k * rows_b;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)base);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((int)(base >> 32));
  return (T*)((__attribute__((address_space(1))) char*)((uint64_t)hi << 32 | lo) + offset);
}

// Sums over a workgroup's rows of lanes of N values for each lane, in every row; lds:
// [waves][lanes][N].
template <int N>
__device__ __forceinline__ void rows_sum(float (&v)[N], int threads, int lanes_log2,
                                         float* lds) {
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & (lanes - 1);
  scatter_sum<N>(v, lanes_log2);
  __syncthreads();
  if ((int)(threadIdx.x & 7) < lanes) {
    float* const to = lds + ((threadIdx.x >> 6) * lanes + lane) * N + scatter_at<N>();
#pragma unroll
    for (int e = 0; e < (N > 7 ? N / 8 : 1); ++e) to[e] = v[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = lds[lane * N + e];
  for (int w = 1; w < threads >> 6; ++w) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += lds[(w * lanes + lane) * N + e];
  }
}

__device__ __forceinline__ Channel plane_params(const LayerArgs& a, int ch) {
  return {0.f, 0.f, a.gamma ? a.gamma[ch] : 1.f, a.beta ? a.beta[ch] : 0.f};
}
// The same with addresses of one register (held channels are few).
__device__ __forceinline__ Channel slot_params(const LayerArgs& a, int ch) {
  const uint32_t at = (uint32_t)ch * (uint32_t)sizeof(float);
  return {0.f, 0.f, a.gamma ? *(const float*)((const char*)a.gamma + at) : 1.f,
          a.beta ? *(const float*)((const char*)a.beta + at) : 0.f};
}

}  // namespace

// A tile's channels are held by the rows of a workgroup, R vectors a thread, or (R = 0) read
// again for each of the sums and the result.  (A tile to a workgroup: in a loop over tiles the
// compiler holds what does not change, and 40 of 128 registers spill.)
//
// 64 images of 256x16x16 bf16 8.2 us, 17 MB: one round of 256 tiles, bound by its latency (loads,
// two sums through LDS, stores).  64 of 128x64x64 34 us, 134 MB at 4.0 TB/s, fetched and written
// once each: the same latency in every round, with nothing of the next tile on its way; fp32
// 54 us, 4.9 TB/s.  2048 channels in tiles of 32 bytes, 64 images of 16x16, 35 us, 3.9 TB/s.
template <typename T, int VW, int R, bool RAGGED>
__global__ __launch_bounds__(1024) void layer_planes_kernel(LayerArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int row = threadIdx.x >> a.lanes_log2, rows = a.threads >> a.lanes_log2;
  const size_t rows_b = (size_t)rows * a.hw * sizeof(T);
  const float inv = 1.f / (float)a.c;
  constexpr int kHeld = R ? R : 1;
  by_act(a.act, [&](auto act) {
    const Tile i = tile_of<VW, RAGGED>(a, a.first_tile + blockIdx.x, lane);
    const T* x = (const T*)a.x + i.first;
    T* y = (T*)a.out + i.first;
    const uint32_t offset = ((uint32_t)row * (uint32_t)a.hw + i.q.at) * sizeof(T);
    Pack<T, VW> f[kHeld] = {};
    const auto each = [&](auto&& g) {  // g(slot, channel, values)
      if constexpr (R) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const int ch = row + k * rows;
          float v[VW];
          unpack<T, VW>(f[k], v);
          if (i.q.in && ch < a.c) g(k, ch, v);
          forget(f[k]);
        }
      } else if (i.q.in) {
        for (int ch = row; ch < a.c; ch += rows) {
          float v[VW];
          unpack<T, VW>(load_run<T, VW>(x + (size_t)ch * a.hw + i.q.at), v);
          g(0, ch, v);
        }
      }
    };
    // (their parameters with them, where the registers hold both)
    constexpr bool kParams = R > 0 && R <= 8;
    Channel params[kParams ? R : 1];
    if constexpr (R) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int ch = row + k * rows;
        if (i.q.in && ch < a.c) {
          f[k] = load_run<T, VW>(slot_at(x, rows_b, k, offset));
          if constexpr (kParams) params[k] = slot_params(a, ch);
        }
      }
    }
    float s[VW] = {}, mean[VW], rstd[VW];
    each([&](int, int, float (&v)[VW]) {
#pragma unroll
      for (int e = 0; e < VW; ++e) s[e] += v[e];
    });
    rows_sum<VW>(s, a.threads, a.lanes_log2, lds);
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      mean[e] = s[e] * inv;
      s[e] = 0.f;
    }
    each([&](int, int, float (&v)[VW]) {
#pragma unroll
      for (int e = 0; e < VW; ++e) s[e] += (v[e] - mean[e]) * (v[e] - mean[e]);
    });
    rows_sum<VW>(s, a.threads, a.lanes_log2, lds);
#pragma unroll
    for (int e = 0; e < VW; ++e) rstd[e] = 1.f / sqrtf(s[e] * inv + a.eps);
    each([&](int k, int ch, float (&v)[VW]) {
      const Channel p = kParams ? params[k] : R ? slot_params(a, ch) : plane_params(a, ch);
#pragma unroll
      for (int e = 0; e < VW; ++e)
        v[e] = norm_value<false, decltype(act)::value, T>(
            v[e], 0.f, {mean[e], rstd[e], p.gamma, p.beta}, make_float2(0.f, 0.f));
      T* to = R ? slot_at(y, rows_b, k, offset) : y + (size_t)ch * a.hw + i.q.at;
      store_run<T, VW>(to, pack<T, VW>(v), a.stream);
    });
    if (a.stats_out && row == 0 && i.q.in) {
      float2* st = (float2*)a.stats_out + (size_t)i.img * a.hw + i.q.at;
#pragma unroll
      for (int e = 0; e < VW; ++e) st[e] = make_float2(mean[e], rstd[e]);
    }
  });
}

// The gradient by the same tiles.  A thread adds up dgamma and dbeta of its channels over the
// workgroup's tiles (R = 0: layer_plane_sums_kernel does).
//
// 5 images of 200x33x41 fp32 with SiLU 10.9 us, 16 MB: one round of 215 tiles, in which fp32's
// exponential and division take as long as the loads, and 22 MB are fetched for the 11 of x and
// dy: an odd map's tiles share lines, and tiles side by side are on different dies.  64 of
// 128x64x64 bf16 46 us, 4.4 TB/s, fetched once.  Over 512 channels tiles are narrower than a
// line, and each die fetches its own: 64 images of 1024x16x16 41 us, twice the bytes; of
// 2048x16x16 120 us, four times, 538 MB.
template <typename T, int VW, int R, bool RAGGED>
__global__ __launch_bounds__(R * VW > kLayerWideChannels ? 512 : 1024) void
layer_grad_planes_kernel(LayerArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int row = threadIdx.x >> a.lanes_log2, rows = a.threads >> a.lanes_log2;
  const size_t rows_b = (size_t)rows * a.hw * sizeof(T);
  const float inv = 1.f / (float)a.c;
  constexpr int kHeld = R ? R : 1;
  float dg[kHeld] = {}, db[kHeld] = {};
  // x and dy become what dx is made of (a smooth activation takes longer than the rest), or are
  // kept, where that would be too many registers.
  constexpr bool kMade = R > 0 && R * VW <= 2 * kLayerWideChannels;
  by_act(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    for (uint32_t t = blockIdx.x; t < a.tiles; t += gridDim.x) {
      const Tile i = tile_of<VW, RAGGED>(a, t, lane);
      const T* x = (const T*)a.x + i.first;
      const T* dy = (const T*)a.dy + i.first;
      T* out = (T*)a.out + i.first;
      const uint32_t offset = ((uint32_t)row * (uint32_t)a.hw + i.q.at) * sizeof(T);
      Pack<T, VW> f[kHeld] = {}, d[kHeld] = {};
      Channel params[kMade ? R : 1];
      const auto each = [&](auto&& g) {  // g(slot, channel, x, dy)
        if constexpr (R) {
#pragma unroll
          for (int k = 0; k < R; ++k) {
            const int ch = row + k * rows;
            float v[VW], w[VW];
            unpack<T, VW>(f[k], v);
            unpack<T, VW>(d[k], w);
            if (i.q.in && ch < a.c) g(k, ch, v, w);
            forget(f[k]);
            forget(d[k]);
          }
        } else if (i.q.in) {
          for (int ch = row; ch < a.c; ch += rows) {
            float v[VW], w[VW];
            unpack<T, VW>(load_run<T, VW>(x + (size_t)ch * a.hw + i.q.at), v);
            unpack<T, VW>(load_run<T, VW>(dy + (size_t)ch * a.hw + i.q.at), w);
            g(0, ch, v, w);
          }
        }
      };
      if constexpr (R) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const int ch = row + k * rows;
          if (i.q.in && ch < a.c) {
            f[k] = load_run<T, VW>(slot_at(x, rows_b, k, offset));
            d[k] = load_run<T, VW>(slot_at(dy, rows_b, k, offset));
            if constexpr (kMade) params[k] = slot_params(a, ch);
          }
        }
      }
      float2 st[VW];
      if (i.q.in) {
        const float2* from = (const float2*)a.stats + (size_t)i.img * a.hw + i.q.at;
#pragma unroll
        for (int e = 0; e < VW; ++e) st[e] = from[e];
      } else {
#pragma unroll
        for (int e = 0; e < VW; ++e) st[e] = make_float2(0.f, 0.f);
      }
      float s[2 * VW] = {}, made[kMade ? R : 1][2 * VW];
      each([&](int k, int ch, float (&v)[VW], float (&w)[VW]) {
        const Channel p = kMade ? params[k] : R ? slot_params(a, ch) : plane_params(a, ch);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          float xh, dz;
          layer_dz<ACT, T>(v[e], w[e], {st[e].x, st[e].y, p.gamma, p.beta}, xh, dz);
          const float t = dz * p.gamma;
          s[e] += t;
          s[VW + e] += t * xh;
          if constexpr (kMade) made[k][e] = xh, made[k][VW + e] = t;
          if (R && (!RAGGED || e >= i.q.skip)) {
            db[k] += dz;
            dg[k] += dz * xh;
          }
        }
      });
      rows_sum<2 * VW>(s, a.threads, a.lanes_log2, lds);
#pragma unroll
      for (int e = 0; e < 2 * VW; ++e) s[e] *= inv;
      // dx = rstd (t - the mean of t - xh times the mean of t xh)
      if constexpr (kMade) {
        float c0[VW], c1[VW];
#pragma unroll
        for (int e = 0; e < VW; ++e) c0[e] = -st[e].y * s[e], c1[e] = -st[e].y * s[VW + e];
#pragma unroll
        for (int k = 0; k < R; ++k) {
          float v[VW];
#pragma unroll
          for (int e = 0; e < VW; ++e)
            v[e] = fmaf(made[k][e], c1[e], fmaf(made[k][VW + e], st[e].y, c0[e]));
          if (i.q.in && row + k * rows < a.c)
            store_run<T, VW>(slot_at(out, rows_b, k, offset), pack<T, VW>(v), a.stream);
        }
      } else {
        asm volatile("" ::: "memory");  // (gamma and beta are read again, not held)
        each([&](int k, int ch, float (&v)[VW], float (&w)[VW]) {
          const Channel p = R ? slot_params(a, ch) : plane_params(a, ch);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            float xh, dz;
            layer_dz<ACT, T>(v[e], w[e], {st[e].x, st[e].y, p.gamma, p.beta}, xh, dz);
            v[e] = st[e].y * (dz * p.gamma - s[e] - xh * s[VW + e]);
          }
          T* to = R ? slot_at(out, rows_b, k, offset) : out + (size_t)ch * a.hw + i.q.at;
          store_run<T, VW>(to, pack<T, VW>(v), a.stream);
        });
      }
    }
  });
  if (!R || !a.part) return;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    db[k] = side_sum(db[k], a.lanes_log2);
    dg[k] = side_sum(dg[k], a.lanes_log2);
    const int ch = row + k * rows;
    if (lane == 0 && ch < a.c) a.part[(size_t)blockIdx.x * a.c + ch] = make_float2(db[k], dg[k]);
  }
}

// dgamma and dbeta of a channel over some images' pixels: a workgroup each.
template <typename T, int VW, bool RAGGED>
__global__ __launch_bounds__(256) void layer_plane_sums_kernel(LayerArgs a) {
  __shared__ float lds[4];
  const int ch = blockIdx.x;
  const Channel p = plane_params(a, ch);
  by_act(a.act, [&](auto act) {
    float dg = 0.f, db = 0.f;
    for (int img = blockIdx.y; img < a.n; img += gridDim.y) {
      const size_t plane = ((size_t)img * a.c + ch) * a.hw;
      const float2* st = (const float2*)a.stats + (size_t)img * a.hw;
      for (long long i = (long long)threadIdx.x * VW; i < a.hw; i += 256 * VW) {
        const Piece q = piece<VW, RAGGED>(i, a.hw);
        float v[VW], w[VW];
        unpack<T, VW>(load_run<T, VW>((const T*)a.x + plane + q.at), v);
        unpack<T, VW>(load_run<T, VW>((const T*)a.dy + plane + q.at), w);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          if (RAGGED && e < q.skip) continue;
          const float2 s = st[q.at + e];
          float xh, dz;
          layer_dz<decltype(act)::value, T>(v[e], w[e], {s.x, s.y, p.gamma, p.beta}, xh, dz);
          db += dz;
          dg += dz * xh;
        }
      }
    }
    db = block_sum(db, lds);
    __syncthreads();
    dg = block_sum(dg, lds);
    if (threadIdx.x == 0) a.part[(size_t)blockIdx.y * a.c + ch] = make_float2(db, dg);
  });
}

namespace {

template <typename T, int VW, int R, bool RAGGED>
void launch_planes(const LayerArgs& a, bool grad, hipStream_t stream) {
  const int lds = (a.threads / 64 * VW * (grad ? 2 : 1) * (int)sizeof(float)) << a.lanes_log2;
  if (!grad) {
    LayerArgs b = a;
    const uint32_t most = (uint32_t)((1ll << 32) / a.threads - 1);  // that one launch takes
    for (; b.first_tile < a.tiles; b.first_tile += most)
      hipLaunchKernelGGL((layer_planes_kernel<T, VW, R, RAGGED>),
                         dim3(std::min(most, a.tiles - b.first_tile)), dim3(a.threads), lds, stream,
                         b);
  } else if constexpr (R <= kLayerGradPlanes)
    hipLaunchKernelGGL((layer_grad_planes_kernel<T, VW, R, RAGGED>), dim3(a.groups),
                       dim3(a.threads), lds, stream, a);
  if (grad && R == 0 && a.part)
    hipLaunchKernelGGL((layer_plane_sums_kernel<T, VW, RAGGED>), dim3(a.c, a.parts), dim3(256), 0,
                       stream, a);
}

template <typename T, int VW, bool RAGGED>
void launch_slots(const LayerArgs& a, bool grad, hipStream_t stream) {
  switch (a.slots) {
    case 0: return launch_planes<T, VW, 0, RAGGED>(a, grad, stream);
    case 1: return launch_planes<T, VW, 1, RAGGED>(a, grad, stream);
    case 2: return launch_planes<T, VW, 2, RAGGED>(a, grad, stream);
    case 4: return launch_planes<T, VW, 4, RAGGED>(a, grad, stream);
    case 8: return launch_planes<T, VW, 8, RAGGED>(a, grad, stream);
    default: return launch_planes<T, VW, 16, RAGGED>(a, grad, stream);
  }
}

template <typename T>
void launch_type(const LayerArgs& a, int vec, bool grad, hipStream_t stream) {
  constexpr int kFull = 16 / (int)sizeof(T);
  if (vec == 1)
    launch_slots<T, 1, false>(a, grad, stream);
  else if (a.hw % kFull)
    launch_slots<T, kFull, true>(a, grad, stream);
  else
    launch_slots<T, kFull, false>(a, grad, stream);
}

}  // namespace

hipError_t launch_layer_planes(const LayerArgs& a, int dtype, int vec, bool grad,
                               hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    launch_type<uint16_t>(a, vec, grad, stream);
  else
    launch_type<uint32_t>(a, vec, grad, stream);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !grad ? e : launch_layer_params(a, stream);
}

}  // namespace huge2
