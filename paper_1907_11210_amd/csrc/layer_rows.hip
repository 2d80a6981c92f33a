// layer_rows.hip -- layer norm of rows of channels: NHWC, lists of tokens, 1x1 maps.
#include <algorithm>

#include "layer_device.hpp"

namespace huge2 {

namespace {

// Sum over the 2^lanes_log2 lanes side by side on a row, in each of them; lds: a value
// for each wave (rows of more than a wave, which are a workgroup's only one).
__device__ __forceinline__ float row_sum(float v, int lanes_log2, float* lds) {
  v = side_sum(v, lanes_log2);
  if (lanes_log2 <= 6) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < 1 << (lanes_log2 - 6); ++w) v += lds[w];
  return v;
}
__device__ __forceinline__ float2 row_sums(float2 v, int lanes_log2, float2* lds) {
  v.x = side_sum(v.x, lanes_log2);
  v.y = side_sum(v.y, lanes_log2);
  if (lanes_log2 <= 6) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < 1 << (lanes_log2 - 6); ++w) {
    v.x += lds[w].x;
    v.y += lds[w].y;
  }
  return v;
}

// gamma and beta of a vector's channels, by 16 bytes.  (By 4 a wave's loads of a row's
// parameters take longer than the row: 64x64x2048, 8 images, 50 us without parameters and 79.)
template <int VW>
__device__ __forceinline__ void load_params(const float* p, int ch, float none, float (&f)[VW]) {
  typedef u32x4 floats __attribute__((aligned(4)));
  if (!p) {
#pragma unroll
    for (int e = 0; e < VW; ++e) f[e] = none;
  } else if constexpr (VW == 1) {
    f[0] = p[ch];
  } else {
#pragma unroll
    for (int e = 0; e < VW; e += 4) {
      const u32x4 v = *(const floats*)(p + ch + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[e + i] = __uint_as_float(v[i]);
    }
  }
}
template <int VW>
__device__ __forceinline__ void vector_params(const LayerArgs& a, int ch, float (&g)[VW],
                                              float (&b)[VW]) {
  load_params<VW>(a.gamma, ch, 1.f, g);
  load_params<VW>(a.beta, ch, 0.f, b);
}

// A lane's gamma and beta for the rows that follow each other in its team: where rows are a
// wave's in LDS ([c] each, rounded up to 4; 2048 channels take 16 KB), else read for each row.
template <int VW, bool WAVE>
struct Params {
  float* lds;
  __device__ __forceinline__ Params(const LayerArgs& a, float* room) : lds(room) {
    if constexpr (WAVE) {
      for (int i = threadIdx.x * 4; i < a.c; i += 1024) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const float* from = p ? a.beta : a.gamma;
          float v[4];
          if (i + 4 <= a.c) {
            load_params<4>(from, i, p ? 0.f : 1.f, v);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = from && i + e < a.c ? from[i + e] : p ? 0.f : 1.f;
          }
          *(float4*)(lds + p * rounded(a.c) + i) = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
      __syncthreads();
    }
  }
  static __device__ __forceinline__ int rounded(int c) { return (c + 3) & ~3; }
  __device__ __forceinline__ void read(const LayerArgs& a, int ch, float (&g)[VW],
                                       float (&b)[VW]) const {
    if constexpr (WAVE) {
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        g[e] = lds[ch + e];
        b[e] = lds[rounded(a.c) + ch + e];
      }
    } else {
      vector_params<VW>(a, ch, g, b);
    }
  }
};

}  // namespace

// How a row's channels fill its lanes' vectors: all of them, some, or with a last vector that
// repeats elements of the one before.
enum RowFill { kFull = 0, kPart = 1, kRagged = 2 };

namespace {

template <int VW, int R, int FILL>
struct Lanes {
  Piece q[R];
  __device__ __forceinline__ Lanes(const LayerArgs& a, int l) {
#pragma unroll
    for (int k = 0; k < R; ++k)
      q[k] = piece<VW, FILL == kRagged>(((long long)(k << a.lanes_log2) + l) * VW, a.c);
  }
  __device__ __forceinline__ bool in(int k) const { return FILL == kFull || q[k].in; }
  // Whether element e of vector k counts.
  __device__ __forceinline__ bool counts(int k, int e) const {
    return in(k) && (FILL != kRagged || e >= q[k].skip);
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* row, Pack<T, VW> (&f)[R]) const {
#pragma unroll
    for (int k = 0; k < R; ++k)
      if (in(k)) f[k] = load_run<T, VW>(row + q[k].at);
  }
};

}  // namespace

// A row is held by 2^lanes_log2 lanes, R vectors each: read once, its mean, the squares
// around it, and the result from registers.  Rows follow each other in a team of lanes, the
// next on its way while one is worked on.  WAVE: teams are waves or parts of them, else a
// workgroup.
//
// Bound by the bytes: 8 images of 64x64x2048 bf16 49 us, 268 MB at 5.5 TB/s (a copy: 5.2, which
// this passes since the results leave past the caches).  In small calls by latency: a load, two
// sums over lanes, a store, 3.7 us of 64 rows of 512.  Teams are waves or less as long as a
// wave's registers hold a row (32 channels a lane), since a wave's sums need no barrier.
template <typename T, int VW, int R, int FILL, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void layer_rows_kernel(LayerArgs a) {
  __shared__ float lds[16];
  extern __shared__ __attribute__((aligned(16))) float kept[];  // WAVE: gamma and beta
  const int lanes = 1 << a.lanes_log2, l = threadIdx.x & (lanes - 1);
  const int teams = a.threads >> a.lanes_log2, team = threadIdx.x >> a.lanes_log2;
  const float inv = 1.f / (float)a.c;
  const Lanes<VW, R, FILL> of(a, l);
  const Params<VW, WAVE> params(a, kept);
  by_act(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    const long long step = (long long)gridDim.x * teams;
    long long r = (long long)blockIdx.x * teams + team;
    Pack<T, VW> f[R] = {};
    if (r < a.rows) of.load((const T*)a.x + r * a.c, f);
    for (; r < a.rows; r += step) {
      float v[R][VW], s[4] = {};
#pragma unroll
      for (int k = 0; k < R; ++k) unpack<T, VW>(f[k], v[k]);
      if (r + step < a.rows) of.load((const T*)a.x + (r + step) * a.c, f);
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int e = 0; e < VW; ++e) s[e & 3] += of.counts(k, e) ? v[k][e] : 0.f;
      const float mean = row_sum((s[0] + s[1]) + (s[2] + s[3]), a.lanes_log2, lds) * inv;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          v[k][e] -= mean;
          const float d = of.counts(k, e) ? v[k][e] : 0.f;
          s[e & 3] += d * d;
        }
      const float rstd =
          1.f / sqrtf(row_sum((s[0] + s[1]) + (s[2] + s[3]), a.lanes_log2, lds) * inv + a.eps);
      T* y = (T*)a.out + r * a.c;
      asm volatile("" ::: "memory");  // (gamma and beta stay where they are)
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float g[VW], b[VW];
        params.read(a, of.q[k].at, g, b);
#pragma unroll
        for (int e = 0; e < VW; ++e) v[k][e] = layer_value<ACT, T>(v[k][e], rstd, g[e], b[e]);
        if (of.in(k)) store_run<T, VW>(y + of.q[k].at, pack<T, VW>(v[k]), a.stream);
      }
      if (a.stats_out && l == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
    }
  });
}

// The gradient by the same rows: x and dy held, the two means, dx from registers.  A thread
// adds up dgamma and dbeta of its channels over the team's rows; the teams' sums are joined
// in LDS, the workgroups' by layer_params_kernel.
//
// Bound by the bytes: 32768 rows of 1024 bf16 41 us, 201 MB at 4.9 TB/s, and 5 us of
// layer_params_kernel; 65536 rows of 128 15.9 us, 3.2 TB/s: four or five rows a
// team one behind the other, each a load, sums over lanes and a store, and the sums' join.
template <typename T, int VW, int R, int FILL, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void layer_grad_rows_kernel(LayerArgs a) {
  __shared__ float2 lds[16];
  // WAVE: gamma and beta, then [teams - 1][lanes * R * VW] sums
  extern __shared__ __attribute__((aligned(16))) float kept[];
  const int lanes = 1 << a.lanes_log2, l = threadIdx.x & (lanes - 1);
  const int teams = a.threads >> a.lanes_log2, team = threadIdx.x >> a.lanes_log2;
  float2* const sums = (float2*)kept;
  const float inv = 1.f / (float)a.c;
  const Lanes<VW, R, FILL> of(a, l);
  float dg[R][VW] = {}, db[R][VW] = {};
  const Params<VW, WAVE> params(a, kept);
  by_act(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    const long long step = (long long)gridDim.x * teams;
    long long r = (long long)blockIdx.x * teams + team;
    Pack<T, VW> f[R] = {}, d[R] = {};
    float2 st = make_float2(0.f, 0.f);
    const auto load = [&](long long row) {
      of.load((const T*)a.x + row * a.c, f);
      of.load((const T*)a.dy + row * a.c, d);
      st = ((const float2*)a.stats)[row];
    };
    if (r < a.rows) load(r);
    for (; r < a.rows; r += step) {
      float xh[R][VW], t[R][VW];
      float2 s = make_float2(0.f, 0.f);
      const float rstd = st.y;
      asm volatile("" ::: "memory");  // (gamma and beta stay where they are)
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW], w[VW], g[VW], b[VW];
        params.read(a, of.q[k].at, g, b);
        unpack<T, VW>(f[k], v);
        unpack<T, VW>(d[k], w);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          float dz;
          layer_dz<ACT, T>(v[e], w[e], {st.x, st.y, g[e], b[e]}, xh[k][e], dz);
          t[k][e] = dz * g[e];
          if (!of.counts(k, e)) continue;
          s.x += t[k][e];
          s.y += t[k][e] * xh[k][e];
          db[k][e] += dz;
          dg[k][e] += dz * xh[k][e];
        }
      }
      if (r + step < a.rows) load(r + step);
      s = row_sums(s, a.lanes_log2, lds);
      // dx = rstd (t - s.x / c - xh s.y / c)
      const float c0 = -rstd * (s.x * inv), c1 = -rstd * (s.y * inv);
      T* out = (T*)a.out + r * a.c;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW];
#pragma unroll
        for (int e = 0; e < VW; ++e) v[e] = fmaf(xh[k][e], c1, fmaf(t[k][e], rstd, c0));
        if (of.in(k)) store_run<T, VW>(out + of.q[k].at, pack<T, VW>(v), a.stream);
      }
    }
  });
  if (!a.part) return;
  if (teams > 1) __syncthreads();  // (gamma and beta have been read)
  float2* mine = sums + (team - 1) * lanes * R * VW;
  if (team > 0) {
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int e = 0; e < VW; ++e)
        mine[(k * VW + e) * lanes + l] = make_float2(db[k][e], dg[k][e]);
  }
  if (teams > 1) __syncthreads();
  if (team > 0) return;
  float2* part = a.part + (size_t)blockIdx.x * a.c;
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      float2 s = make_float2(db[k][e], dg[k][e]);
      for (int t = 0; t < teams - 1; ++t) {
        const float2 v = sums[(t * R * VW + k * VW + e) * lanes + l];
        s.x += v.x;
        s.y += v.y;
      }
      if (of.counts(k, e)) part[of.q[k].at + e] = s;
    }
}

// Rows of any length (over 32 or 16 channels a thread of the largest workgroup), a workgroup
// each, read again for each of the sums and the result, from the caches as far as those hold the
// rows in work: 1024 rows of 32768 bf16 36 us, 134 MB at 3.7 TB/s, the gradient 48 and 27 of
// layer_long_sums_kernel.
template <typename T, int VW, bool RAGGED, bool GRAD>
__global__ __launch_bounds__(1024) void layer_long_kernel(LayerArgs a) {
  __shared__ float2 lds[16];
  const float inv = 1.f / (float)a.c;
  const long long step = (long long)blockDim.x * VW;
  by_act(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
      const T* x = (const T*)a.x + r * a.c;
      const T* dy = (const T*)a.dy + r * a.c;
      T* out = (T*)a.out + r * a.c;
      const auto each = [&](auto&& f) {
        for (long long i = (long long)threadIdx.x * VW; i < a.c; i += step) {
          const Piece q = piece<VW, RAGGED>(i, a.c);
          float v[VW], w[VW] = {};
          unpack<T, VW>(load_run<T, VW>(x + q.at), v);
          if constexpr (GRAD) unpack<T, VW>(load_run<T, VW>(dy + q.at), w);
          f(q, v, w);
        }
      };
      if constexpr (!GRAD) {
        float2 s = make_float2(0.f, 0.f);
        each([&](const Piece& q, float (&v)[VW], float (&)[VW]) {
#pragma unroll
          for (int e = 0; e < VW; ++e)
            if (!RAGGED || e >= q.skip) s.x += v[e];
        });
        const float mean = row_sums(s, 10, lds).x * inv;
        s = make_float2(0.f, 0.f);
        each([&](const Piece& q, float (&v)[VW], float (&)[VW]) {
#pragma unroll
          for (int e = 0; e < VW; ++e)
            if (!RAGGED || e >= q.skip) s.x += (v[e] - mean) * (v[e] - mean);
        });
        const float rstd = 1.f / sqrtf(row_sums(s, 10, lds).x * inv + a.eps);
        each([&](const Piece& q, float (&v)[VW], float (&)[VW]) {
          float g[VW], b[VW];
          vector_params<VW>(a, q.at, g, b);
#pragma unroll
          for (int e = 0; e < VW; ++e)
            v[e] = norm_value<false, ACT, T>(v[e], 0.f, {mean, rstd, g[e], b[e]},
                                             make_float2(0.f, 0.f));
          store_run<T, VW>(out + q.at, pack<T, VW>(v), a.stream);
        });
        if (a.stats_out && threadIdx.x == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
      } else {
        const float2 st = ((const float2*)a.stats)[r];
        float2 s = make_float2(0.f, 0.f);
        each([&](const Piece& q, float (&v)[VW], float (&w)[VW]) {
          float g[VW], b[VW];
          vector_params<VW>(a, q.at, g, b);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            if (RAGGED && e < q.skip) continue;
            float xh, dz;
            layer_dz<ACT, T>(v[e], w[e], {st.x, st.y, g[e], b[e]}, xh, dz);
            s.x += dz * g[e];
            s.y += dz * g[e] * xh;
          }
        });
        s = row_sums(s, 10, lds);
        s.x *= inv, s.y *= inv;
        each([&](const Piece& q, float (&v)[VW], float (&w)[VW]) {
          float g[VW], b[VW];
          vector_params<VW>(a, q.at, g, b);
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            float xh, dz;
            layer_dz<ACT, T>(v[e], w[e], {st.x, st.y, g[e], b[e]}, xh, dz);
            v[e] = st.y * (dz * g[e] - s.x - xh * s.y);
          }
          store_run<T, VW>(out + q.at, pack<T, VW>(v), a.stream);
        });
      }
    }
  });
}

// dgamma and dbeta of long rows: a workgroup has 256 vectors of channels and every
// gridDim.y-th row.
template <typename T, int VW, bool RAGGED>
__global__ __launch_bounds__(256) void layer_long_sums_kernel(LayerArgs a) {
  const Piece q = piece<VW, RAGGED>(((long long)blockIdx.x * 256 + threadIdx.x) * VW, a.c);
  if (!q.in) return;
  by_act(a.act, [&](auto act) {
    float g[VW], b[VW], dg[VW] = {}, db[VW] = {};
    vector_params<VW>(a, q.at, g, b);
    for (long long r = blockIdx.y; r < a.rows; r += gridDim.y) {
      float v[VW], w[VW];
      unpack<T, VW>(load_run<T, VW>((const T*)a.x + r * a.c + q.at), v);
      unpack<T, VW>(load_run<T, VW>((const T*)a.dy + r * a.c + q.at), w);
      const float2 st = ((const float2*)a.stats)[r];
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        float xh, dz;
        layer_dz<decltype(act)::value, T>(v[e], w[e], {st.x, st.y, g[e], b[e]}, xh, dz);
        db[e] += dz;
        dg[e] += dz * xh;
      }
    }
#pragma unroll
    for (int e = 0; e < VW; ++e)
      if (!RAGGED || e >= q.skip)
        a.part[(size_t)blockIdx.y * a.c + q.at + e] = make_float2(db[e], dg[e]);
  });
}

// dgamma and dbeta from the workgroups' sums, 2^cols_log2 channels side by side.  Bound by launch
// and latency: 4 channels of fewer than 1024 (983 sums of 128 channels 3.9 us, 6.9 by 16), 16 of
// more, whose lines 4 would read four times (491 of 1024 4.7 us either way, of 2048 5.2 and 7.2,
// 256 of 16384 7.5 and 22.9).
__global__ __launch_bounds__(1024) void layer_params_kernel(LayerArgs a, int cols_log2) {
  __shared__ float2 lds[16][16];
  const int cols = 1 << cols_log2, col = threadIdx.x & (cols - 1), row = threadIdx.x >> cols_log2;
  const int ch = (blockIdx.x << cols_log2) + col, rows = 1024 >> cols_log2;
  float2 s = make_float2(0.f, 0.f);
  if (ch < a.c) {
#pragma unroll 16
    for (int r = row; r < a.parts; r += rows) {
      const float2 v = a.part[(size_t)r * a.c + ch];
      s.x += v.x;
      s.y += v.y;
    }
  }
  for (int m = cols; m < 64; m <<= 1) {
    s.x += __shfl_xor(s.x, m);
    s.y += __shfl_xor(s.y, m);
  }
  if ((int)(threadIdx.x & 63) < cols) lds[threadIdx.x >> 6][col] = s;
  __syncthreads();
  if ((int)threadIdx.x >= cols || ch >= a.c) return;
  s = lds[0][col];
  for (int w = 1; w < 16; ++w) {
    s.x += lds[w][col].x;
    s.y += lds[w][col].y;
  }
  if (a.dbeta) a.dbeta[ch] = s.x;
  if (a.dgamma) a.dgamma[ch] = s.y;
}

hipError_t launch_layer_params(const LayerArgs& a, hipStream_t stream) {
  const int log2 = a.c < 1024 ? 2 : 4;
  if (a.part)
    hipLaunchKernelGGL(layer_params_kernel, dim3((unsigned)((a.c + (1ll << log2) - 1) >> log2)),
                       dim3(1024), 0, stream, a, log2);
  return hipGetLastError();
}

namespace {

template <typename T, int VW, bool RAGGED>
void launch_long(const LayerArgs& a, bool grad, hipStream_t stream) {
  if (!grad) {
    hipLaunchKernelGGL((layer_long_kernel<T, VW, RAGGED, false>), dim3(a.groups), dim3(1024), 0,
                       stream, a);
    return;
  }
  hipLaunchKernelGGL((layer_long_kernel<T, VW, RAGGED, true>), dim3(a.groups), dim3(1024), 0,
                     stream, a);
  if (a.part)
    hipLaunchKernelGGL((layer_long_sums_kernel<T, VW, RAGGED>),
                       dim3((a.c + 256 * VW - 1) / (256 * VW), a.parts), dim3(256), 0, stream, a);
}

template <typename T, int VW, int R, int FILL>
void launch_held(const LayerArgs& a, bool grad, hipStream_t stream) {
  const int teams = a.threads >> a.lanes_log2;
  // gamma and beta; then sums of all teams but one
  const int params = (a.c + 3) / 4 * 4 * (int)sizeof(float2);
  const int lds = std::max(params, (teams - 1) * R * VW * (int)sizeof(float2) << a.lanes_log2);
  constexpr bool kWide = R * VW == kLayerWideChannels;  // teams of waves have no others
  if (a.lanes_log2 <= 6) {
    if (!grad)
      hipLaunchKernelGGL((layer_rows_kernel<T, VW, R, FILL, true>), dim3(a.groups),
                         dim3(a.threads), params, stream, a);
    else if constexpr (R * VW <= kLayerGradChannels)
      hipLaunchKernelGGL((layer_grad_rows_kernel<T, VW, R, FILL, true>), dim3(a.groups),
                         dim3(a.threads), lds, stream, a);
  } else if constexpr (kWide) {
    if (!grad)
      hipLaunchKernelGGL((layer_rows_kernel<T, VW, R, FILL, false>), dim3(a.groups),
                         dim3(a.threads), 0, stream, a);
    else
      hipLaunchKernelGGL((layer_grad_rows_kernel<T, VW, R, FILL, false>), dim3(a.groups),
                         dim3(a.threads), 0, stream, a);
  }
}

template <typename T, int VW, int FILL>
void launch_rows(const LayerArgs& a, bool grad, hipStream_t stream) {
  switch (a.slots) {
    case 0: return launch_long<T, VW, FILL == kRagged>(a, grad, stream);
    case 1: return launch_held<T, VW, 1, FILL>(a, grad, stream);
    case 2: return launch_held<T, VW, 2, FILL>(a, grad, stream);
    case 4: return launch_held<T, VW, 4, FILL>(a, grad, stream);
    default:
      if constexpr (VW == 4) launch_held<T, VW, 8, FILL>(a, grad, stream);
  }
}

template <typename T>
void launch_type(const LayerArgs& a, int vec, bool grad, hipStream_t stream) {
  constexpr int kVec = 16 / (int)sizeof(T);
  if (vec == 1)
    launch_held<T, 1, 1, kPart>(a, grad, stream);
  else if (a.c % kVec)
    launch_rows<T, kVec, kRagged>(a, grad, stream);
  else if (a.slots == 0 || a.c != kVec * a.slots << a.lanes_log2)
    launch_rows<T, kVec, kPart>(a, grad, stream);
  else
    launch_rows<T, kVec, kFull>(a, grad, stream);
}

}  // namespace

hipError_t launch_layer_rows(const LayerArgs& a, int dtype, int vec, bool grad,
                             hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    launch_type<uint16_t>(a, vec, grad, stream);
  else
    launch_type<uint32_t>(a, vec, grad, stream);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !grad ? e : launch_layer_params(a, stream);
}

}  // namespace huge2
