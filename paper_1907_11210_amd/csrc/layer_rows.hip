// layer_rows.hip -- layer norm of rows of channels: NHWC, lists of tokens, 1x1 maps.
#include "layer_device.hpp"

namespace huge2 {

namespace {

// Sum over the 2^lanes_log2 lanes side by side on a row, in each of them; lds: a float
// for each wave (rows of more than a wave, which are a workgroup's only one).
__device__ __forceinline__ float row_sum(float v, int lanes_log2, float* lds) {
  if (lanes_log2 > 6) return block_sum(v, lds);
  for (int m = (1 << lanes_log2) >> 1; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ float2 row_sums(float2 v, int lanes_log2, float2* lds) {
  for (int m = (1 << min(lanes_log2, 6)) >> 1; m; m >>= 1) {
    v.x += __shfl_xor(v.x, m);
    v.y += __shfl_xor(v.y, m);
  }
  if (lanes_log2 <= 6) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < (int)blockDim.x >> 6; ++w) {
    v.x += lds[w].x;
    v.y += lds[w].y;
  }
  return v;
}

// gamma and beta of a vector's channels.
template <int VW>
__device__ __forceinline__ void vector_params(const LayerArgs& a, int ch, float (&g)[VW],
                                              float (&b)[VW]) {
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    g[e] = a.gamma ? a.gamma[ch + e] : 1.f;
    b[e] = a.beta ? a.beta[ch + e] : 0.f;
  }
}

}  // namespace

// A row is held by 2^lanes_log2 lanes, R vectors each: read once, its mean, the squares
// around it, and the result from registers.  Rows follow each other in a team of lanes,
// which keeps its channels' gamma and beta.
template <typename T, int VW, int R, bool RAGGED>
__global__ __launch_bounds__(1024) void layer_rows_kernel(LayerArgs a) {
  __shared__ float lds[16];
  const int lanes = 1 << a.lanes_log2, l = threadIdx.x & (lanes - 1);
  const int teams = blockDim.x >> a.lanes_log2, team = threadIdx.x >> a.lanes_log2;
  const float inv = 1.f / (float)a.c;
  by_act(a.act, [&](auto act) {
    Piece q[R];
    float g[R][VW], b[R][VW];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      q[k] = piece<VW, RAGGED>((k * lanes + l) * VW, a.c);
      vector_params<VW>(a, q[k].at, g[k], b[k]);
    }
    for (long long r = (long long)blockIdx.x * teams + team; r < a.rows;
         r += (long long)gridDim.x * teams) {
      const T* x = (const T*)a.x + r * a.c;
      Pack<T, VW> f[R] = {};
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (q[k].in) f[k] = load_run<T, VW>(x + q[k].at);
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW];
        unpack<T, VW>(f[k], v);
#pragma unroll
        for (int e = 0; e < VW; ++e)
          if (q[k].in && (!RAGGED || e >= q[k].skip)) s += v[e];
        forget(f[k]);
      }
      const float mean = row_sum(s, a.lanes_log2, lds) * inv;
      s = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW];
        unpack<T, VW>(f[k], v);
#pragma unroll
        for (int e = 0; e < VW; ++e)
          if (q[k].in && (!RAGGED || e >= q[k].skip)) s += (v[e] - mean) * (v[e] - mean);
        forget(f[k]);
      }
      const float rstd = 1.f / sqrtf(row_sum(s, a.lanes_log2, lds) * inv + a.eps);
      T* y = (T*)a.out + r * a.c;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW];
        unpack<T, VW>(f[k], v);
#pragma unroll
        for (int e = 0; e < VW; ++e)
          v[e] = norm_value<false, decltype(act)::value, T>(v[e], 0.f, {mean, rstd, g[k][e], b[k][e]},
                                                            make_float2(0.f, 0.f));
        if (q[k].in) store_run<T, VW>(y + q[k].at, pack<T, VW>(v), a.stream);
      }
      if (a.stats_out && l == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
    }
  });
}

// The gradient by the same rows: x and dy held, the two means, dx from registers.  A thread
// adds up dgamma and dbeta of its channels over the team's rows; the teams' sums are joined
// in LDS, the workgroups' by layer_params_kernel.
template <typename T, int VW, int R, bool RAGGED>
__global__ __launch_bounds__(1024) void layer_grad_rows_kernel(LayerArgs a) {
  __shared__ float2 lds[16];
  extern __shared__ float2 sums[];  // [teams - 1][lanes * R * VW], rows of up to a wave
  const int lanes = 1 << a.lanes_log2, l = threadIdx.x & (lanes - 1);
  const int teams = blockDim.x >> a.lanes_log2, team = threadIdx.x >> a.lanes_log2;
  const float inv = 1.f / (float)a.c;
  Piece q[R];
  float dg[R][VW], db[R][VW];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    q[k] = piece<VW, RAGGED>((k * lanes + l) * VW, a.c);
#pragma unroll
    for (int e = 0; e < VW; ++e) dg[k][e] = db[k][e] = 0.f;
  }
  by_act(a.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    float g[R][VW], b[R][VW];
#pragma unroll
    for (int k = 0; k < R; ++k) vector_params<VW>(a, q[k].at, g[k], b[k]);
    for (long long r = (long long)blockIdx.x * teams + team; r < a.rows;
         r += (long long)gridDim.x * teams) {
      const T* x = (const T*)a.x + r * a.c;
      const T* dy = (const T*)a.dy + r * a.c;
      Pack<T, VW> f[R] = {}, d[R] = {};
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (q[k].in) {
          f[k] = load_run<T, VW>(x + q[k].at);
          d[k] = load_run<T, VW>(dy + q[k].at);
        }
      const float2 st = ((const float2*)a.stats)[r];
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW], w[VW];
        unpack<T, VW>(f[k], v);
        unpack<T, VW>(d[k], w);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          if (!q[k].in || (RAGGED && e < q[k].skip)) continue;
          float xh, dz;
          layer_dz<ACT, T>(v[e], w[e], {st.x, st.y, g[k][e], b[k][e]}, xh, dz);
          const float t = dz * g[k][e];
          s.x += t;
          s.y += t * xh;
          db[k][e] += dz;
          dg[k][e] += dz * xh;
        }
        forget(f[k]);
        forget(d[k]);
      }
      s = row_sums(s, a.lanes_log2, lds);
      s.x *= inv, s.y *= inv;
      T* out = (T*)a.out + r * a.c;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float v[VW], w[VW];
        unpack<T, VW>(f[k], v);
        unpack<T, VW>(d[k], w);
#pragma unroll
        for (int e = 0; e < VW; ++e) {
          float xh, dz;
          layer_dz<ACT, T>(v[e], w[e], {st.x, st.y, g[k][e], b[k][e]}, xh, dz);
          v[e] = st.y * (dz * g[k][e] - s.x - xh * s.y);
        }
        if (q[k].in) store_run<T, VW>(out + q[k].at, pack<T, VW>(v), a.stream);
      }
    }
  });
  if (!a.part) return;
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
      if (q[k].in && (!RAGGED || e >= q[k].skip)) part[q[k].at + e] = s;
    }
}

// Rows of any length, a workgroup each, read again for each of the sums and the result.
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
        const float mean = row_sums(s, 7, lds).x * inv;
        s = make_float2(0.f, 0.f);
        each([&](const Piece& q, float (&v)[VW], float (&)[VW]) {
#pragma unroll
          for (int e = 0; e < VW; ++e)
            if (!RAGGED || e >= q.skip) s.x += (v[e] - mean) * (v[e] - mean);
        });
        const float rstd = 1.f / sqrtf(row_sums(s, 7, lds).x * inv + a.eps);
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
        s = row_sums(s, 7, lds);
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

// dgamma and dbeta from the workgroups' sums: 16 channels, 64 rows of threads.
__global__ __launch_bounds__(1024) void layer_params_kernel(LayerArgs a) {
  __shared__ float2 lds[16][16];
  const int col = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int ch = blockIdx.x * 16 + col;
  float2 s = make_float2(0.f, 0.f);
  if (ch < a.c) {
#pragma unroll 4
    for (int r = row; r < a.parts; r += 64) {
      const float2 v = a.part[(size_t)r * a.c + ch];
      s.x += v.x;
      s.y += v.y;
    }
  }
#pragma unroll
  for (int m = 16; m < 64; m <<= 1) {
    s.x += __shfl_xor(s.x, m);
    s.y += __shfl_xor(s.y, m);
  }
  if ((threadIdx.x & 63) < 16) lds[threadIdx.x >> 6][col] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || ch >= a.c) return;
  s = lds[0][col];
  for (int w = 1; w < 16; ++w) {
    s.x += lds[w][col].x;
    s.y += lds[w][col].y;
  }
  if (a.dbeta) a.dbeta[ch] = s.x;
  if (a.dgamma) a.dgamma[ch] = s.y;
}

hipError_t launch_layer_params(const LayerArgs& a, hipStream_t stream) {
  if (a.part)
    hipLaunchKernelGGL(layer_params_kernel, dim3((a.c + 15) / 16), dim3(1024), 0, stream, a);
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

template <typename T, int VW, int R, bool RAGGED>
void launch_held(const LayerArgs& a, bool grad, hipStream_t stream) {
  const int teams = a.threads >> a.lanes_log2;
  const int lds = (teams - 1) * R * VW * (int)sizeof(float2) << a.lanes_log2;
  if (!grad)
    hipLaunchKernelGGL((layer_rows_kernel<T, VW, R, RAGGED>), dim3(a.groups), dim3(a.threads), 0,
                       stream, a);
  else if constexpr (R * VW <= kLayerGradChannels)
    hipLaunchKernelGGL((layer_grad_rows_kernel<T, VW, R, RAGGED>), dim3(a.groups),
                       dim3(a.threads), lds, stream, a);
}

template <typename T, int VW, bool RAGGED>
void launch_rows(const LayerArgs& a, bool grad, hipStream_t stream) {
  switch (a.slots) {
    case 0: return launch_long<T, VW, RAGGED>(a, grad, stream);
    case 1: return launch_held<T, VW, 1, RAGGED>(a, grad, stream);
    case 2: return launch_held<T, VW, 2, RAGGED>(a, grad, stream);
    case 4: return launch_held<T, VW, 4, RAGGED>(a, grad, stream);
    default:
      if constexpr (VW == 4) launch_held<T, VW, 8, RAGGED>(a, grad, stream);
  }
}

template <typename T>
void launch_type(const LayerArgs& a, int vec, bool grad, hipStream_t stream) {
  constexpr int kFull = 16 / (int)sizeof(T);
  if (vec == 1)
    launch_held<T, 1, 1, false>(a, grad, stream);
  else if (a.c % kFull)
    launch_rows<T, kFull, true>(a, grad, stream);
  else
    launch_rows<T, kFull, false>(a, grad, stream);
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
