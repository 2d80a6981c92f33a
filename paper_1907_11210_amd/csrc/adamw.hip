// adamw.hip -- one AdamW step over many tensors (huge2_train.h).
#include "train.hpp"
#include "train_device.hpp"

namespace huge2 {

namespace {

constexpr float kCodeMax = 448.f;       // largest e4m3 number
constexpr float kCodeMin = 0x1p-9f;     // smallest positive one
constexpr float kTopLeast = 0x1p-100f;  // a block's largest magnitude below this counts as none

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void decode4(uint32_t codes, float scale, float (&f)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  f[0] = lo.x * scale, f[1] = lo.y * scale, f[2] = hi.x * scale, f[3] = hi.y * scale;
}

// Largest magnitude of a wave's 4 x 64 values, as bits: a NaN's bits lie above
// infinity's and those above any number's, so that it is not lost.
__device__ __forceinline__ float wave_top(const float (&f)[4]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
#pragma unroll
  for (int m = 32; m; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  return __uint_as_float(top);
}

// The numbers of four values whose block's largest magnitude is top.
template <bool KEEP>
__device__ __forceinline__ uint32_t encode4(const float (&f)[4], float top, float* scale) {
  const bool none = top < kTopLeast;
  *scale = none ? 0.f : top * (1.f / kCodeMax);
  const float inv = none ? 0.f : kCodeMax / top;
  float c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    c[e] = f[e] * inv;
    if (KEEP && c[e] > 0.f && c[e] < kCodeMin) c[e] = kCodeMin;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
  return (uint32_t)w;
}

// Four elements from element i of an array of n (i a multiple of 4, the array
// 16-byte aligned); zeros behind its end.
template <typename T, bool STREAM = false>
__device__ __forceinline__ void load4(const void* base, long long i, long long n, float (&f)[4]) {
  const T* p = (const T*)base + i;
  if (i + 4 <= n) {
    if constexpr (STREAM)
      unpack<T, 4>(load_stream<T, 4>(p), f);
    else
      unpack<T, 4>(load_pack<T, 4>(p), f);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = i + e < n ? to_f32<T>(p[e]) : 0.f;
  }
}
template <typename T, bool STREAM = false>
__device__ __forceinline__ void store4(void* base, long long i, long long n, const float (&f)[4]) {
  T* p = (T*)base + i;
  if (i + 4 <= n) {
    store_pack<T, 4>(p, pack<T, 4>(f), STREAM);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) store_pack<T, 1>(p + e, pack<T, 1>({f[e]}));
  }
}
__device__ __forceinline__ uint32_t load_codes(const void* base, long long i, long long n) {
  const uint8_t* p = (const uint8_t*)base + i;
  if (i + 4 <= n) return *(const uint32_t*)p;
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < n) w |= (uint32_t)p[e] << (8 * e);
  return w;
}
__device__ __forceinline__ void store_codes(void* base, long long i, long long n, uint32_t w) {
  uint8_t* p = (uint8_t*)base + i;
  if (i + 4 <= n) {
    *(uint32_t*)p = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[e] = (uint8_t)(w >> (8 * e));
  }
}

}  // namespace

// A workgroup updates adam_work consecutive elements of one tensor, each of its
// four waves blocks of 256, four elements a lane, so that a block of 8-bit moments is
// one wave's own and its largest magnitude needs no LDS.  All loads come before the
// first store.
//
// STREAM: fp32 parameters and moments, which nothing reads before the next step, pass
// the caches both ways, and gradients and copies find room there.
//
// Bound by bytes: 134 M fp32 parameters, 28 bytes each, 645 us (5.8 TB/s); with 8-bit
// moments and bf16 gradients and copies 67 M, 197 us (5.4 TB/s).
template <int BITS, bool STREAM>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
  const uint2 work = a.works[blockIdx.x];
  const void* grad = a.grads[work.x];
  if (!grad) return;
  const AdamTensorDev t = a.tensors[work.x];
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float keep = 1.f - a.lr * t.weight_decay;
  const long long first = (long long)work.y * adam_work(BITS) + threadIdx.x * 4;
  constexpr int kIter = adam_work(BITS) / 1024;
  float p[kIter][4], g[kIter][4], m[kIter][4], v[kIter][4];
#pragma unroll
  for (int j = 0; j < kIter; ++j) {
    const long long i = first + j * 1024;
    if (t.bf16)
      load4<uint16_t>(t.param, i, t.count, p[j]);
    else
      load4<uint32_t, STREAM>(t.param, i, t.count, p[j]);
    if (t.grad_bf16)
      load4<uint16_t>(grad, i, t.count, g[j]);
    else
      load4<uint32_t>(grad, i, t.count, g[j]);
    if constexpr (BITS == 32) {
      load4<uint32_t, STREAM>(t.m, i, t.count, m[j]);
      load4<uint32_t, STREAM>(t.v, i, t.count, v[j]);
    } else {
      const bool in = i < t.count;  // a whole wave's block, or none of it, up to the last
      const long long block = i / kAdamBlock;
      decode4(load_codes(t.m, i, t.count), in ? t.m_scale[block] : 0.f, m[j]);
      decode4(load_codes(t.v, i, t.count), in ? t.v_scale[block] : 0.f, v[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j][e] *= v[j][e];
    }
  }
#pragma unroll
  for (int j = 0; j < kIter; ++j) {
    const long long i = first + j * 1024;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float ge = g[j][e] * gs;
      m[j][e] = a.beta1 * m[j][e] + a.rest1 * ge;
      v[j][e] = a.beta2 * v[j][e] + a.rest2 * (ge * ge);
      const float root = sqrtf(v[j][e]);
      p[j][e] = p[j][e] * keep - a.step_size * (m[j][e] / (root * a.root + a.eps));
      if (BITS == 8) v[j][e] = root;
    }
    if (t.bf16)
      store4<uint16_t>(t.param, i, t.count, p[j]);
    else
      store4<uint32_t, STREAM>(t.param, i, t.count, p[j]);
    if (t.copy) store4<uint16_t>(t.copy, i, t.count, p[j]);
    if constexpr (BITS == 32) {
      store4<uint32_t, STREAM>(t.m, i, t.count, m[j]);
      store4<uint32_t, STREAM>(t.v, i, t.count, v[j]);
    } else {
      float ms, vs;
      const uint32_t mc = encode4<false>(m[j], wave_top(m[j]), &ms);
      const uint32_t vc = encode4<true>(v[j], wave_top(v[j]), &vs);
      store_codes(t.m, i, t.count, mc);
      store_codes(t.v, i, t.count, vc);
      if ((threadIdx.x & 63) == 0 && i < t.count) {
        t.m_scale[i / kAdamBlock] = ms;
        t.v_scale[i / kAdamBlock] = vs;
      }
    }
  }
}

hipError_t launch_adamw(const AdamArgs& a, unsigned works, int state_bits, bool past_caches,
                        hipStream_t stream) {
  const auto kernel = state_bits == 8 ? past_caches ? adamw_kernel<8, true> : adamw_kernel<8, false>
                      : past_caches   ? adamw_kernel<32, true>
                                      : adamw_kernel<32, false>;
  hipLaunchKernelGGL(kernel, dim3(works), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace huge2
