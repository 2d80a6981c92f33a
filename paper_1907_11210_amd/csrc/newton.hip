// newton.hip -- orthogonalised matrices by Newton-Schulz products (huge2_train.h).
//
// A step takes X (m x n, m <= n, no singular value above its bound) to a X + b A X + c A A X
// with A = X X^T: three products, of which the first two are symmetric and half of their tiles
// are computed.  The products take fp16 operands times powers of two, sums are fp32.
//
// Two parts a value, hi + lo, are 22 bits, and hi hi + hi lo + lo hi gives fp32's accuracy: after
// five steps 4e-7 of the result's norm against 2e-7 for products in fp32, and 4e-6 against 2e-6
// where singular values fall with the square of their rank.
//
// One part is 11 bits.  Two things keep its error below 7e-4 of the result's norm, whatever the
// singular values (2e-3 and, for steep ones, 2e-2 without them; bf16 1e-2 and 0.15).  The term
// a X, which carries what small singular values grow from, is formed from both parts.  And A is
// stored less mu I, mu the mean of its diagonal, which in the last steps is near 1 and would
// round off what the other elements hold: with A = A' + mu I,
//   a I + b A + c A A = (a + b mu + c mu^2) I + B,  B = (b + 2 c mu) A' + c A' A'.
#include "huge2_train.h"
#include "newton.hpp"
#include "train_device.hpp"

namespace huge2 {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane from global memory to LDS, lane after lane.
__device__ __forceinline__ void load_to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// All of this wave's loads into LDS have arrived and its reads have been taken, in all waves.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct Parts4 {
  half4 hi, lo;
};
__device__ __forceinline__ Parts4 split4(const float (&v)[4]) {
  Parts4 p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    p.hi[e] = (_Float16)v[e];
    p.lo[e] = (_Float16)(v[e] - (float)p.hi[e]);
  }
  return p;
}

// Four lanes side by side, four values each: lane q gets the q-th of each of them.
__device__ __forceinline__ half4 transpose4(half4 v) {
  const uint2 u = __builtin_bit_cast(uint2, v);
  const int q = threadIdx.x & 3;
  const uint32_t pick = q & 1 ? 0x07060302u : 0x05040100u;
  uint32_t s[4];
#define HUGE2_LANE(i)                                                                         \
  {                                                                                           \
    const uint32_t x = __builtin_amdgcn_update_dpp(0, (int)u.x, (i) * 0x55, 0xf, 0xf, true);  \
    const uint32_t y = __builtin_amdgcn_update_dpp(0, (int)u.y, (i) * 0x55, 0xf, 0xf, true);  \
    s[i] = q < 2 ? x : y;                                                                     \
  }
  HUGE2_LANE(0) HUGE2_LANE(1) HUGE2_LANE(2) HUGE2_LANE(3)
#undef HUGE2_LANE
  const uint2 r = make_uint2(__builtin_amdgcn_perm(s[1], s[0], pick),
                             __builtin_amdgcn_perm(s[3], s[2], pick));
  return __builtin_bit_cast(half4, r);
}

__device__ __forceinline__ float block_total(float v, float* lds) {
  v = lanes_sum(v, 1);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// The update of element i: the input, or the momentum's (m: the new one).
__device__ __forceinline__ float update(const NsInput& a, float g, float m) {
  return !a.muon ? g : a.nesterov ? a.momentum * m + a.rest * g : m;
}
__device__ __forceinline__ float input(const void* p, int bf16, long long i) {
  return bf16 ? to_f32<uint16_t>(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}

}  // namespace

// The momentum's update, and sums of squares of what is orthogonalised.  In 64 bits: squares
// of any two floats' sum neither overflow nor vanish.
__global__ __launch_bounds__(256) void ns_norm_kernel(NsInput a) {
  __shared__ double lds[4];
  const uint2 work = a.works[blockIdx.x];
  const NsMatrix t = a.mats[work.x];
  const void* src = a.src[work.x];
  if (!src) return;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const long long first = (long long)work.y * t.norm_chunk;
  const long long end = min(first + t.norm_chunk, t.count);
  double s = 0;
  for (long long i = first + threadIdx.x; i < end; i += 256) {
    const float g = input(src, t.grad_bf16, i) * gs;
    float m = 0.f;
    if (a.muon) {
      m = a.momentum * t.momentum[i] + a.rest * g;
      t.momentum[i] = m;
    }
    const double u = update(a, g, m);
    s += u * u;
  }
  for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) t.norm[work.y] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// X = U / (norm + eps) and its transpose as fragments, a block of 64 x 64 of the input to a
// workgroup.
template <int PARTS>
__global__ __launch_bounds__(256) void ns_pack_kernel(NsInput a) {
  __shared__ float tile[kNsBlock][kNsBlock + 1];
  __shared__ double sums[4];
  const uint2 work = a.works[blockIdx.x];
  const NsMatrix t = a.mats[work.x];
  const void* src = a.src[work.x];
  if (!src) return;
  double s = 0;
  for (int i = threadIdx.x; i < t.norm_count; i += 256) s += t.norm[i];
  for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  const double inv = 1.0 / (sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + a.eps);
  const int rows = t.tall ? t.n : t.m, cols = t.tall ? t.m : t.n;
  const int across = (t.tall ? t.mp : t.np) / kNsBlock;
  const int r0 = (int)(work.y / across) * kNsBlock, c0 = (int)(work.y % across) * kNsBlock;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 4
  for (int r = wave; r < kNsBlock; r += 4) {
    float v = 0.f;
    if (r0 + r < rows && c0 + lane < cols) {
      const long long i = (long long)(r0 + r) * cols + c0 + lane;
      const float g = input(src, t.grad_bf16, i) * gs;
      v = (float)(update(a, g, a.muon ? t.momentum[i] : 0.f) * inv);
    }
    tile[r][lane] = v * a.out_scale;
  }
  __syncthreads();
  // pieces of 8 elements of a fragment's row: two orientations, 64 rows, 8 pieces a row
  half_bits* const to[2] = {t.tall ? t.t0 : t.x, t.tall ? t.x : t.t0};
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const int depth = (o == 0) == (t.tall == 0) ? t.np : t.mp;  // columns of the fragments' matrix
    const int fr = o == 0 ? r0 : c0, fk = o == 0 ? c0 : r0;
    const bool second = PARTS == 2 || to[o] == t.t0;
#pragma unroll
    for (int p = threadIdx.x; p < 64 * 8; p += 256) {
      // (a fragment's rows side by side: 32 pieces of 16 bytes)
      const int r = (p & 31) | (p >> 8) << 5, k = (p >> 5 & 7) * 8;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = o == 0 ? tile[r][k + e] : tile[k + e][r];
      half8 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        hi[e] = (_Float16)v[e];
        lo[e] = (_Float16)(v[e] - (float)hi[e]);
      }
      const int kk = fk + k;
      const size_t at = ((size_t)((fr + r) / 32) * (depth / 16) + kk / 16) * kNsFrag +
                        (kk / 8 & 1) * 256 + (r & 31) * 8;
      *(half8*)(to[o] + at) = hi;
      if (second) *(half8*)(to[o] + (size_t)t.mp * t.np + at) = lo;
    }
  }
}

namespace {

// A tile of SIZE x SIZE of a product P Q^T by four waves, each a quarter.
template <int PARTS, int SIZE>
struct Product {
  static constexpr int kStage = ns_stage(PARTS), kWave = SIZE / 2, kBlocks = kWave / 32;
  static constexpr int kFrags = kStage / 16;                 // of a stage and row of fragments
  static constexpr int kRows = SIZE / 32;                    // rows of fragments of P, of Q
  static constexpr int kStageFrags = 2 * kRows * kFrags * PARTS;
  static constexpr int kBytes = kStageFrags * 1024;
  typedef f32x16 Acc[kBlocks][kBlocks];

  // Stage s: fragments [P, Q][row][column][part] in LDS.
  static __device__ __forceinline__ void issue(const half_bits* const (&op)[2],
                                               const size_t (&plane)[2], const int (&row0)[2],
                                               const int (&rows)[2], int depth, int s, char* lds) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < kStageFrags / 4; ++i) {
      const int f = i * 4 + wave, part = f % PARTS, col = f / PARTS % kFrags;
      const int row = f / PARTS / kFrags % kRows, side = f / PARTS / kFrags / kRows;
      // (rows behind the end: the last once more, for results that are not stored)
      const int r = min(row0[side] + row, rows[side] - 1);
      const half_bits* from = op[side] + part * plane[side] +
                              ((size_t)r * (depth / 16) + s * kFrags + col) * kNsFrag + lane * 8;
      load_to_lds(from, lds + f * 1024);
    }
  }

  static __device__ __forceinline__ void multiply(const char* lds, Acc& acc) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wi = wave >> 1, wj = wave & 1;
#pragma unroll
    for (int k = 0; k < kFrags; ++k) {
      half8 p[kBlocks][PARTS], q[kBlocks][PARTS];
#pragma unroll
      for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int h = 0; h < PARTS; ++h) {
          const auto at = [&](int row) { return ((row * kFrags + k) * PARTS + h) * 1024 + lane * 16; };
          p[i][h] = *(const half8*)(lds + at(wi * kBlocks + i));
          q[i][h] = *(const half8*)(lds + at(kRows + wj * kBlocks + i));
        }
#pragma unroll
      for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[i][0], q[j][0], acc[i][j], 0, 0, 0);
          if constexpr (PARTS == 2) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[i][0], q[j][1], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[i][1], q[j][0], acc[i][j], 0, 0, 0);
          }
        }
    }
  }

  static __device__ __forceinline__ void run(const NsArgs& a, const NsMatrix& t, const NsWork& w,
                                             char* lds, Acc& acc) {
    const half_bits* const op[2] = {a.kind == kNsGram ? t.x : a.kind == kNsSquare ? t.a : t.b,
                                    a.kind == kNsGram ? t.x : a.kind == kNsSquare ? t.a
                                    : a.from               ? t.t1
                                                           : t.t0};
    const int depth = a.kind == kNsGram ? t.np : t.mp;
    const size_t square = (size_t)t.mp * t.mp, whole = (size_t)t.mp * t.np;
    const size_t plane[2] = {a.kind == kNsGram ? whole : square,
                             a.kind == kNsSquare ? square : whole};
    const int row0[2] = {w.ti * kRows, w.tj * kRows};
    const int rows[2] = {t.mp / 32, (a.kind == kNsApply ? t.np : t.mp) / 32};
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    issue(op, plane, row0, rows, depth, w.k0, lds);
    for (int s = w.k0; s < w.k1; ++s) {
      stage_barrier();
      char* const now = lds + (s - w.k0 & 1) * kBytes;
      char* const next = lds + (s - w.k0 + 1 & 1) * kBytes;
      if (s + 1 < w.k1) issue(op, plane, row0, rows, depth, s + 1, next);
      multiply(now, acc);
    }
  }

  // Partial sums lie as the threads hold them.
  static __device__ __forceinline__ void store_part(float* part, int slot, const Acc& acc) {
    float* to = part + (size_t)slot * kNsSlot + threadIdx.x * 4;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(float4*)(to + ((i * kBlocks + j) * 4 + g) * 1024) =
              make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                          acc[i][j][4 * g + 3]);
  }
  static __device__ __forceinline__ void load_parts(const float* part, int slot, int slots,
                                                    Acc& acc) {
    const float* from = part + (size_t)slot * kNsSlot + threadIdx.x * 4;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int k = 0; k < slots; ++k) {
            const float4 v =
                *(const float4*)(from + (size_t)k * kNsSlot + ((i * kBlocks + j) * 4 + g) * 1024);
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
          }
          acc[i][j][4 * g] = s.x, acc[i][j][4 * g + 1] = s.y;
          acc[i][j][4 * g + 2] = s.z, acc[i][j][4 * g + 3] = s.w;
        }
  }

  // Four elements of a lane, at rows i to i + 3 and column j of the tile's matrix: where they lie
  // in its transpose's fragments (`depth` columns), and after transpose4 in its own.
  static __device__ __forceinline__ size_t across(int i, int j, int depth) {
    return ((size_t)(j / 32) * (depth / 16) + i / 16) * kNsFrag + (i / 8 & 1) * 256 + (j & 31) * 8 +
           (i & 4);
  }
  static __device__ __forceinline__ size_t along(int i, int j, int depth) {
    const int r = i + (j & 3), k = j & ~3;
    return ((size_t)(r / 32) * (depth / 16) + k / 16) * kNsFrag + (k / 8 & 1) * 256 + (r & 31) * 8 +
           (k & 4);
  }
  static __device__ __forceinline__ void put(half_bits* to, size_t at, half4 v) {
    *(half4*)(to + at) = v;
  }

  static __device__ __forceinline__ void finish(const NsArgs& a, const NsMatrix& t,
                                                const NsWork& w, float* lds, Acc& acc) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i0 = w.ti * SIZE + (wave >> 1) * kWave + (lane >> 5) * 4;
    const int j0 = w.tj * SIZE + (wave & 1) * kWave + (lane & 31);
    const size_t square = (size_t)t.mp * t.mp, whole = (size_t)t.mp * t.np;
    float mu;
    if (a.kind == kNsGram) {
      mu = 1.f / (float)t.m;  // (any value would do: in the first step X has norm 1)
      if (a.step > 0) {
        float s = 0.f;
        for (int i = threadIdx.x; i < t.x_tiles; i += 256) s += t.squares[i];
        mu = block_total(s, lds) / (float)t.m;
      }
      if (w.ti == 0 && w.tj == 0 && threadIdx.x == 0) *t.mu = mu;
    } else {
      mu = *t.mu;
    }
    const float linear = a.b + 2.f * a.c * mu, constant = a.a + mu * (a.b + mu * a.c);
    float squares = 0.f;
#pragma unroll
    for (int bi = 0; bi < kBlocks; ++bi) {
#pragma unroll
      for (int bj = 0; bj < kBlocks; ++bj) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int i = i0 + bi * 32 + g * 8, j = j0 + bj * 32;
          if (i >= t.mp || j >= (a.kind == kNsApply ? t.np : t.mp)) continue;  // whole blocks
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[bi][bj][4 * g + e] * a.in_scale;
          if (a.kind == kNsGram) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (i + e == j && j < t.m) v[e] -= mu;
              v[e] *= a.out_scale;
            }
            const Parts4 p = split4(v);
            const size_t to = along(i, j, t.mp);
            put(t.a, to, transpose4(p.hi));
            put(t.a + square, to, transpose4(p.lo));
            if (w.ti != w.tj) {
              put(t.a, across(i, j, t.mp), p.hi);
              put(t.a + square, across(i, j, t.mp), p.lo);
            }
          } else if (a.kind == kNsSquare) {
            const size_t at = across(i, j, t.mp);  // (A is symmetric)
            const half4 hi = *(const half4*)(t.a + at), lo = *(const half4*)(t.a + square + at);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = (a.c * v[e] + linear * (((float)hi[e] + (float)lo[e]) * a.own_scale)) *
                     a.out_scale;
            const Parts4 p = split4(v);
            const size_t to = along(i, j, t.mp);
            put(t.b, to, transpose4(p.hi));
            if (PARTS == 2) put(t.b + square, to, transpose4(p.lo));
            if (w.ti != w.tj) {
              put(t.b, at, p.hi);
              if (PARTS == 2) put(t.b + square, at, p.lo);
            }
          } else {
            const size_t at = across(i, j, t.mp);
            const half_bits* own = a.from ? t.t1 : t.t0;
            const half4 hi = *(const half4*)(own + at), lo = *(const half4*)(own + whole + at);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] += constant * (((float)hi[e] + (float)lo[e]) * a.own_scale);
            if (!a.last) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                squares += v[e] * v[e];
                v[e] *= a.out_scale;
              }
              const Parts4 p = split4(v);
              const size_t to = along(i, j, t.np);
              put(t.x, to, transpose4(p.hi));
              if (PARTS == 2) put(t.x + whole, to, transpose4(p.lo));
              put((a.from ? t.t0 : t.t1), at, p.hi);
              put((a.from ? t.t0 : t.t1) + whole, at, p.lo);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (i + e < t.m && j < t.n) result(a, t, i + e, j, v[e]);
            }
          }
        }
      }
    }
    if (a.kind == kNsApply && !a.last) {
      squares = block_total(squares, lds);
      if (threadIdx.x == 0) {
        const int across_tiles = (t.np + SIZE - 1) / SIZE;
        t.squares[w.ti * across_tiles + w.tj] = squares;
      }
    }
  }

  static __device__ __forceinline__ void result(const NsArgs& a, const NsMatrix& t, int i, int j,
                                                float v) {
    const long long at = t.tall ? (long long)j * t.m + i : (long long)i * t.n + j;
    if (a.out) {
      if (t.bf16)
        ((uint16_t*)a.out)[t.out_at + at] = f32_to_bf16_rne(v);
      else
        ((float*)a.out)[t.out_at + at] = v;
      return;
    }
    const float p = input(t.param, t.bf16, at);
    const float r = p * (1.f - a.lr * t.decay) - a.lr * t.scale * v;
    if (t.bf16)
      ((uint16_t*)t.param)[at] = f32_to_bf16_rne(r);
    else
      ((float*)t.param)[at] = r;
    if (t.copy) ((uint16_t*)t.copy)[at] = f32_to_bf16_rne(r);
  }
};

}  // namespace

template <int PARTS>
__global__ __launch_bounds__(256, 2) void ns_product_kernel(NsArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const NsWork w = a.works[blockIdx.x];
  if (a.skip[w.matrix >> 6] >> (w.matrix & 63) & 1) return;
  const NsMatrix t = a.mats[w.matrix];
  const auto tile = [&](auto product) {
    typedef decltype(product) Of;
    typename Of::Acc acc;
    Of::run(a, t, w, lds, acc);
    if (w.slot >= 0) {
      Of::store_part(a.part, w.slot, acc);
    } else {
      __syncthreads();
      Of::finish(a, t, w, (float*)lds, acc);
    }
  };
  if (w.size)
    tile(Product<PARTS, kNsLarge>());
  else
    tile(Product<PARTS, kNsSmall>());
}

// Adds up the partial tiles, in their order.
template <int PARTS>
__global__ __launch_bounds__(256) void ns_join_kernel(NsArgs a) {
  __shared__ float lds[4];
  const NsWork w = a.works[blockIdx.x];
  if (a.skip[w.matrix >> 6] >> (w.matrix & 63) & 1) return;
  const NsMatrix t = a.mats[w.matrix];
  const auto tile = [&](auto product) {
    typedef decltype(product) Of;
    typename Of::Acc acc;
    Of::load_parts(a.part, w.slot, w.slots, acc);
    Of::finish(a, t, w, lds, acc);
  };
  if (w.size)
    tile(Product<PARTS, kNsLarge>());
  else
    tile(Product<PARTS, kNsSmall>());
}

hipError_t launch_ns_norm(const NsInput& a, unsigned works, hipStream_t stream) {
  hipLaunchKernelGGL(ns_norm_kernel, dim3(works), dim3(256), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_ns_pack(const NsInput& a, unsigned works, int parts, hipStream_t stream) {
  hipLaunchKernelGGL(parts == 2 ? ns_pack_kernel<2> : ns_pack_kernel<1>, dim3(works), dim3(256), 0,
                     stream, a);
  return hipGetLastError();
}
hipError_t launch_ns_product(const NsArgs& a, unsigned works, int parts, hipStream_t stream) {
  const int lds = 2 * (parts == 2 ? Product<2, kNsLarge>::kBytes : Product<1, kNsLarge>::kBytes);
  hipLaunchKernelGGL(parts == 2 ? ns_product_kernel<2> : ns_product_kernel<1>, dim3(works),
                     dim3(256), lds, stream, a);
  return hipGetLastError();
}
hipError_t launch_ns_join(const NsArgs& a, unsigned works, int parts, hipStream_t stream) {
  hipLaunchKernelGGL(parts == 2 ? ns_join_kernel<2> : ns_join_kernel<1>, dim3(works), dim3(256), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace huge2
