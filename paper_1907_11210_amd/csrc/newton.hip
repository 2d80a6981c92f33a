// newton.hip -- orthogonalised matrices by Newton-Schulz products (huge2_train.h).
//
// A step takes X (m x n, m <= n, no singular value above its bound) to a X + b A X + c A A X
// with A = X X^T: three products, of which the first two are symmetric and half of their tiles
// are computed.  The products take fp16 operands times powers of two, sums are fp32.
//
// Two parts a value, hi + lo, are 22 bits, and hi hi + hi lo + lo hi gives fp32's accuracy: after
// five steps 4e-7 of the result's norm (products in fp32 2e-7), 4e-6 (2e-6) where singular values
// fall with the square of their rank, 2e-5 to 5e-4 (4e-6 to 4e-3) where all but a few are nothing
// and what roundings leave in their place grows 480 times.
//
// One part is 11 bits: 7e-4 of the result's norm, of falling singular values 3e-4, of small
// matrices more (16 x 16 2e-3).  Of a matrix of low rank what is left in place of its missing
// singular values is up to 6e-2 of 3 x 3, 3e-2 of 8 x 8, 1e-2 from 32 x 32 on where entries are of
// few sizes and round alike, else 0.25 / m (bf16 products 0.15 and more).  Two things keep it
// there.  The term a X, which carries what small singular values grow from, is formed from both
// parts (else 2e-2 where they fall).  And A is stored less mu I, mu the mean of its diagonal, which
// in the last steps is near 1 and would round off what the other elements hold (else 2e-3): with
// A = A' + mu I,
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
// All but the last LEFT of this wave's loads into LDS have arrived and its reads have been
// taken, and so in all waves.
template <int LEFT>
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// (By value: of two members of a structure the compiler else selects the addresses, and the
// structure goes to scratch memory.)
template <typename T>
__device__ __forceinline__ T pick(bool first, T a, T b) {
  return first ? a : b;
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

// Four from element i, zeros from `end` on.  (A batch's matrices begin at any element.)
__device__ __forceinline__ void input4(const void* p, int bf16, long long i, long long end,
                                       float (&v)[4]) {
  typedef u32x4 u32x4_any __attribute__((aligned(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  typedef u32x2 u32x2_any __attribute__((aligned(2)));
  if (i + 4 <= end) {
    if (bf16) {
      const u32x2 w = *(const u32x2_any*)((const uint16_t*)p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    } else {
      const u32x4 w = *(const u32x4_any*)((const float*)p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = i + e < end ? input(p, bf16, i + e) : 0.f;
  }
}

}  // namespace

// The momentum's update, and sums of squares of what is orthogonalised.  In 64 bits: squares
// of any two floats' sum neither overflow nor vanish.  Bound by the bytes where there are enough:
// 88 M elements of bf16 gradients and fp32 momenta 150 to 156 us, 881 MB at 5.7 to 5.9 TB/s
// (eight vectors in flight 161 us; 48 small matrices 13.5 us, 20.3 with eight).  At most 1024 sums
// of a matrix: with 512 33.6 M bf16 elements took 57 us, now 33 to 35.
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
  constexpr int kAhead = 4;  // vectors of four in flight
  for (long long i = first + threadIdx.x * 4; i < end; i += kAhead * 1024) {
    float g[kAhead][4], m[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      input4(src, t.grad_bf16, i + k * 1024, end, g[k]);
      if (a.muon) input4(t.momentum, 0, i + k * 1024, end, m[k]);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long long at = i + k * 1024;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[k][e] *= gs;
        if (a.muon) m[k][e] = a.momentum * m[k][e] + a.rest * g[k][e];
        const double u = update(a, g[k][e], m[k][e]);
        s += u * u;
      }
      if (!a.muon) continue;
      if (at + 4 <= end) {
        *(float4*)(t.momentum + at) = make_float4(m[k][0], m[k][1], m[k][2], m[k][3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + e < end) t.momentum[at + e] = m[k][e];
      }
    }
  }
  for (int m = 32; m; m >>= 1) s += __shfl_xor(s, m);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) t.norm[work.y] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// X = U / (norm + eps) and its transpose as fragments, a block of 64 x 64 of the input to a
// workgroup.  Bound by the bytes, most of them written, in pieces of 512: of 33.6 M bf16 elements
// 75 us, 337 MB at 4.5 TB/s (with one part 62 us, 269 MB at 4.3); of 88 M and their momenta 241,
// 5.1 TB/s (215, 4.9 TB/s; read by one element a lane instead of four 77 and 355 us with one
// part).  (The products then need no transpose: read by the other axis, a fragment would be 16
// loads of 2 bytes a lane.)
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
  // four neighbours of each fourth of the rows to a thread, all on their way at once
  const int col = (threadIdx.x & 15) * 4, row = threadIdx.x >> 4;
  float g[4][4], m[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = r0 + row + 16 * k;
    const long long first = (long long)r * cols, end = r < rows ? first + cols : 0;
    input4(src, t.grad_bf16, first + c0 + col, end, g[k]);
    if (a.muon) input4(t.momentum, 0, first + c0 + col, end, m[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = (float)(update(a, g[k][e] * gs, a.muon ? m[k][e] : 0.f) * inv);
      tile[row + 16 * k][col + e] = v * a.out_scale;
    }
  __syncthreads();
  // pieces of 8 elements of a fragment's row: two orientations, 64 rows, 8 pieces a row
  half_bits* const to[2] = {pick(t.tall != 0, t.t0, t.x), pick(t.tall != 0, t.x, t.t0)};
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const int depth = (o == 0) == (t.tall == 0) ? t.np : t.mp;  // columns of the fragments' matrix
    const int fr = o == 0 ? r0 : c0, fk = o == 0 ? c0 : r0;
    const bool second = PARTS == 2 || a.keep_lo || to[o] == t.t0;
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

// A tile of a product P Q^T by four waves, each a quarter: KIND's operands, and what becomes of
// the sums.
//
// Bound by the matrix units and the reads of LDS that feed them: of one matrix of 4096x8192 B X
// with two parts, three products each, takes 666 us, 825 GF at 1240 TFLOP/s (large library
// products of fp16 1080), its matrix units busy for 77% of the cycles, without conflicts of LDS
// banks; A, half of the tiles, 358 us and 16 of the join, 1100 TFLOP/s of what is needed; A A 185
// and 9, 1060.  With one part 287 us, 275 GF at 958 TFLOP/s, busy for 55%; 162 and 17, 770; 79
// and 7, 800.  Where matrices are smaller, bound by what the dies' caches fetch, X once as it is
// and once transposed: 48 of 33x700 to 644x89 117 MB and 48 written in the 29 us of B X, 5.7 TB/s;
// 6 of 1000x333 58 MB in 16, 3.6 TB/s, two rounds of tiles.  What made it
// fast on the large matrix: operands stored as fragments, so that loads go straight into LDS and
// reads are 16 bytes a lane side by side; three or four stages on their way and a wait that counts
// them instead of a wait for all; fragments read a stage ahead of their products; the order of
// instructions (below); the epilogue as a loop over blocks (its straight code was read from memory
// once and took longer than the work).
template <int PARTS, int KIND, int SIZE>
struct Product {
  static constexpr NsTile kTile = kNsTiles[SIZE];
  static constexpr bool kGram = KIND == kNsGram, kSquare = KIND == kNsSquare;
  static constexpr bool kApply = KIND == kNsApply || KIND == kNsLast;
  // blocks of 32 x 32 along the sides of a wave's quarter
  static constexpr int kDown = kTile.rows / 64, kRight = kTile.cols / 64;
  static constexpr int kOfWave = kDown * kRight;
  static constexpr int kFrags = kTile.stage / 16 / PARTS;  // of a stage and row of fragments
  static constexpr int kBuffers = kTile.buffers;
  static constexpr int kP = kTile.rows / 32, kQ = kTile.cols / 32;  // rows of fragments
  static constexpr int kStageFrags = (kP + kQ) * kFrags * PARTS;
  static constexpr int kLoads = kStageFrags / 4;  // of a wave and stage
  static constexpr int kBytes = kStageFrags * 1024;
  typedef f32x16 Acc[kOfWave];

  static __device__ __forceinline__ int wave() {
    return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  }

  struct Frags {
    half8 p[kFrags][kDown][PARTS], q[kFrags][kRight][PARTS];
  };
  // Fragments lie in a stage's buffer as [P, Q][row][column][part].
  static __device__ __forceinline__ void read(const char* lds, Frags& f) {
    const int lane = threadIdx.x & 63;
    const auto at = [&](int row, int k, int h) {
      return *(const half8*)(lds + ((row * kFrags + k) * PARTS + h) * 1024 + lane * 16);
    };
#pragma unroll
    for (int k = 0; k < kFrags; ++k)
#pragma unroll
      for (int h = 0; h < PARTS; ++h) {
#pragma unroll
        for (int i = 0; i < kDown; ++i) f.p[k][i][h] = at((wave() >> 1) * kDown + i, k, h);
#pragma unroll
        for (int i = 0; i < kRight; ++i) f.q[k][i][h] = at(kP + (wave() & 1) * kRight + i, k, h);
      }
  }
  static __device__ __forceinline__ void multiply(const Frags& f, Acc& acc) {
#pragma unroll
    for (int k = 0; k < kFrags; ++k) {
      // (the products of one sum apart from each other)
#pragma unroll
      for (int h = 0; h < (PARTS == 2 ? 3 : 1); ++h)
#pragma unroll
        for (int i = 0; i < kDown; ++i)
#pragma unroll
          for (int j = 0; j < kRight; ++j)
            acc[i * kRight + j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                f.p[k][i][h == 2], f.q[k][j][h == 1], acc[i * kRight + j], 0, 0, 0);
    }
  }

  static __device__ __forceinline__ void run(const NsArgs& a, const NsMatrix& t, const NsWork& w,
                                             char* lds, Acc& acc) {
    const int lane = threadIdx.x & 63;
    const half_bits* const t_now = pick(a.from != 0, t.t1, t.t0);
    const half_bits* const b = t.b;
    const bool turn = turned(t);
    const half_bits* const op[2] = {kGram ? t.x : kSquare ? t.a : pick(turn, t_now, b),
                                    kGram ? t.x : kSquare ? t.a : pick(turn, b, t_now)};
    const int depth = (kGram ? t.np : t.mp) / 16;  // columns of fragments
    const size_t square = (size_t)t.mp * t.mp, whole = (size_t)t.mp * t.np;
    const size_t plane[2] = {kGram || turn ? whole : square, kSquare || turn ? square : whole};
    const int rows[2] = {(turn ? t.np : t.mp) / 32, (kApply && !turn ? t.np : t.mp) / 32};
    // a wave's fragments of stage k0
    const half_bits* from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int f = i * 4 + wave(), part = f % PARTS, col = f / PARTS % kFrags;
      const int row = f / PARTS / kFrags;
      const bool second = row >= kP;
      // (rows behind the end: the last once more, for results that are not stored)
      const int r = min(pick(second, w.tj * kQ + row - kP, w.ti * kP + row),
                        pick(second, rows[1], rows[0]) - 1);
      from[i] = pick(second, op[1], op[0]) + part * pick(second, plane[1], plane[0]) +
                ((size_t)r * depth + (size_t)w.k0 * kFrags + col) * kNsFrag;
    }
#pragma unroll
    for (int k = 0; k < kOfWave; ++k)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[k][e] = 0.f;
    // While a stage is multiplied from registers, the next is read from LDS and the ones behind
    // it arrive.  (Behind the last stage it arrives again, so that every wait counts the same
    // loads.)
    const int stages = w.k1 - w.k0;
    int ahead = 0;  // stages whose loads have been issued
    int into = 0;   // the buffer that the next of them goes to
    const auto load = [&] {
      const int step = ahead + 1 < stages ? kFrags * kNsFrag : 0;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        load_to_lds(from[i] + lane * 8, lds + into * kBytes + (i * 4 + wave()) * 1024);
        from[i] += step;
      }
      ++ahead;
      into = into + 1 == kBuffers ? 0 : into + 1;
    };
    Frags f[2];
#pragma unroll
    for (int k = 0; k < kBuffers; ++k) load();
    stage_barrier<(kBuffers - 1) * kLoads>();
    read(lds, f[0]);
    int next_buffer = 1;
    const auto step = [&](Frags& now, Frags& next) {
      stage_barrier<(kBuffers - 2) * kLoads>();
      __builtin_amdgcn_sched_barrier(0);
      read(lds + next_buffer * kBytes, next);
      load();
      multiply(now, acc);
      order();
      __builtin_amdgcn_sched_barrier(0);
      next_buffer = next_buffer + 1 == kBuffers ? 0 : next_buffer + 1;
    };
    int s = 0;
#pragma unroll 1
    for (; s + 2 <= stages; s += 2) {
      step(f[0], f[1]);
      step(f[1], f[0]);
    }
    if (s < stages) step(f[0], f[1]);
    stage_barrier<0>();
  }
  // The order of a stage's instructions: reads and loads between products, which they else delay.
  static __device__ __forceinline__ void order() {
    constexpr int kReads = kFrags * PARTS * (kDown + kRight);
    constexpr int kProducts = kFrags * (PARTS == 2 ? 3 : 1) * kOfWave;
    constexpr int kEach = (kReads + kLoads + kProducts - 1) / kProducts + 1;
    constexpr int kWith = (kReads + kEach - 1) / kEach;  // products followed by reads
    unroll_stages<kProducts>([](auto i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      constexpr int kAt = decltype(i)::value;
      if constexpr (kAt < kWith)
        __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);
      else if constexpr (kAt - kWith < kLoads)
        __builtin_amdgcn_sched_group_barrier(0x010, kLoads > kProducts - kWith ? kLoads : 1, 0);
    });
  }

  // Partial sums lie as the threads hold them.
  static __device__ __forceinline__ void store_part(float* part, int slot, const Acc& acc) {
    float* to = part + slot * kTile.slot() + threadIdx.x * 4;
#pragma unroll
    for (int k = 0; k < kOfWave; ++k)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(float4*)(to + (k * 4 + g) * 1024) = make_float4(acc[k][4 * g], acc[k][4 * g + 1],
                                                          acc[k][4 * g + 2], acc[k][4 * g + 3]);
  }
  // A block's sums over the parts, in their order.
  static __device__ __forceinline__ void load_parts(const float* part, int slot, int slots,
                                                    int block, f32x16& acc) {
    const float* from = part + slot * kTile.slot() + block * 4096 + threadIdx.x * 4;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll 4
    for (int k = 0; k < slots; ++k) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 v = *(const float4*)(from + k * kTile.slot() + g * 1024);
        acc[4 * g] += v.x, acc[4 * g + 1] += v.y, acc[4 * g + 2] += v.z, acc[4 * g + 3] += v.w;
      }
    }
  }

  static __device__ __forceinline__ float mean_square(const NsArgs& a, const NsMatrix& t,
                                                      const NsWork& w, float* lds) {
    if (!kGram) return *t.mu;
    float mu = 1.f / (float)t.m;  // (any value would do: in the first step X has norm 1)
    if (a.step > 0) {
      float s = 0.f;
      for (int i = threadIdx.x; i < t.squares_count; i += 256) s += t.squares[i];
      mu = block_total(s, lds) / (float)t.m;
    }
    if (w.ti == 0 && w.tj == 0 && threadIdx.x == 0) *t.mu = mu;
    return mu;
  }

  // The last step's product is X^T = T B where the input was taken transposed, so that lanes
  // have neighbours of the result's rows.
  static __device__ __forceinline__ bool turned(const NsMatrix& t) {
    return KIND == kNsLast && t.tall;
  }

  // Blocks of 32 x 32: of a tile, by the wave and its number.
  static __device__ __forceinline__ int block_row(const NsWork& w, int k) {
    return w.ti * kP + (wave() >> 1) * kDown + k / kRight;
  }
  static __device__ __forceinline__ int block_column(const NsWork& w, int k) {
    return w.tj * kQ + (wave() & 1) * kRight + k % kRight;
  }
  // (Of a symmetric product a block on or over the diagonal, which is stored twice.)
  static __device__ __forceinline__ bool inside(const NsMatrix& t, int bi, int bj) {
    if (turned(t)) return bi * 32 < t.np && bj * 32 < t.mp;
    return bi * 32 < t.mp && (kApply ? bj * 32 < t.np : bj * 32 < t.mp && bj >= bi);
  }
  // A lane has four elements of each of four groups of rows, at one column.  In the fragments of
  // the block's transpose (`depth` columns of them) they lie at across + 256 g, in its own after
  // transpose4 at along + 64 g.
  static __device__ __forceinline__ half_bits* across(half_bits* p, int bi, int bj, int depth) {
    const int lane = threadIdx.x & 63;
    return p + ((size_t)bj * depth + 2 * bi) * kNsFrag + ((lane & 31) * 8 + (lane >> 5) * 4);
  }
  static __device__ __forceinline__ half_bits* along(half_bits* p, int bi, int bj, int depth) {
    const int lane = threadIdx.x & 63, r = (lane >> 5) * 4 + (lane & 3), k = lane & 28;
    return p + ((size_t)bi * depth + 2 * bj) * kNsFrag +
           ((k >> 4) * kNsFrag + (k >> 3 & 1) * 256 + r * 8 + (k & 4));
  }

  // What is added to a block's sums: A', which is symmetric, or X.
  struct Own {
    half4 hi[4], lo[4];
  };
  static __device__ __forceinline__ void load_own(const NsArgs& a, const NsMatrix& t, int bi,
                                                  int bj, Own& own) {
    if (kGram || !inside(t, bi, bj)) return;
    const size_t plane = (size_t)t.mp * (kSquare ? t.mp : t.np);
    const half_bits* hi = turned(t) ? across(t.x, bi, bj, t.np / 16)
                                    : across(kSquare ? t.a : pick(a.from != 0, t.t1, t.t0), bi, bj,
                                             t.mp / 16);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      own.hi[g] = *(const half4*)(hi + g * 256);
      own.lo[g] = *(const half4*)(hi + plane + g * 256);
    }
  }

  // What becomes of a block's sums.
  static __device__ __forceinline__ void finish(const NsArgs& a, const NsMatrix& t, float mu,
                                                int bi, int bj, const Own& own,
                                                const float (&params)[16], const f32x16& acc,
                                                float& squares) {
    if (!inside(t, bi, bj)) return;
    const int lane = threadIdx.x & 63;
    const size_t plane = (size_t)t.mp * (kApply ? t.np : t.mp);
    const float linear =
        (kApply ? a.a + mu * (a.b + mu * a.c) : a.b + 2.f * a.c * mu) * a.own_scale;
    const float factor = kSquare ? a.c * a.in_scale : a.in_scale;
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      v[e] = factor * acc[e];
      if (!kGram) v[e] += linear * ((float)own.hi[e / 4][e % 4] + (float)own.lo[e / 4][e % 4]);
    }
    if constexpr (KIND == kNsLast) {
      result(a, t, bi, bj, params, v);
      return;
    }
    if (kGram && bi == bj) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if ((lane >> 5) * 4 + e / 4 * 8 + e % 4 == (lane & 31) && bj * 32 + (lane & 31) < t.m)
          v[e] -= mu;
    }
    half_bits* const to = along(kGram ? t.a : kSquare ? t.b : t.x, bi, bj,
                                (kApply ? t.np : t.mp) / 16);
    half_bits* const at =
        across(kGram ? t.a : kSquare ? t.b : pick(a.from != 0, t.t0, t.t1), bi, bj, t.mp / 16);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (kApply) squares += v[4 * g + e] * v[4 * g + e];
        f[e] = v[4 * g + e] * a.out_scale;
      }
      const Parts4 p = split4(f);
      *(half4*)(to + g * 64) = transpose4(p.hi);
      if (PARTS == 2 || kGram || (kApply && a.keep_lo))
        *(half4*)(to + plane + g * 64) = transpose4(p.lo);
      if (kApply || bi != bj) {
        *(half4*)(at + g * 256) = p.hi;
        if (PARTS == 2 || !kSquare) *(half4*)(at + plane + g * 256) = p.lo;
      }
    }
  }

  // The last step's values: the caller's result, or the parameters' update.  f(element of the
  // lane's 16, element of the matrix) of those inside.
  template <typename F>
  static __device__ __forceinline__ void each_result(const NsMatrix& t, int bi, int bj, F&& f) {
    const int rows = pick(t.tall != 0, t.n, t.m), cols = pick(t.tall != 0, t.m, t.n);
    const int lane = threadIdx.x & 63, i = bi * 32 + (lane >> 5) * 4, j = bj * 32 + (lane & 31);
    if (j >= cols) return;
    const long long at = (long long)i * cols + j;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = e / 4 * 8 + e % 4;
      if (i + r < rows) f(e, at + (long long)r * cols);
    }
  }
  static __device__ __forceinline__ void load_params(const NsArgs& a, const NsMatrix& t, int bi,
                                                     int bj, float (&p)[16]) {
    if (KIND != kNsLast || a.out || !inside(t, bi, bj)) return;
    each_result(t, bi, bj, [&](int e, long long at) { p[e] = input(t.param, t.bf16, at); });
  }
  static __device__ __forceinline__ void result(const NsArgs& a, const NsMatrix& t, int bi, int bj,
                                                const float (&p)[16], const float (&v)[16]) {
    const float keep = 1.f - a.lr * t.decay, rate = a.lr * t.scale;
    void* const to = pick(a.out != nullptr, a.out, t.param);
    each_result(t, bi, bj, [&](int e, long long at) {
      const float r = a.out ? v[e] : p[e] * keep - rate * v[e];
      if (t.bf16)
        ((uint16_t*)to)[t.out_at + at] = f32_to_bf16_rne(r);
      else
        ((float*)to)[t.out_at + at] = r;
      if (!a.out && t.copy) ((uint16_t*)t.copy)[at] = f32_to_bf16_rne(r);
    });
  }

  // A tile's sums of squares, of each of kOfWave blocks of its waves where they are joined
  // one by one, else of all and zeros.
  static __device__ __forceinline__ void put_squares(const NsMatrix& t, const NsWork& w, int block,
                                                     float squares, float* lds) {
    if (KIND != kNsApply) return;
    squares = block_total(squares, lds);
    const int tile = w.ti * ((t.np + kTile.cols - 1) / kTile.cols) + w.tj;
    if (block >= 0) {
      if (threadIdx.x == 0) t.squares[tile * kOfWave + block] = squares;
    } else if (threadIdx.x < kOfWave) {
      t.squares[tile * kOfWave + threadIdx.x] = threadIdx.x ? 0.f : squares;
    }
  }

  static __device__ __forceinline__ void tile(const NsArgs& a, const NsMatrix& t, const NsWork& w,
                                              char* lds) {
    // (before the product where the registers hold them, else two blocks ahead)
    constexpr bool kBefore = kOfWave <= 4;
    constexpr int kOwn = kBefore ? kOfWave : 2;
    Own own[kOwn];
    float next_params[16];
    const auto load_owns = [&] {
#pragma unroll
      for (int k = 0; k < kOwn; ++k) load_own(a, t, block_row(w, k), block_column(w, k), own[k]);
    };
    const auto params_of = [&](int k) {
      load_params(a, t, block_row(w, k), block_column(w, k), next_params);
    };
    if (kOfWave == 1 && w.slot < 0) params_of(0);
    if (kBefore && w.slot < 0) load_owns();
    Acc acc;
    run(a, t, w, lds, acc);
    if (w.slot >= 0) return store_part(a.part, w.slot, acc);
    if (!kBefore) load_owns();
    if (kOfWave > 1) params_of(0);
    const float mu = mean_square(a, t, w, (float*)lds);
    float squares = 0.f;
    // (One block's code, which is run once: four times as long it waits for its own loads.)
#pragma unroll 1
    for (int k = 0; k < kOfWave; ++k) {
      Own now;
      f32x16 sums;
#pragma unroll
      for (int i = 0; i < kOfWave; ++i) {
        if (k != i) continue;  // (a branch of the whole wave)
        sums = acc[i];
        now = own[i % kOwn];
        asm volatile("");  // (not a chain of selections)
      }
      if (kOwn < kOfWave && k + kOwn < kOfWave) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
          if (k % kOwn == i)
            load_own(a, t, block_row(w, k + kOwn), block_column(w, k + kOwn), own[i]);
      }
      float params[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) params[e] = next_params[e];
      if (k + 1 < kOfWave) params_of(k + 1);
      finish(a, t, mu, block_row(w, k), block_column(w, k), now, params, sums, squares);
    }
    put_squares(t, w, -1, squares, (float*)lds);
  }
  static __device__ __forceinline__ void join(const NsArgs& a, const NsMatrix& t, const NsWork& w,
                                              int block, float* lds) {
    const int bi = block_row(w, block), bj = block_column(w, block);
    Own own;
    load_own(a, t, bi, bj, own);
    float params[16];
    load_params(a, t, bi, bj, params);
    f32x16 acc;
    load_parts(a.part, w.slot, w.slots, block, acc);
    const float mu = mean_square(a, t, w, lds);
    float squares = 0.f;
    finish(a, t, mu, bi, bj, own, params, acc, squares);
    put_squares(t, w, block, squares, lds);
  }
};

}  // namespace

template <int PARTS, int KIND, int SIZE>
__global__ __launch_bounds__(256, kNsTiles[SIZE].waves) void ns_product_kernel(NsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[kNsTiles[SIZE].lds()];
  const NsWork w = a.works[blockIdx.x];
  if (a.skip[w.matrix >> 6] >> (w.matrix & 63) & 1) return;
  const NsMatrix t = a.mats[w.matrix];
  Product<PARTS, KIND, SIZE>::tile(a, t, w, lds);
}

// Adds up the partial tiles, in their order, a block of each wave's to a workgroup: 6 to 20 us,
// bound by latency (16 tiles of 16 parts: 34 MB).
template <int PARTS, int KIND, int SIZE>
__global__ __launch_bounds__(256) void ns_join_kernel(NsArgs a) {
  __shared__ float lds[4];
  const NsWork w = a.works[blockIdx.x];
  if (a.skip[w.matrix >> 6] >> (w.matrix & 63) & 1) return;
  const NsMatrix t = a.mats[w.matrix];
  Product<PARTS, KIND, SIZE>::join(a, t, w, blockIdx.y, lds);
}

namespace {

template <int PARTS, int KIND, int SIZE>
void launch_size(const NsArgs& a, unsigned works, bool join, hipStream_t stream) {
  // (partial sums of a tile: a workgroup for each block of a wave)
  if (join)
    hipLaunchKernelGGL((ns_join_kernel<PARTS, KIND, SIZE>), dim3(works, kNsTiles[SIZE].blocks()),
                       dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((ns_product_kernel<PARTS, KIND, SIZE>), dim3(works), dim3(256), 0, stream,
                       a);
}
template <int PARTS, int KIND>
void launch_kind(const NsArgs& a, unsigned works, int size, bool join, hipStream_t stream) {
  switch (size) {
    case 0: return launch_size<PARTS, KIND, 0>(a, works, join, stream);
    case 1: return launch_size<PARTS, KIND, 1>(a, works, join, stream);
    default: return launch_size<PARTS, KIND, 2>(a, works, join, stream);
  }
}
template <int PARTS>
hipError_t launch_parts(const NsArgs& a, unsigned works, int size, bool join, hipStream_t stream) {
  switch (a.kind) {
    case kNsGram: launch_kind<PARTS, kNsGram>(a, works, size, join, stream); break;
    case kNsSquare: launch_kind<PARTS, kNsSquare>(a, works, size, join, stream); break;
    case kNsApply: launch_kind<PARTS, kNsApply>(a, works, size, join, stream); break;
    default: launch_kind<PARTS, kNsLast>(a, works, size, join, stream);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ns_norm(const NsInput& a, unsigned works, hipStream_t stream) {
  hipLaunchKernelGGL(ns_norm_kernel, dim3(works), dim3(256), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_ns_pack(const NsInput& a, unsigned works, int parts, hipStream_t stream) {
  hipLaunchKernelGGL(parts == 2 ? ns_pack_kernel<2> : ns_pack_kernel<1>, dim3(works), dim3(256), 0,
                     stream, a);
  return hipGetLastError();
}
hipError_t launch_ns_product(const NsArgs& a, unsigned works, int size, bool join, int parts,
                             hipStream_t stream) {
  return parts == 2 ? launch_parts<2>(a, works, size, join, stream)
                    : launch_parts<1>(a, works, size, join, stream);
}

}  // namespace huge2
