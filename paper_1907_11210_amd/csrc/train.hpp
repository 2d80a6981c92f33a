// train.hpp -- kernel arguments and launchers of the operators around the
// convolutions (huge2_train.h): group norm, embedding, AdamW.
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

#include "huge2.h"

namespace huge2 {

// A launch's threads along an axis are counted in 32 bits.
constexpr bool launchable(long long blocks, long long threads) {
  return blocks < (1ll << 32) / threads;
}

// ---- group norm (norm.hip) ---------------------------------------------------

// Three forms share these arguments: slabs held in registers (one pass over x), slabs
// cut into runs of pixels (two), and the general form (two, and a merge between).
// Runs: the maps of an image are cut into `chunks` of `chunk_len` pixels.
struct NormArgs {
  const void* x;
  const void* dy;
  const float* stats;  // [n][groups][2]: mean, rstd (the gradient's input)
  const float* gamma;  // null: ones
  const float* beta;   // null: zeros
  void* out;           // y or dx
  float* stats_out;    // the forward's, the caller's or the plan's
  float2* part;        // [n][chunks][c]: sums per channel
  float2* gpart;       // [n][chunks][groups]: sums per group
  float2* coef;        // gradient: [n][groups], the two group means
  float* dgamma;
  float* dbeta;
  int n, c, hw, groups, d;
  uint32_t d_mul, d_shift;  // floor(channel / d) = (channel * d_mul) >> d_shift
  int act;
  float eps;
  int stream;  // the result is stored past the caches
  int chunks, chunk_len;
  int lanes_log2;  // lanes of a wave side by side on one row (pixel or plane)
  int cblocks;     // NHWC: blocks of lanes * vector width channels; slabs of an image

  // Slabs: a workgroup's channels and pixels.
  int slabs;           // workgroups
  int threads, slots;  // of a workgroup; vectors a thread holds, 0: runs
  int rows_log2;       // NHWC: pixels side by side in a workgroup
  int lds_bytes;       // NHWC
  int slab_c;          // NHWC: channels of a slab
  int span;            // NHWC: vectors may cross groups
  int join_log2;       // NHWC: lanes that join a group
  uint32_t dl_mul, dl_shift;  // NHWC: division by a group's entries in a row
  int along;           // NCHW: vectors a thread has of one plane
  // Gradient: workgroups behind the slabs' that add up dgamma and dbeta from x and dy
  // themselves, 0: from the slabs' sums in a launch of its own.
  int direct;
  int direct_log2;            // NCHW: lanes side by side on one channel
  uint32_t px_mul, px_shift;  // division by the pixels (NCHW: vectors) of a map
};
// The most slots: what leaves a workgroup of 1024 threads without spills (128
// registers a thread; the gradient holds two tensors, and a vector that may cross
// groups two more values for each of its channels).
constexpr int slab_most(int vec, bool grad, bool span) {
  return !grad ? 16 : vec < 8 ? 8 : span ? 4 : 7;
}

hipError_t launch_norm(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream);
hipError_t launch_norm_grad(const NormArgs& a, int dtype, int nhwc, int vec, hipStream_t stream);
hipError_t launch_norm_nhwc(const NormArgs& a, int dtype, int vec, hipStream_t stream);
hipError_t launch_norm_grad_nhwc(const NormArgs& a, int dtype, int vec, hipStream_t stream);
hipError_t launch_norm_nchw(const NormArgs& a, int dtype, int vec, hipStream_t stream);
hipError_t launch_norm_grad_nchw(const NormArgs& a, int dtype, int vec, hipStream_t stream);
hipError_t launch_norm_params(const NormArgs& a, hipStream_t stream);

// ---- embedding (embedding.hip) -------------------------------------------------

struct EmbedArgs {
  const void* ids;
  const void* table;
  void* y;
  long long tokens;
  int rows, dim;
  int id64;
  float scale;
  int lanes_log2;
  int stream;  // y is stored past the caches
};
hipError_t launch_embedding(const EmbedArgs& a, int dtype, int vec, hipStream_t stream);

constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits;
constexpr int kSortTile = 1024;  // tokens of a sorting workgroup, one a thread
// Up to kMostPlaced tokens a pass takes one launch or (over kMostRecounted) two:
// workgroups place kPlaceTile each, by digits of up to kMostDigits values.
constexpr int kMostRecounted = 4096, kMostPlaced = 1 << 17, kPlaceTile = 512;
constexpr int kMostDigitBits = 12, kMostDigits = 1 << kMostDigitBits;
constexpr int kChunk = 16;     // sorted tokens of a chunk, or a multiple
// The form without a sort: its most tokens, rows that a workgroup clears, its threads.
// (512 tokens 5.5 to 10.6 us as few or all have one id, 15 and more with a sort; 2048
// tokens 15 to 34 against 25 to 19.)
constexpr int kMostFew = 1024, kFewRows = 64, kFewThreads = 512;
constexpr int kZeroRows = 16;  // rows of the table that a wave looks up
constexpr int kFewParts = 8;   // parts that a wave adds alone

struct EmbedGradArgs {
  const void* ids;
  const void* dy;
  void* dtable;
  int tokens, rows, dim;
  int id64;
  float scale;
  // tokens in the order of (id, token): keys (an id, or `rows` for one outside the
  // table) and token numbers, twice: a sorting pass reads one and writes the other
  int* key[2];
  int* token[2];
  int* hist;      // [kDigits][tiles], or [tiles][digits]
  int tiles;      // sorting workgroups
  int passes;     // of digit_bits each, or with digit_bits 0 of kDigitBits
  int digit_bits;
  float* part;    // [chunks][2][dim]: sums of rows that cross a chunk's ends
  int chunks, chunk_len;
  int lanes_log2;
  int past_caches;  // dy is read past the caches
};
hipError_t launch_embedding_grad(const EmbedGradArgs& a, int dtype, int vec, hipStream_t stream);

// ---- AdamW (adamw.hip) -----------------------------------------------------------

constexpr int kAdamBlock = 256;    // elements that share a scale
// Elements of a workgroup of 256.  Four a thread with moments in 32 bits: 134 M
// parameters 675 us, 14 M with bf16 gradients and copies 74, 0.3 M in 20 tensors 5.0; eight
// a thread 700, 77 and 5.7; sixteen 690, 83 and 8.2.  Eight with moments in 8 bits, where
// a thread's loads are short: 67 M 201 us, 2 M in 160 tensors 13.0; four a thread 215 and
// 12.2, sixteen 215 and 16.1.
constexpr int adam_work(int state_bits) { return state_bits == 8 ? 2048 : 1024; }
constexpr int kAdamTensors = 256;  // tensors of a launch: their gradients are kernel arguments

struct AdamTensorDev {
  void* param;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  long long count;
  int bf16, grad_bf16;
  float weight_decay;
  int pad;
};
struct AdamArgs {
  const AdamTensorDev* tensors;  // of the launch
  const uint2* works;            // (tensor of the launch, run of adam_work elements)
  const float* grad_scale;
  float beta1, beta2, rest1, rest2;  // rest: 1 - beta
  float lr, eps;
  float step_size;  // lr / (1 - beta1^step)
  float root;       // 1 / sqrt(1 - beta2^step)
  const void* grads[kAdamTensors];
};
hipError_t launch_adamw(const AdamArgs& a, unsigned works, int state_bits, bool past_caches,
                        hipStream_t stream);

}  // namespace huge2
