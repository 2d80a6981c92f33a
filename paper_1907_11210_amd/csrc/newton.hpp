// newton.hpp -- kernel arguments and launchers of the Newton-Schulz products (newton.hip):
// orthogonalised matrices and the Muon step.
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

namespace huge2 {

// Operands of the products are fp16 in fragments of 32 rows by 16 columns, 1 KB each, as a
// matrix instruction takes them: lane l has row l % 32, columns 8 (l / 32) to + 8.  A matrix of
// R rows and K columns is [R / 32][K / 16] fragments, both sizes rounded up to kNsPad, zeros
// behind the end.  Two such planes, of the value and of what it leaves over, are 22 bits.
constexpr int kNsPad = 64, kNsFrag = 512;  // elements
constexpr int kNsMatrices = 256;  // of a group: their gradients are kernel arguments
constexpr int kNsBlock = 64;      // rows and columns of a packing workgroup

typedef uint16_t half_bits;

// X is m x n, m <= n: a matrix with more rows than columns is taken transposed.
struct NsMatrix {
  half_bits* x;       // X [m][n], hi and lo (of one part lo for the last step alone)
  half_bits* t0;      // its transpose [n][m], hi and lo: of even steps
  half_bits* t1;      // ... and of odd ones
  half_bits* a;       // X X^T - mu I [m][m], hi and lo
  half_bits* b;       // [m][m]: hi, and with two parts lo
  float* squares;     // [squares_count]: of X's elements, by tiles and their blocks
  double* norm;       // [norm_count]: sums of squares of the input
  float* mu;          // trace(X X^T) / m
  int m, n, mp, np;   // mp, np: rounded up to kNsPad
  int tall;           // the input is n x m
  int squares_count;
  int norm_count;
  int norm_chunk;     // elements of a sum
  long long count;    // m * n
  // what the last step writes: y behind the call's pointer, or a parameter
  long long out_at;   // elements
  void* param;
  void* copy;
  float* momentum;
  int bf16, grad_bf16;
  float decay, scale;
};

struct NsWork {
  int matrix, ti, tj;
  int k0, k1;  // stages of the product
  int slot;    // of the partial tiles, -1: the whole sum; a join: the first
  int slots;   // a join: how many
};
// A workgroup's part of a product: rows of P by rows of Q, `stage` columns of them at a time
// (half as many with two parts), of which `buffers` fit its LDS.  256x128 leaves 8 blocks of sums
// a wave, 128 registers, beside two stages' fragments: with 72 KB of LDS two workgroups a unit,
// of which one computes while the other waits at its barrier.  A wave reads 6 fragments for 8
// products of them, with 128x128 4 for 4, with 64x64 2 for 1: what tile_size weighs against
// the number of tiles.
struct NsTile {
  int rows, cols, stage, buffers;
  int waves;  // of a SIMD, which its registers leave room for
  constexpr int lds() const { return (rows + cols) * stage * 2 * buffers; }
  constexpr size_t slot() const { return (size_t)rows * cols; }  // elements of a partial tile
  constexpr int blocks() const { return rows / 64 * (cols / 64); }  // of 32 x 32 to a wave
};
constexpr int kNsSizes = 3;
constexpr NsTile kNsTiles[kNsSizes] = {
    {64, 64, 64, 3, 3}, {128, 128, 32, 4, 2}, {256, 128, 32, 3, 2}};
// Products: A = X X^T, A A, B X, and B X of the last step.
enum NsKind { kNsGram = 0, kNsSquare = 1, kNsApply = 2, kNsLast = 3 };

struct NsArgs {
  const NsMatrix* mats;
  const NsWork* works;
  float* part;
  int kind, step;
  int from;              // the step reads t0 or t1 and writes the other
  float a, b, c;         // of the step's polynomial
  float in_scale;        // of a product's sum
  float own_scale;       // of the values that are added to it
  float out_scale;       // of what is stored
  int keep_lo;           // the next step is the last
  float lr;
  void* out;             // null: parameters
  uint64_t skip[kNsMatrices / 64];  // matrices without a gradient
};
struct NsInput {
  const NsMatrix* mats;
  const uint2* works;    // (matrix, chunk of a sum or packed block)
  int muon, nesterov;
  int keep_lo;           // there is one step
  float momentum, rest;  // rest: 1 - momentum
  double eps;
  float out_scale;
  const float* grad_scale;
  const void* src[kNsMatrices];
};

hipError_t launch_ns_norm(const NsInput& a, unsigned works, hipStream_t stream);
hipError_t launch_ns_pack(const NsInput& a, unsigned works, int parts, hipStream_t stream);
// size: of the tiles, their place in kNsTiles.
hipError_t launch_ns_product(const NsArgs& a, unsigned works, int size, bool join, int parts,
                             hipStream_t stream);

}  // namespace huge2
