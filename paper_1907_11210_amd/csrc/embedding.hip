// embedding.hip -- embedding lookup with a scale, and the table's gradient by
// sorted tokens (huge2_train.h).
#include <algorithm>

#include "train.hpp"
#include "train_device.hpp"

namespace huge2 {

namespace {

// The id of a token, or `rows` if it is outside the table.
__device__ __forceinline__ int known_id(const void* ids, int id64, long long t, int rows) {
  const long long id = id64 ? ((const long long*)ids)[t] : (long long)((const int*)ids)[t];
  return id >= 0 && id < rows ? (int)id : rows;
}

__device__ __forceinline__ int digit_of(int key, int pass) {
  return key >> (pass * kDigitBits) & (kDigits - 1);
}

}  // namespace

// A row of 2^lanes_log2 lanes to a token, kLookups tokens each, whose ids and then
// whose rows are all in flight together.
constexpr int kLookups = 4;
template <typename T, int VW>
__global__ __launch_bounds__(256) void embedding_kernel(EmbedArgs a, int cblocks) {
  const int lanes = 1 << a.lanes_log2, per = 256 >> a.lanes_log2;
  const int cb = blockIdx.x % cblocks;
  const long long t0 = (long long)(blockIdx.x / cblocks) * per * kLookups + (threadIdx.x >> a.lanes_log2);
  const int col = (cb * lanes + (threadIdx.x & (lanes - 1))) * VW;
  if (col >= a.dim) return;
  int id[kLookups];
#pragma unroll
  for (int j = 0; j < kLookups; ++j) {
    const long long t = t0 + j * per;
    id[j] = t < a.tokens ? known_id(a.ids, a.id64, t, a.rows) : a.rows;
  }
  float f[kLookups][VW];
#pragma unroll
  for (int j = 0; j < kLookups; ++j) {
    if (id[j] < a.rows) {
      unpack<T, VW>(load_pack<T, VW>((const T*)a.table + (size_t)id[j] * a.dim + col), f[j]);
    } else {
#pragma unroll
      for (int e = 0; e < VW; ++e) f[j][e] = 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < kLookups; ++j) {
    const long long t = t0 + j * per;
    if (t >= a.tokens) break;
    // (a row outside the table is zeros whatever the scale)
    const float scale = id[j] < a.rows ? a.scale : 0.f;
#pragma unroll
    for (int e = 0; e < VW; ++e) f[j][e] *= scale;
    store_pack<T, VW>((T*)a.y + (size_t)t * a.dim + col, pack<T, VW>(f[j]));
  }
}

// ---- the order of the tokens: a stable radix sort by id ---------------------------

// Counts of each digit in a tile.
__global__ __launch_bounds__(kSortTile) void sort_count_kernel(EmbedGradArgs a, int pass) {
  __shared__ int count[kDigits];
  for (int i = threadIdx.x; i < kDigits; i += kSortTile) count[i] = 0;
  __syncthreads();
  const int t = blockIdx.x * kSortTile + threadIdx.x;
  if (t < a.tokens) {
    const int key = pass == 0 ? known_id(a.ids, a.id64, t, a.rows) : a.key[pass & 1][t];
    atomicAdd(&count[digit_of(key, pass)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kDigits; i += kSortTile)
    a.hist[(size_t)i * a.tiles + blockIdx.x] = count[i];
}

// Exclusive sums of one digit's counts over the tiles; their total behind them.
__global__ __launch_bounds__(256) void sort_scan_kernel(EmbedGradArgs a) {
  __shared__ int lds[4];
  int* h = a.hist + (size_t)blockIdx.x * a.tiles;
  int base = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += 256) {
    const int t = t0 + threadIdx.x;
    const int mine = t < a.tiles ? h[t] : 0;
    int s = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int o = __shfl_up(s, m);
      if ((threadIdx.x & 63) >= m) s += o;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    int before = base;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += lds[w];
    if (t < a.tiles) h[t] = before + s - mine;
    base += lds[0] + lds[1] + lds[2] + lds[3];
  }
  if (threadIdx.x == 0) a.hist[(size_t)kDigits * a.tiles + blockIdx.x] = base;
}

// Each token to its place: behind all smaller digits, the earlier tiles' equal
// ones, the earlier waves' and the lower lanes'.
__global__ __launch_bounds__(kSortTile) void sort_scatter_kernel(EmbedGradArgs a, int pass) {
  constexpr int kWaves = kSortTile / 64;
  __shared__ int count[kWaves][kDigits];
  __shared__ int base[kDigits];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < kWaves * kDigits; i += kSortTile) (&count[0][0])[i] = 0;
  if (wave == 0) {  // exclusive sums of the digits' totals, four a lane
    const int* total = a.hist + (size_t)kDigits * a.tiles;
    int v[4], s = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = total[lane * 4 + e], s += v[e];
    int up = s;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int o = __shfl_up(up, m);
      if (lane >= m) up += o;
    }
    int at = up - s;
#pragma unroll
    for (int e = 0; e < 4; ++e) base[lane * 4 + e] = at, at += v[e];
  }
  __syncthreads();
  const int t = blockIdx.x * kSortTile + threadIdx.x;
  const bool in = t < a.tokens;
  int key = 0, token = t;
  if (in) {
    key = pass == 0 ? known_id(a.ids, a.id64, t, a.rows) : a.key[pass & 1][t];
    if (pass) token = a.token[pass & 1][t];
  }
  const int digit = digit_of(key, pass);
  unsigned long long same = __ballot(in);
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const unsigned long long one = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? one : ~one;
  }
  const int rank = __popcll(same & ((1ull << lane) - 1));
  if (in && rank == 0) count[wave][digit] = __popcll(same);
  __syncthreads();
  if (threadIdx.x < kDigits) {
    int at = base[threadIdx.x] + a.hist[(size_t)threadIdx.x * a.tiles + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int n = count[w][threadIdx.x];
      count[w][threadIdx.x] = at;
      at += n;
    }
  }
  __syncthreads();
  if (in) {
    const int to = count[wave][digit] + rank;
    a.key[(pass + 1) & 1][to] = key;
    a.token[(pass + 1) & 1][to] = token;
  }
}

// ---- sums over equal ids -------------------------------------------------------------

namespace {

template <typename T, int VW>
__device__ __forceinline__ void store_row(const EmbedGradArgs& a, int row, int col,
                                          const float (&acc)[VW]) {
  float f[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) f[e] = acc[e] * a.scale;
  store_pack<T, VW>((T*)a.dtable + (size_t)row * a.dim + col, pack<T, VW>(f));
}
template <int VW>
__device__ __forceinline__ void store_part(const EmbedGradArgs& a, int chunk, int which, int col,
                                           const float (&acc)[VW]) {
  float* p = a.part + ((size_t)chunk * 2 + which) * a.dim + col;
#pragma unroll
  for (int e = 0; e < VW; ++e) p[e] = acc[e];
}

}  // namespace

// A row of lanes to a chunk of sorted tokens and a block of columns: adds up the
// gradients of equal ids in order.  A row of the table whose tokens all lie in the
// chunk is written; what a chunk's first row has behind tokens of an earlier chunk
// goes to part[chunk][0], what its last row has before a later chunk to
// part[chunk][1].
template <typename T, int VW>
__global__ __launch_bounds__(256) void embedding_sum_kernel(EmbedGradArgs a, int cblocks) {
  const int lanes = 1 << a.lanes_log2;
  const int* key = a.key[a.passes & 1];
  const int* token = a.token[a.passes & 1];
  const int chunk = (blockIdx.x / cblocks) * (256 >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  const int col = (blockIdx.x % cblocks * lanes + (threadIdx.x & (lanes - 1))) * VW;
  if (chunk >= a.chunks || col >= a.dim) return;
  const int c0 = chunk * a.chunk_len, c1 = min(a.tokens, c0 + a.chunk_len);
  int cur = key[c0];
  bool head = c0 > 0 && key[c0 - 1] == cur;
  float acc[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) acc[e] = 0.f;
  constexpr int kDeep = 8;
  for (int i = c0; i < c1 && cur < a.rows; i += kDeep) {
    int k[kDeep];
    Pack<T, VW> g[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) k[j] = i + j < c1 ? key[i + j] : a.rows;
#pragma unroll
    for (int j = 0; j < kDeep; ++j)
      if (k[j] < a.rows)
        g[j] = load_pack<T, VW>((const T*)a.dy + (size_t)token[i + j] * a.dim + col);
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      if (i + j >= c1) break;
      if (k[j] != cur) {
        if (head)
          store_part<VW>(a, chunk, 0, col, acc);
        else
          store_row<T, VW>(a, cur, col, acc);
        head = false;
        cur = k[j];
#pragma unroll
        for (int e = 0; e < VW; ++e) acc[e] = 0.f;
        if (cur >= a.rows) break;
      }
      float f[VW];
      unpack<T, VW>(g[j], f);
#pragma unroll
      for (int e = 0; e < VW; ++e) acc[e] += f[e];
    }
  }
  if (cur >= a.rows) return;
  const bool open = c1 < a.tokens && key[c1] == cur;
  if (head)
    store_part<VW>(a, chunk, 0, col, acc);
  else if (open)
    store_part<VW>(a, chunk, 1, col, acc);
  else
    store_row<T, VW>(a, cur, col, acc);
}

// The rows that cross chunks: a row of lanes to the chunk in which such a row
// begins adds the chunks' parts in order.
template <typename T, int VW>
__global__ __launch_bounds__(256) void embedding_join_kernel(EmbedGradArgs a, int cblocks) {
  const int lanes = 1 << a.lanes_log2;
  const int* key = a.key[a.passes & 1];
  int chunk = (blockIdx.x / cblocks) * (256 >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  const int col = (blockIdx.x % cblocks * lanes + (threadIdx.x & (lanes - 1))) * VW;
  if (chunk + 1 >= a.chunks || col >= a.dim) return;
  const int c0 = chunk * a.chunk_len, c1 = c0 + a.chunk_len;
  const int row = key[c1 - 1];
  if (row >= a.rows || key[c1] != row) return;
  if (key[c0] == row && c0 > 0 && key[c0 - 1] == row) return;  // begins earlier
  float acc[VW];
  const float* p = a.part + ((size_t)chunk * 2 + 1) * a.dim + col;
#pragma unroll
  for (int e = 0; e < VW; ++e) acc[e] = p[e];
  for (;;) {
    ++chunk;
    p = a.part + (size_t)chunk * 2 * a.dim + col;
#pragma unroll
    for (int e = 0; e < VW; ++e) acc[e] += p[e];
    const int end = (chunk + 1) * a.chunk_len;
    if (end >= a.tokens || key[end] != row) break;
  }
  store_row<T, VW>(a, row, col, acc);
}

// Zeros to the rows that no token has.
template <typename T, int VW>
__global__ __launch_bounds__(256) void embedding_zero_kernel(EmbedGradArgs a) {
  const int* key = a.key[a.passes & 1];
  const int lanes = 1 << a.lanes_log2;
  const int row = blockIdx.x * (256 >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  if (row >= a.rows) return;
  int lo = 0, hi = a.tokens;  // the first token of this row or a later one
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (key[mid] < row)
      lo = mid + 1;
    else
      hi = mid;
  }
  if (lo < a.tokens && key[lo] == row) return;
  float zero[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) zero[e] = 0.f;
  for (int col = (threadIdx.x & (lanes - 1)) * VW; col < a.dim; col += lanes * VW)
    store_pack<T, VW>((T*)a.dtable + (size_t)row * a.dim + col, pack<T, VW>(zero));
}

namespace {

template <typename T, int VW>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t stream) {
  const long long per = (256 >> a.lanes_log2) * kLookups;
  const int cblocks = (a.dim / VW + (1 << a.lanes_log2) - 1) >> a.lanes_log2;
  const long long grid = (a.tokens + per - 1) / per * cblocks;
  hipLaunchKernelGGL((embedding_kernel<T, VW>), dim3((unsigned)grid), dim3(256), 0, stream, a,
                     cblocks);
  return hipGetLastError();
}

template <typename T, int VW>
hipError_t launch_grad(const EmbedGradArgs& a, hipStream_t stream) {
  const dim3 wg(256);
  const int per = 256 >> a.lanes_log2;
  const int cblocks = (a.dim / VW + (1 << a.lanes_log2) - 1) >> a.lanes_log2;
  for (int pass = 0; pass < a.passes && a.tokens; ++pass) {
    hipLaunchKernelGGL(sort_count_kernel, dim3(a.tiles), dim3(kSortTile), 0, stream, a, pass);
    hipLaunchKernelGGL(sort_scan_kernel, dim3(kDigits), wg, 0, stream, a);
    hipLaunchKernelGGL(sort_scatter_kernel, dim3(a.tiles), dim3(kSortTile), 0, stream, a, pass);
  }
  hipLaunchKernelGGL((embedding_zero_kernel<T, VW>), dim3((unsigned)(((long long)a.rows + per - 1) / per)),
                     wg, 0, stream, a);
  if (a.tokens) {
    const long long grid = (long long)((a.chunks + per - 1) / per) * cblocks;
    hipLaunchKernelGGL((embedding_sum_kernel<T, VW>), dim3((unsigned)grid), wg, 0, stream, a,
                       cblocks);
    if (a.chunks > 1)
      hipLaunchKernelGGL((embedding_join_kernel<T, VW>), dim3((unsigned)grid), wg, 0, stream, a,
                         cblocks);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbedArgs& a, int dtype, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    return vec == 8   ? launch_lookup<uint16_t, 8>(a, stream)
           : vec == 2 ? launch_lookup<uint16_t, 2>(a, stream)
                      : launch_lookup<uint16_t, 1>(a, stream);
  return vec == 4 ? launch_lookup<uint32_t, 4>(a, stream) : launch_lookup<uint32_t, 1>(a, stream);
}

hipError_t launch_embedding_grad(const EmbedGradArgs& a, int dtype, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    return vec == 8   ? launch_grad<uint16_t, 8>(a, stream)
           : vec == 2 ? launch_grad<uint16_t, 2>(a, stream)
                      : launch_grad<uint16_t, 1>(a, stream);
  return vec == 4 ? launch_grad<uint32_t, 4>(a, stream) : launch_grad<uint32_t, 1>(a, stream);
}

}  // namespace huge2
