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
// whose rows are all in flight together (1, 2 and 8 were no faster).
//
// Bound by the result's bytes: 65536 tokens of 256 bf16 out of 8192, out of the caches: 9.8 us
// for 34 MB, and 22 MB of the table's 4 read by the XCDs together; 64 tokens of 100: 2.8 us.
constexpr int kLookups = 4;
template <typename T, int VW>
__global__ __launch_bounds__(256) void embedding_kernel(EmbedArgs a, int cblocks) {
  const int lanes = 1 << a.lanes_log2, per = 256 >> a.lanes_log2;
  const int cb = blockIdx.x % cblocks;
  const long long t0 =
      (long long)(blockIdx.x / cblocks) * per * kLookups + (threadIdx.x >> a.lanes_log2);
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
    store_pack<T, VW>((T*)a.y + (size_t)t * a.dim + col, pack<T, VW>(f[j]), a.stream);
  }
}

// ---- the order of the tokens: a stable radix sort by id ---------------------------

// One pass, up to kMostPlaced tokens: a workgroup places kPlaceTile of them, behind
// all smaller digits, the equal ones of the tokens before its own, of its earlier
// waves and of lower lanes.  For this it adds up the tiles' counts (COUNTED: those
// that sort_tile_counts_kernel left), or counts all tokens itself, one launch less
// and as much more work as there are workgroups: 42 cycles of its compute unit's LDS
// atomics for 64 tokens, 4.7 us for 512 tokens, 6.3 for 4096, 11.5 for 16384, 15.8 for
// 32768 (in two launches 11.2 for 16384 with 2048 digits, 10.1 for 32768 with 256).
// Above, all workgroups reading all tiles' counts is what grows: three launches.
__global__ __launch_bounds__(kPlaceTile) void sort_tile_counts_kernel(EmbedGradArgs a, int pass) {
  __shared__ int count[kMostDigits];
  const int digits = 1 << a.digit_bits;
  for (int i = threadIdx.x; i < digits; i += kPlaceTile) count[i] = 0;
  __syncthreads();
  const int t = blockIdx.x * kPlaceTile + threadIdx.x;
  if (t < a.tokens) {
    const int key = pass == 0 ? known_id(a.ids, a.id64, t, a.rows) : a.key[pass & 1][t];
    atomicAdd(&count[key >> (pass * a.digit_bits) & (digits - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < digits; i += kPlaceTile)
    a.hist[((size_t)blockIdx.x << a.digit_bits) + i] = count[i];
}

template <bool COUNTED>
__global__ __launch_bounds__(1024) void sort_place_kernel(EmbedGradArgs a, int pass) {
  __shared__ int all[kMostDigits], before[kMostDigits], lds[16];
  const int digits = 1 << a.digit_bits, mask = digits - 1, shift = pass * a.digit_bits;
  const int* from = a.key[pass & 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int first = blockIdx.x * kPlaceTile, t = first + threadIdx.x;
  const bool in = threadIdx.x < kPlaceTile && t < a.tokens;
  int key = 0, token = t;
  if (in) {
    key = pass == 0 ? known_id(a.ids, a.id64, t, a.rows) : from[t];
    if (pass) token = a.token[pass & 1][t];
  }
  for (int i = threadIdx.x; i < digits; i += 1024) all[i] = before[i] = 0;
  __syncthreads();
  if constexpr (COUNTED) {
    // four digits a thread, as many tiles side by side as there are threads for
    const int quads = digits >> 2, rows = 1024 / quads, d = (threadIdx.x & (quads - 1)) * 4;
    int4 sum = make_int4(0, 0, 0, 0), sum_before = sum;
#pragma unroll 8
    for (int tile = threadIdx.x / quads; tile < a.tiles; tile += rows) {
      const int4 n = *(const int4*)(a.hist + ((size_t)tile << a.digit_bits) + d);
      const int m = tile < (int)blockIdx.x ? -1 : 0;
      sum.x += n.x, sum.y += n.y, sum.z += n.z, sum.w += n.w;
      sum_before.x += n.x & m, sum_before.y += n.y & m;
      sum_before.z += n.z & m, sum_before.w += n.w & m;
    }
    const int v[4] = {sum.x, sum.y, sum.z, sum.w};
    const int u[4] = {sum_before.x, sum_before.y, sum_before.z, sum_before.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (v[e]) atomicAdd(&all[d + e], v[e]);
      if (u[e]) atomicAdd(&before[d + e], u[e]);
    }
  } else {
    const auto count = [&](int t0, int t1) {
      for (int i = t0 + threadIdx.x; i < t1; i += 1024) {
        const int digit =
            (pass == 0 ? known_id(a.ids, a.id64, i, a.rows) : from[i]) >> shift & mask;
        // one addition where many are the same: they would queue up at one address
        const int lead = __builtin_amdgcn_readfirstlane(digit);
        const unsigned long long same = __ballot(digit == lead);
        if (__popcll(same) <= 16 || digit != lead)
          atomicAdd(&all[digit], 1);
        else if (__ffsll(same) - 1 == lane)
          atomicAdd(&all[lead], __popcll(same));
      }
    };
    count(0, first);
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += 1024) before[i] = all[i];
    __syncthreads();
    count(first, a.tokens);
  }
  __syncthreads();
  // exclusive sums of the digits' counts, kMostDigits / 1024 neighbours a thread
  constexpr int kPer = kMostDigits / 1024;
  int v[kPer], s = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = threadIdx.x * kPer + e;
    v[e] = i < digits ? all[i] : 0;
    s += v[e];
  }
  int up = s;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(up, m);
    if (lane >= m) up += o;
  }
  if (lane == 63) lds[wave] = up;
  __syncthreads();
  int at = up - s;
  for (int w = 0; w < wave; ++w) at += lds[w];
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = threadIdx.x * kPer + e;
    if (i < digits) before[i] += at;
    at += v[e];
  }
  int digit = 0, rank = 0;
  unsigned long long same = 0;
  if (wave < kPlaceTile / 64) {
    digit = key >> shift & mask;
    same = __ballot(in);
    for (int b = 0; b < a.digit_bits; ++b) {
      const unsigned long long one = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? one : ~one;
    }
    rank = __popcll(same & ((1ull << lane) - 1));
  }
  for (int w = 0; w < kPlaceTile / 64; ++w) {  // the waves in order
    __syncthreads();
    if (w == wave && in) {
      const int base = before[digit];
      if (rank == 0) before[digit] = base + __popcll(same);
      a.key[(pass + 1) & 1][base + rank] = key;
      a.token[(pass + 1) & 1][base + rank] = token;
    }
  }
}

// For more tokens, three launches a pass.

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

// The first of the sorted tokens lo .. hi whose key is at least `key`; seven keys
// are looked at together, since it is their latency that a search takes.
__device__ __forceinline__ int lower_bound(const int* keys, int lo, int hi, int key) {
  while (lo < hi) {
    const int step = (hi - lo + 7) / 8;
    int less = 0, probe[8];
#pragma unroll
    for (int i = 1; i < 8; ++i) probe[i] = keys[min(lo + i * step, hi) - 1];
#pragma unroll
    for (int i = 1; i < 8; ++i) less += (lo + i * step <= hi) & (probe[i] < key);
    const int from = lo + less * step;
    if (less < 7) hi = min(hi, from + step - 1);
    lo = from;
  }
  return lo;
}

// Zeros to those of kZeroRows rows that no token has: a wave looks them all up at
// once, a lane each.
template <typename T, int VW>
__device__ __forceinline__ void zero_rows(const EmbedGradArgs& a, const int* key, long long part) {
  const long long first = part * kZeroRows;
  const int lane = threadIdx.x & 63;
  const long long row = first + lane;
  bool empty = lane < kZeroRows && row < a.rows;
  if (empty) {
    const int at = lower_bound(key, 0, a.tokens, (int)row);
    empty = at >= a.tokens || key[at] != (int)row;
  }
  float zero[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) zero[e] = 0.f;
  for (unsigned long long left = __ballot(empty); left; left &= left - 1) {
    T* p = (T*)a.dtable + (size_t)(first + __ffsll(left) - 1) * a.dim;
    for (int col = lane * VW; col < a.dim; col += 64 * VW)
      store_pack<T, VW>(p + col, pack<T, VW>(zero));
  }
}

}  // namespace

// A row of lanes to a chunk of sorted tokens and a block of columns: adds up the
// gradients of equal ids in order, 8 or 16 rows in flight.  A row of the table whose
// tokens all lie in the chunk is written; what a chunk's first row has behind tokens
// of an earlier chunk goes to part[chunk][0], what its last row has before a later
// chunk to part[chunk][1].  Behind the chunks' workgroups, those of the rows without
// tokens.
//
// Bound by the reads of dy, rows anywhere in memory, and the table's bytes.  A chunk is
// short (16 tokens) so that a few thousand tokens already make a few thousand waves; the
// parts then are an eighth of the reads at most.  PAST: dy is read past the caches.
// 32768 tokens of 1024 bf16, 40000 ids: 25 us for 150 MB; 16384 of 256 fp32, 1024 ids: 6.9.
template <typename T, int VW, bool WAVE, bool PAST>
__global__ __launch_bounds__(256) void embedding_sum_kernel(EmbedGradArgs a, int cblocks,
                                                            unsigned sum_blocks) {
  const int* __restrict__ key = a.key[a.passes & 1];
  const int* __restrict__ token = a.token[a.passes & 1];
  if (blockIdx.x >= sum_blocks) {
    zero_rows<T, VW>(a, key, (long long)(blockIdx.x - sum_blocks) * 4 + (threadIdx.x >> 6));
    return;
  }
  const int lanes = 1 << a.lanes_log2;
  int chunk = (blockIdx.x / cblocks) * (256 >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  if (WAVE) chunk = __builtin_amdgcn_readfirstlane(chunk);
  int col = (blockIdx.x % cblocks * lanes + (threadIdx.x & (lanes - 1))) * VW;
  if (chunk >= a.chunks) return;
  // lanes behind the last column stay (the others read keys out of theirs), on column
  // 0, and store nothing
  const bool in = col < a.dim;
  if (!in) col = 0;
  const int c0 = chunk * a.chunk_len, c1 = min(a.tokens, c0 + a.chunk_len);
  // (everything that can be is loaded before the first wait)
  const int last = a.tokens - 1;
  int before = key[max(c0 - 1, 0)], next = key[min(c1, last)], cur = key[c0];
  if (WAVE) {
    before = __builtin_amdgcn_readfirstlane(before);
    next = __builtin_amdgcn_readfirstlane(next);
    cur = __builtin_amdgcn_readfirstlane(cur);
  }
  bool head = c0 > 0 && before == cur;
  float acc[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) acc[e] = 0.f;
  // WAVE: a whole wave to a chunk, whose keys and tokens are scalars, out of one load
  constexpr int kDeep = WAVE ? kChunk : kChunk / 2;
  for (int i = c0; i < c1 && cur < a.rows; i += kDeep) {
    int k[kDeep], t[kDeep];
    Pack<T, VW> g[kDeep];
    if constexpr (WAVE) {
      const int at = min(i + (int)(threadIdx.x & (kDeep - 1)), last);
      const int mine = key[at], token_mine = token[at];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        k[j] = __builtin_amdgcn_readlane(mine, j);
        t[j] = __builtin_amdgcn_readlane(token_mine, j);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        const int at = min(i + j, last);
        k[j] = key[at];
        t[j] = token[at];
      }
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j)
      if (i + j < c1 && k[j] < a.rows) {
        const T* p = (const T*)a.dy + (size_t)t[j] * a.dim + col;
        if constexpr (PAST)
          g[j] = load_stream<T, VW>(p);
        else
          g[j] = load_pack<T, VW>(p);
      }
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      if (i + j < c1 && cur < a.rows) {
        if (k[j] != cur) {
          if (!in)
            ;
          else if (head)
            store_part<VW>(a, chunk, 0, col, acc);
          else
            store_row<T, VW>(a, cur, col, acc);
          head = false;
          cur = k[j];
#pragma unroll
          for (int e = 0; e < VW; ++e) acc[e] = 0.f;
        }
        if (cur < a.rows) {
          float f[VW];
          unpack<T, VW>(g[j], f);
#pragma unroll
          for (int e = 0; e < VW; ++e) acc[e] += f[e];
        }
      }
    }
  }
  if (cur >= a.rows || !in) return;
  if (head)
    store_part<VW>(a, chunk, 0, col, acc);
  else if (c1 <= last && next == cur)
    store_part<VW>(a, chunk, 1, col, acc);
  else
    store_row<T, VW>(a, cur, col, acc);
}

// The rows that cross chunks: a wave to the chunk in which such a row begins adds
// the chunks' parts in order; a row of more than kFewParts parts is shared by the
// workgroup's 16 waves, whose sums are added in wave order.
//
// Bound by the latency of loads one behind the other: keys, parts.  16384 tokens of
// 256 fp32 and 1024 ids: 5.5 us; 32768 of 1024 bf16, skewed over 40000 ids: 9.0; 65536
// of 512 bf16, all that are not padding one id, 2048 parts: 26.5.
template <typename T, int VW>
__global__ __launch_bounds__(1024) void embedding_join_kernel(EmbedGradArgs a, int cblocks) {
  __shared__ int2 many[16];  // first part, parts
  __shared__ float sums[16][64 * VW];
  const int* __restrict__ key = a.key[a.passes & 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int chunk = blockIdx.x / cblocks * 16 + wave;
  const int col = (blockIdx.x % cblocks * 64 + lane) * VW;
  const bool in = col < a.dim;
  const auto add = [&](float (&acc)[VW], int part) {
    const float* p = a.part + (size_t)part * a.dim + col;
    float f[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) f[e] = p[e];
#pragma unroll
    for (int e = 0; e < VW; ++e) acc[e] += f[e];
  };
  // the keys at the chunk's ends and where the next chunks begin, all together
  const int c0 = chunk * a.chunk_len, c1 = c0 + a.chunk_len, last = a.tokens - 1;
  const int before = key[min(max(c0 - 1, 0), last)], first = key[min(c0, last)];
  const int row = key[min(c1 - 1, last)];
  int begin[kFewParts + 1], parts = 0;
#pragma unroll
  for (int j = 0; j <= kFewParts; ++j) begin[j] = key[min(c1 + j * a.chunk_len, last)];
  if (c1 <= last && row < a.rows && begin[0] == row && !(first == row && c0 > 0 && before == row)) {
#pragma unroll
    for (int j = 0; j <= kFewParts; ++j)  // sorted: those that it reaches come first
      parts += (c1 + j * a.chunk_len <= last) & (begin[j] == row);
    if (parts > kFewParts) {  // the lanes look at 64 chunks' beginnings at once
      int hi = (last - c1) / a.chunk_len + 1;
      while (parts < hi) {
        const int step = (hi - parts + 63) / 64, j = parts + (lane + 1) * step - 1;
        const int more = __popcll(__ballot(j < hi && key[min(c1 + j * a.chunk_len, last)] == row));
        parts += more * step;
        hi = min(hi, parts + step - 1);
        parts = min(parts, hi);
      }
    }
  }
  float acc[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) acc[e] = 0.f;
  if (lane == 0) many[wave] = make_int2(chunk, parts > kFewParts ? parts : 0);
  if (parts && parts <= kFewParts && in) {
    add(acc, chunk * 2 + 1);
#pragma unroll
    for (int j = 0; j < kFewParts; ++j)
      if (j < parts) add(acc, (chunk + 1 + j) * 2);
    store_row<T, VW>(a, row, col, acc);
  }
  __syncthreads();
  for (int w = 0; w < 16; ++w) {
    const int2 m = many[w];
    if (m.y == 0) continue;
#pragma unroll
    for (int e = 0; e < VW; ++e) acc[e] = 0.f;
    if (in) {
#pragma unroll 8
      for (int j = wave; j < m.y; j += 16) add(acc, (m.x + 1 + j) * 2);
    }
#pragma unroll
    for (int e = 0; e < VW; ++e) sums[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    if (wave == w && in) {
      for (int q = 0; q < 16; ++q)
        if (q != wave) {
#pragma unroll
          for (int e = 0; e < VW; ++e) acc[e] += sums[q][e * 64 + lane];
        }
      add(acc, m.x * 2 + 1);
      store_row<T, VW>(a, row, col, acc);
    }
    __syncthreads();
  }
}

// Up to kMostFew tokens: all in one launch, no order and no workspace.  A workgroup
// to a token looks for the tokens of the same id among all; if its own is the first of
// them, it adds up their gradients in order, the waves sharing the columns or, where
// the tokens are many, the tokens.  Behind those, workgroups of kFewRows rows
// clear the ones that no token has.
//
// Bound by latency, three loads one behind the other (5.5 us where the sort, the sums
// and the join took 15); every workgroup reading all ids is what limits the tokens.
template <typename T, int VW>
__global__ __launch_bounds__(kFewThreads) void embedding_few_kernel(EmbedGradArgs a) {
  __shared__ int list[kMostFew];
  __shared__ int counts[kMostFew / 64];
  constexpr int kWaves = kFewThreads / 64, kSteps = kMostFew / kFewThreads;
  __shared__ float sums[kWaves][64 * VW];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= a.tokens) {
    const int first = (blockIdx.x - a.tokens) * kFewRows;
    for (int i = threadIdx.x; i < kFewRows; i += kFewThreads) list[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < a.tokens; t += kFewThreads) {
      const int row = known_id(a.ids, a.id64, t, a.rows) - first;
      if (row >= 0 && row < kFewRows) list[row] = 1;  // (`rows` itself may mark a row beyond)
    }
    __syncthreads();
    float zero[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) zero[e] = 0.f;
    for (int r = wave; r < kFewRows && first + r < a.rows; r += kWaves) {
      if (list[r]) continue;
      T* p = (T*)a.dtable + (size_t)(first + r) * a.dim;
      for (int col = lane * VW; col < a.dim; col += 64 * VW)
        store_pack<T, VW>(p + col, pack<T, VW>(zero));
    }
    return;
  }
  const int mine = known_id(a.ids, a.id64, blockIdx.x, a.rows);
  // a bit for each token, kFewThreads tokens a step
  unsigned long long same[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const int t = k * kFewThreads + threadIdx.x;
    same[k] =
        __ballot(t < a.tokens && known_id(a.ids, a.id64, min(t, a.tokens - 1), a.rows) == mine);
    if (lane == 0) counts[k * kWaves + wave] = __popcll(same[k]);
  }
  if (mine >= a.rows) return;
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    int at = n;
    for (int w = 0; w < kWaves; ++w) {
      at += w < wave ? counts[k * kWaves + w] : 0;
      n += counts[k * kWaves + w];
    }
    if (same[k] >> lane & 1)
      list[at + __popcll(same[k] & ((1ull << lane) - 1))] = k * kFewThreads + threadIdx.x;
  }
  __syncthreads();
  if (list[0] != (int)blockIdx.x) return;
  constexpr int kAhead = 16;
  const auto add = [&](int from, int to, int col, float (&acc)[VW]) {
    for (int i = from; i < to; i += kAhead) {
      Pack<T, VW> g[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < to) g[j] = load_pack<T, VW>((const T*)a.dy + (size_t)list[i + j] * a.dim + col);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i + j < to) {
          float f[VW];
          unpack<T, VW>(g[j], f);
#pragma unroll
          for (int e = 0; e < VW; ++e) acc[e] += f[e];
        }
      }
    }
  };
  const bool share = n > kAhead;  // the tokens
  for (int c0 = share ? 0 : wave * 64 * VW; c0 < a.dim; c0 += share ? 64 * VW : kFewThreads * VW) {
    const int col = c0 + lane * VW;
    const bool in = col < a.dim;
    float acc[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) acc[e] = 0.f;
    if (!share) {
      if (in) {
        add(0, n, col, acc);
        store_row<T, VW>(a, mine, col, acc);
      }
      continue;
    }
    const int each = (n + kWaves - 1) / kWaves;
    if (in) add(min(n, wave * each), min(n, (wave + 1) * each), col, acc);
#pragma unroll
    for (int e = 0; e < VW; ++e) sums[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    if (wave == 0 && in) {
      for (int w = 1; w < kWaves; ++w) {
#pragma unroll
        for (int e = 0; e < VW; ++e) acc[e] += sums[w][e * 64 + lane];
      }
      store_row<T, VW>(a, mine, col, acc);
    }
    __syncthreads();
  }
}

namespace {

template <typename T, int VW>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t stream) {
  const long long per = (256 >> a.lanes_log2) * kLookups;
  const int cblocks = (a.dim / VW + (1 << a.lanes_log2) - 1) >> a.lanes_log2;
  const long long most = ((1 << 24) - 1) / cblocks * per;  // tokens that a launch can have
  for (long long t = 0; t < a.tokens; t += most) {
    EmbedArgs b = a;
    b.ids = (const char*)a.ids + t * (a.id64 ? 8 : 4);
    b.y = (T*)a.y + t * a.dim;
    b.tokens = a.tokens - t < most ? a.tokens - t : most;
    const long long grid = (b.tokens + per - 1) / per * cblocks;
    hipLaunchKernelGGL((embedding_kernel<T, VW>), dim3((unsigned)grid), dim3(256), 0, stream, b,
                       cblocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int VW>
hipError_t launch_grad(const EmbedGradArgs& a, hipStream_t stream) {
  const dim3 wg(256);
  if (a.tokens <= kMostFew) {
    const unsigned rows = (unsigned)(((long long)a.rows + kFewRows - 1) / kFewRows);
    hipLaunchKernelGGL((embedding_few_kernel<T, VW>), dim3(a.tokens + rows),
                       dim3(kFewThreads), 0, stream, a);
    return hipGetLastError();
  }
  const int per = 256 >> a.lanes_log2;
  const int cblocks = (a.dim / VW + (1 << a.lanes_log2) - 1) >> a.lanes_log2;
  for (int pass = 0; pass < a.passes && a.tokens; ++pass) {
    if (a.digit_bits) {
      if (a.tokens <= kMostRecounted) {
        hipLaunchKernelGGL(sort_place_kernel<false>, dim3(a.tiles), dim3(1024), 0, stream, a, pass);
      } else {
        hipLaunchKernelGGL(sort_tile_counts_kernel, dim3(a.tiles), dim3(kPlaceTile), 0, stream, a,
                           pass);
        hipLaunchKernelGGL(sort_place_kernel<true>, dim3(a.tiles), dim3(1024), 0, stream, a, pass);
      }
      continue;
    }
    hipLaunchKernelGGL(sort_count_kernel, dim3(a.tiles), dim3(kSortTile), 0, stream, a, pass);
    hipLaunchKernelGGL(sort_scan_kernel, dim3(kDigits), wg, 0, stream, a);
    hipLaunchKernelGGL(sort_scatter_kernel, dim3(a.tiles), dim3(kSortTile), 0, stream, a, pass);
  }
  const unsigned sums = (unsigned)((a.chunks + per - 1) / per * cblocks);
  const unsigned zeros = (unsigned)(((long long)a.rows + 4 * kZeroRows - 1) / (4 * kZeroRows));
  constexpr bool kWide = sizeof(T) * VW == 16;
  const auto sum = a.lanes_log2 < 6         ? embedding_sum_kernel<T, VW, false, false>
                   : kWide && a.past_caches ? embedding_sum_kernel<T, VW, true, kWide>
                                            : embedding_sum_kernel<T, VW, true, false>;
  hipLaunchKernelGGL(sum, dim3(sums + zeros), wg, 0, stream, a, cblocks, sums);
  if (a.chunks > 1) {
    // four columns a lane: a row with most of the tokens has more workgroups then
    constexpr int kJoin = VW < 4 ? VW : 4;
    const int blocks = (a.dim / kJoin + 63) / 64;
    hipLaunchKernelGGL((embedding_join_kernel<T, kJoin>), dim3((a.chunks + 15) / 16 * blocks),
                       dim3(1024), 0, stream, a, blocks);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbedArgs& a, int dtype, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    return vec == 8   ? launch_lookup<uint16_t, 8>(a, stream)
           : vec == 4 ? launch_lookup<uint16_t, 4>(a, stream)
           : vec == 2 ? launch_lookup<uint16_t, 2>(a, stream)
                      : launch_lookup<uint16_t, 1>(a, stream);
  return vec == 4   ? launch_lookup<uint32_t, 4>(a, stream)
         : vec == 2 ? launch_lookup<uint32_t, 2>(a, stream)
                    : launch_lookup<uint32_t, 1>(a, stream);
}

hipError_t launch_embedding_grad(const EmbedGradArgs& a, int dtype, int vec, hipStream_t stream) {
  if (dtype == HUGE2_BF16)
    return vec == 8   ? launch_grad<uint16_t, 8>(a, stream)
           : vec == 4 ? launch_grad<uint16_t, 4>(a, stream)
           : vec == 2 ? launch_grad<uint16_t, 2>(a, stream)
                      : launch_grad<uint16_t, 1>(a, stream);
  return vec == 4   ? launch_grad<uint32_t, 4>(a, stream)
         : vec == 2 ? launch_grad<uint32_t, 2>(a, stream)
                    : launch_grad<uint32_t, 1>(a, stream);
}

}  // namespace huge2
