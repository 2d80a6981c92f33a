// train.cpp -- the C ABI of the operators around the convolutions (declared in
// include/huge2_train.h): checks, plans, workspaces.
#include "huge2_train.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>
#include <new>
#include <numeric>
#include <vector>

#include "kernels.hpp"
#include "train.hpp"

using namespace huge2;

enum class NormForm { kSlab, kRun, kGeneral };

struct huge2_norm_plan {
  huge2_norm_desc desc;
  int vec;  // elements of a load
  NormArgs args[2];  // forward, gradient
  NormForm form[2];
  void* ws;
  char kernel_name[2][96];
};

struct huge2_embedding_grad_plan {
  huge2_embedding_desc desc;
  int64_t max_tokens;
  int vec, lanes_log2;
  void* ws;
  char kernel_name[2][48];  // few tokens, many
};

struct huge2_adamw_plan {
  struct Launch {
    int tensor, tensors;
    size_t work, works;
  };
  int state_bits;
  int count;
  bool past_caches;
  std::vector<Launch> launches;
  void* table;  // AdamTensorDev [count], then uint2 [works]
  size_t works_at;
  std::vector<size_t> grad_bytes;         // [count]
  std::vector<uintptr_t> begins, ends;    // of what a step writes, in ascending order
};

namespace {

// HUGE2_FAULT=alloc, launch: as in capi.cpp (tests of the error paths).
bool fault(const char* what) {
  const char* f = std::getenv("HUGE2_FAULT");
  return f && std::strcmp(f, what) == 0;
}

bool aligned(const void* p, size_t to = 16) { return ((uintptr_t)p & (to - 1)) == 0; }
bool bad(const void* p, size_t to = 16) { return !p || !aligned(p, to); }
struct Span {
  const void* p;
  size_t bytes;
};
bool overlap(const Span& a, const Span& b) {
  return a.p && b.p && (uintptr_t)a.p < (uintptr_t)b.p + b.bytes &&
         (uintptr_t)b.p < (uintptr_t)a.p + a.bytes;
}
// Whether what a call writes overlaps what it reads, or another thing that it writes.
bool overlaps(std::initializer_list<Span> writes, std::initializer_list<Span> reads) {
  for (const Span* w = writes.begin(); w != writes.end(); ++w) {
    for (const Span* o = writes.begin(); o != w; ++o)
      if (overlap(*w, *o)) return true;
    for (const Span& r : reads)
      if (overlap(*w, r)) return true;
  }
  return false;
}
bool is_dtype(int d) { return d == HUGE2_F32 || d == HUGE2_BF16; }
int elem_size(int dtype) { return dtype == HUGE2_BF16 ? 2 : 4; }
size_t round256(size_t v) { return (v + 255) / 256 * 256; }
int log2_ceil(long long v) {
  int l = 0;
  while ((1ll << l) < v) ++l;
  return l;
}

// The widest load of the type that divides a run of `len` elements: 16 bytes, 4
// or one element.
int vector_width(int dtype, long long len) {
  const int full = 16 / elem_size(dtype);
  if (len % full == 0) return full;
  return dtype == HUGE2_BF16 && len % 2 == 0 ? 2 : 1;
}

// A result that fills much of the 256 MB Infinity Cache is stored past it; a smaller
// one stays there for the layer that reads it.
bool streams(size_t bytes) { return bytes >= (size_t)64 << 20; }

huge2_status device_alloc(void** out, size_t bytes) {
  *out = nullptr;
  if (bytes == 0) return HUGE2_OK;
  if (fault("alloc")) return HUGE2_ERR_ALLOC;
  if (hipMalloc(out, bytes) == hipSuccess) return HUGE2_OK;
  (void)hipGetLastError();
  (void)huge2_plan_destroy(nullptr);  // what the one-shot calls keep
  if (hipMalloc(out, bytes) == hipSuccess) return HUGE2_OK;
  (void)hipGetLastError();
  *out = nullptr;
  return HUGE2_ERR_ALLOC;
}

huge2_status device_free(void* p) {
  if (p && hipFree(p) != hipSuccess) {
    (void)hipGetLastError();
    return HUGE2_ERR_HIP;
  }
  return HUGE2_OK;
}

huge2_status launched(hipError_t e) {
  if (e == hipSuccess) return HUGE2_OK;
  (void)hipGetLastError();
  return HUGE2_ERR_HIP;
}

// ---- group norm -----------------------------------------------------------------

bool valid(const huge2_norm_desc& d) {
  return d.n >= 1 && d.c >= 1 && d.h >= 1 && d.w >= 1 && d.groups >= 1 && d.c % d.groups == 0 &&
         (d.layout == HUGE2_NCHW || d.layout == HUGE2_NHWC) && is_dtype(d.dtype) &&
         d.activation >= HUGE2_NORM_NONE && d.activation <= HUGE2_NORM_SILU &&
         std::isfinite(d.eps) && d.eps > 0.f;
}

size_t norm_bytes(const huge2_norm_desc& d) {
  return (size_t)d.n * d.c * d.h * d.w * elem_size(d.dtype);
}

// NHWC slabs are whole groups and whole vectors of channels; the workgroup's most
// threads, and what follows from channels and threads.  (The slab_ and run_ functions
// return false where their form does not fit.)
int slab_threads(const NormArgs& a, int vec, bool grad, int lanes) {
  // entries of 8 bytes a channel stay under 64 KB of LDS
  return vec == 8 && (grad ? lanes >= 64 : a.span != 0) ? 512 : 1024;
}
void slab_set(NormArgs* a, int vec, bool grad, int c, int threads) {
  const int lanes = 1 << log2_ceil(c / vec), groups = c / a->d;
  a->slab_c = c;
  a->lanes_log2 = log2_ceil(lanes);
  a->cblocks = (a->c + c - 1) / c;
  a->threads = threads;
  a->rows_log2 = log2_ceil(threads / lanes);
  a->join_log2 = 0;
  while (a->join_log2 < 6 && (2 << a->join_log2) * groups <= threads) ++a->join_log2;
  division_magic((uint32_t)(a->span ? a->d : a->d / vec), &a->dl_mul, &a->dl_shift);
  const int entries = grad ? threads * vec / (lanes <= 32 ? 2 : 1) + std::max(threads, lanes * vec)
                           : threads * (a->span ? vec : 1) + groups;
  a->lds_bytes = entries * (int)sizeof(float2);
}

// Slabs of all pixels, held in registers: 64 bytes of a pixel where that fits, and twice
// as many again while there are two workgroups for each compute unit all the same (64 images
// of 8x8x2048 bf16: 512 bytes).
bool slab_nhwc(NormArgs* a, int esz, int vec, bool grad) {
  const int base = std::lcm(a->d, vec);
  a->span = a->d % vec != 0;
  const int most = slab_most(vec, grad, a->span != 0);
  const auto slots = [&](int lanes, int threads) {
    const int rows = threads / lanes;
    return ((long long)a->hw + rows - 1) / rows;  // (hw may be 2^31 - 1)
  };
  const auto lanes_of = [&](int c) { return 1 << log2_ceil(c / vec); };
  const auto fits = [&](long long c) {
    if (c > a->c || c / vec > 1024) return false;
    const int lanes = lanes_of((int)c), most_threads = slab_threads(*a, vec, grad, lanes);
    return lanes <= most_threads && slots(lanes, most_threads) <= most;
  };
  if (!fits(base)) return false;
  int c = base;
  while (fits(2ll * c) && (c * esz < 64 || (long long)a->n * ((a->c + 2 * c - 1) / (2 * c)) >= 512))
    c *= 2;
  const int lanes = lanes_of(c), most_threads = slab_threads(*a, vec, grad, lanes);
  int threads = std::max(64, lanes);
  const long long slabs = (long long)a->n * ((a->c + c - 1) / c);
  while (threads < most_threads &&
         (slots(lanes, threads) > most ||
          (slots(lanes, threads) > 4 && slabs * (threads / 32) <= 8192)))
    threads *= 2;
  slab_set(a, vec, grad, c, threads);
  if (!launchable(slabs, threads)) return false;
  a->slabs = (int)slabs;
  a->slots = (int)slots(lanes, threads);
  a->chunks = 1;
  a->chunk_len = a->hw;
  return true;
}

// Slabs cut into runs of pixels: 64 bytes of a pixel, up to 512 while there are two
// workgroups for each compute unit all the same (every workgroup of the second pass
// joins all runs of its groups: few groups, few runs).  Of runs as many as fill the
// compute units with the waves that their registers allow, at least four pixels a
// thread.  The gradient's sums are 8 bytes for each channel of a run: there wide groups
// have four pixels side by side, and a run 32 pixels where that leaves a workgroup for
// each compute unit (39 x 3x59x1344 with 4 pixels a run 53 us, so 40; the forward is
// slower with the larger workgroups, 32 against 28 us for 13 x 41x29x1216).
bool run_nhwc(NormArgs* a, int esz, int vec, bool grad) {
  const int base = std::lcm(a->d, vec);
  a->span = a->d % vec != 0;
  if (base > a->c || base / vec > 1024) return false;
  const auto lanes_of = [&](int c) { return 1 << log2_ceil(c / vec); };
  const auto threads_of = [&](int c) {
    const int lanes = lanes_of(c), most = slab_threads(*a, vec, grad, lanes);
    return std::max(lanes, std::min(std::max(256, (grad ? 4 : 1) * lanes), most));
  };
  const auto units_of = [&](int c) { return (long long)a->n * ((a->c + c - 1) / c); };
  const auto most_chunks = [&](int c) {
    const long long rows = threads_of(c) / lanes_of(c), units = units_of(c);
    const long long most = grad ? std::max((a->hw + 31ll) / 32, 256 / units) : 1 << 20;
    return std::min({std::max(64ll, (512 + units - 1) / units), most,
                     (a->hw + 4 * rows - 1) / (4 * rows)});
  };
  int c = base;
  while (2ll * c <= a->c && 2 * c / vec <= 64 && c * esz < 512 &&
         (c * esz < 64 || units_of(2 * c) * std::min(64ll, most_chunks(2 * c)) >= 512))
    c *= 2;
  if (lanes_of(c) > slab_threads(*a, vec, grad, lanes_of(c))) return false;
  slab_set(a, vec, grad, c, threads_of(c));
  const long long units = units_of(c), waves = units * (a->threads / 64);
  const long long chunks = std::min(((grad ? 4096 : 8192) + waves - 1) / waves, most_chunks(c));
  a->chunk_len = (int)((a->hw + chunks - 1) / chunks);
  a->chunks = (int)(((long long)a->hw + a->chunk_len - 1) / a->chunk_len);
  if (!launchable(units * a->chunks + a->c, a->threads)) return false;
  a->slabs = (int)(units * a->chunks);
  a->slots = 0;
  return true;
}

// In NCHW a slab is a group: planes of up to 64 lanes, as many planes side by side
// as leave four vectors a thread, or more where the waves then run at once (8192 of
// them: 57x2 pixels, 50 channels a group, 640 groups, gradient: 21.5 -> 19 us).
bool slab_nchw(NormArgs* a, int vec, bool grad) {
  const int vecs = a->hw / vec, lanes = 1 << std::min(6, log2_ceil(vecs));
  const int along = (int)(((long long)vecs + lanes - 1) / lanes), most = slab_most(vec, grad, false);
  if (along > most) return false;
  int threads = 64;
  const auto slots = [&] {
    const int planes = threads / lanes;
    return (long long)along * ((a->d + planes - 1) / planes);
  };
  while (threads < 1024 && threads / lanes < a->d &&
         (slots() > most || (slots() > 4 && (long long)a->n * a->groups * (threads / 32) <= 8192)))
    threads *= 2;
  if (slots() > most || !launchable((long long)a->n * a->groups, threads)) return false;
  a->lanes_log2 = log2_ceil(lanes);
  a->along = along;
  a->threads = threads;
  a->slots = (int)slots();
  a->slabs = a->n * a->groups;
  a->chunks = 1;
  return true;
}

// Where the maps of all images together are small, the gradient's launch also has
// workgroups that add up dgamma and dbeta from x and dy once more, 4096 vectors of each
// at most, 16 a thread (32 images of 8x8x512 in NHWC, twice as much: 12.7 us and 9.3 with
// a launch behind), and all of them 16 MiB (64 images of 8x8x2048 in NCHW 17.8 and 19.5 us,
// fp32 33.8 and 27.4).  16 images of 8x8x512 in NHWC: 6.8 and 8.6 us; 4 of 4x4x512 3.9 and 7.
constexpr long long kDirectVectors = 4096;
constexpr size_t kDirectBytes = (size_t)16 << 20;
void direct_nhwc(NormArgs* a, int vec) {
  const int lanes = 1 << a->lanes_log2, most_threads = slab_threads(*a, vec, true, lanes);
  const long long vectors = (long long)a->n * a->hw * lanes;
  int threads = a->threads;
  while (threads < std::min(256, most_threads) && vectors > threads * 8 &&
         (long long)a->slabs * (threads / 32) <= 2048)
    threads *= 2;
  if (vectors > std::min(kDirectVectors, threads * 16ll) ||
      !launchable((long long)a->slabs + a->cblocks, threads))
    return;
  if (threads != a->threads) {
    slab_set(a, vec, true, a->slab_c, threads);
    a->slots = (a->hw + threads / lanes - 1) / (threads / lanes);
  }
  a->direct = a->cblocks;
  division_magic((uint32_t)a->hw, &a->px_mul, &a->px_shift);
}
void direct_nchw(NormArgs* a, int vec) {
  const long long vectors = (long long)a->n * (a->hw / vec);  // of a channel
  a->direct_log2 = std::min(6, log2_ceil((vectors + 3) / 4));
  const int channels = a->threads >> a->direct_log2, blocks = (a->c + channels - 1) / channels;
  if (vectors * channels > std::min(kDirectVectors, a->threads * 16ll) ||
      !launchable((long long)a->slabs + blocks, a->threads))
    return;
  a->direct = blocks;
  division_magic((uint32_t)(a->hw / vec), &a->px_mul, &a->px_shift);
}

// Slabs too few to fill the compute units, whose two launches another form fills: the
// forward where a thread has many vectors, so that a launch more costs less (NHWC: 2 images
// of 38x53x768 bf16 16.2 -> 9.8 us, 8 of 42x28x384 12.1 -> 10.3; with less than 10 vectors
// 7 to 9 either way; NCHW: 2 of 60x46x60, 4 groups, 11.5 -> 7.6), the gradient where it has
// a launch for dgamma and dbeta anyway (NHWC: 6 images of 27x87x128 15.6 -> 10.8; NCHW: 8
// of 64x40x40 12.9 -> 9.2, 4 of 816x26x14 fp32 15.4 -> 10.5).  With a slab for each compute
// unit the slabs win: 64 of 32x32x128 17.3 and 24; but not with half a memory line of each
// pixel: 54 of 29x79x64 fp32 by 32 bytes 37.7 and 32.4, 64 of 64x64x64 bf16 56.3 and 38.3.
// (The forward, which holds half as much, wins with 32 bytes all the same: 64 of 64x64x64 in
// 16 groups bf16 25.5 and 29.9, 64 of 64x64x128 in 32 38.4 and 45.0.)
bool weak_slabs(const NormArgs& a, bool nhwc, int esz, int vec, bool grad) {
  if (grad && nhwc && a.slab_c * esz < 64 && a.slab_c < a.c) return !a.direct;
  if (a.slabs >= 256) return false;
  if (!grad)
    return vec * esz == 16 && (nhwc ? a.slots >= 10 : a.slots * vec >= 48 && a.slabs < 64);
  if (a.direct || (nhwc && a.threads < 1024)) return false;
  return a.n > 1 || (a.slots > 4 && a.slabs < 64);
}

// The general form.  Runs of pixels: enough workgroups for eight a compute unit,
// each run long enough that its sums are few next to its pixels.  False where there
// are too many.
bool norm_runs(NormArgs* a, bool nhwc, int vec) {
  long long chunks, units;
  const long long hw = a->hw;
  if (nhwc) {
    const int vecs = a->c / vec;
    a->lanes_log2 = std::min(6, log2_ceil(vecs));
    a->cblocks = (vecs + (1 << a->lanes_log2) - 1) >> a->lanes_log2;
    units = (long long)a->n * a->cblocks;
    chunks = std::min((2048 + units - 1) / units, (hw + 63) / 64);
  } else {
    const long long vecs = hw / vec;
    units = (long long)a->n * a->c;
    chunks = std::max(std::min((8192 + units - 1) / units, (vecs + 255) / 256),
                      (vecs + 1023) / 1024);
    a->lanes_log2 = std::min(6, log2_ceil((vecs + chunks - 1) / chunks));
  }
  a->chunk_len = (int)((hw + chunks - 1) / chunks);
  if (!nhwc) a->chunk_len = (a->chunk_len + vec - 1) / vec * vec;
  a->chunks = (int)((hw + a->chunk_len - 1) / a->chunk_len);
  const long long parts = ((long long)a->d * a->chunks << a->lanes_log2) / 256 + 1;
  return launchable(units * a->chunks, 256) &&
         launchable((long long)a->n * a->groups * parts + a->c, 256);
}

huge2_status norm_create(huge2_norm_plan** out, const huge2_norm_desc* desc) {
  if (!out) return HUGE2_ERR_INVALID_ARG;
  *out = nullptr;
  if (!desc || !valid(*desc)) return HUGE2_ERR_INVALID_ARG;
  const huge2_norm_desc& d = *desc;
  const long long hw = (long long)d.h * d.w;
  if (hw >= (1ll << 31) || hw * d.c >= (1ll << 31) || hw * d.c * d.n >= (1ll << 40))
    return HUGE2_ERR_UNSUPPORTED;
  const bool nhwc = d.layout == HUGE2_NHWC;
  NormArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n = d.n, a.c = d.c, a.hw = (int)hw, a.groups = d.groups, a.d = d.c / d.groups;
  a.act = d.activation;
  a.eps = d.eps;
  const int vec = vector_width(d.dtype, nhwc ? d.c : hw);
  division_magic((uint32_t)a.d, &a.d_mul, &a.d_shift);
  if (!launchable(d.c / 16 + 1, 256)) return HUGE2_ERR_UNSUPPORTED;
  huge2_norm_plan* p = new (std::nothrow) huge2_norm_plan();
  if (!p) return HUGE2_ERR_ALLOC;
  p->desc = d;
  p->vec = vec;
  size_t part_b = 0, gpart_b = 0;
  for (int g = 0; g < 2; ++g) {
    NormArgs& b = p->args[g];
    const int esz = elem_size(d.dtype);
    b = a;
    const auto fit = [&](auto&& form) {
      b = a;
      return form();
    };
    if (nhwc ? fit([&] { return slab_nhwc(&b, esz, vec, g != 0); })
             : fit([&] { return slab_nchw(&b, vec, g != 0); }))
      p->form[g] = NormForm::kSlab;
    else if (nhwc && fit([&] { return run_nhwc(&b, esz, vec, g != 0); }))
      p->form[g] = NormForm::kRun;
    else if (fit([&] { return norm_runs(&b, nhwc, vec); }))
      p->form[g] = NormForm::kGeneral;
    else {
      delete p;
      return HUGE2_ERR_UNSUPPORTED;
    }
    if (g && p->form[g] == NormForm::kSlab && d.n > 1 && norm_bytes(d) <= kDirectBytes)
      nhwc ? direct_nhwc(&b, vec) : direct_nchw(&b, vec);
    if (p->form[g] == NormForm::kSlab && weak_slabs(b, nhwc, esz, vec, g != 0)) {
      const NormArgs slabs = b;
      if (fit([&] { return nhwc ? run_nhwc(&b, esz, vec, g != 0) : norm_runs(&b, false, vec); }))
        p->form[g] = nhwc ? NormForm::kRun : NormForm::kGeneral;
      else
        b = slabs;
    }
    // 64x64x2048 batch 8: 72 against 82 us, since the first pass then need not write the
    // last call's result back.  Not in pieces of less than 64 bytes: 176 against 66 us
    // with 16 bytes of a pixel to a workgroup; and in NCHW not by less than 16 bytes: 104
    // against 100 us for 32 images of 300x31x123 fp32 (NHWC, 250 and 251 channels: 53 against
    // 57 by 4 bytes, bf16, and 78 against 82, fp32).
    b.stream = streams(norm_bytes(d)) &&
               (!nhwc ? vec * esz == 16
                      : p->form[g] == NormForm::kGeneral || b.slab_c * esz >= 64);
    if (g || p->form[g] == NormForm::kGeneral)
      part_b = std::max(part_b, round256((size_t)d.n * b.chunks * d.c * sizeof(float2)));
    if (p->form[g] == NormForm::kRun)
      gpart_b = std::max(gpart_b, round256((size_t)d.n * b.chunks * d.groups * sizeof(float2)));
    const char* const layout = nhwc ? "nhwc" : "nchw";
    char* const name = p->kernel_name[g];
    const size_t room = sizeof(p->kernel_name[g]);
    if (p->form[g] == NormForm::kSlab)
      std::snprintf(name, room, "norm_slab_%s%s_kernel v%d t%d r%d", g && nhwc ? "grad_" : "",
                    layout, vec, b.threads, b.slots);
    else if (p->form[g] == NormForm::kRun)
      std::snprintf(name, room, "norm_run_%snhwc_kernel v%d t%d k%d", g ? "grad_" : "", vec,
                    b.threads, b.chunks);
    else
      std::snprintf(name, room, "norm_sums_%s_kernel v%d k%d", layout, vec, b.chunks);
  }
  const size_t group_b = round256((size_t)d.n * d.groups * sizeof(float2));
  const huge2_status st = device_alloc(&p->ws, part_b + gpart_b + group_b);
  if (st != HUGE2_OK) {
    delete p;
    return st;
  }
  for (NormArgs& b : p->args) {
    b.part = (float2*)p->ws;
    b.gpart = (float2*)((char*)p->ws + part_b);
    b.coef = (float2*)((char*)p->ws + part_b + gpart_b);
    b.stats_out = (float*)b.coef;  // where the caller has no place for them
  }
  *out = p;
  return HUGE2_OK;
}

huge2_status norm_run(const huge2_norm_plan* p, const void* x, const float* gamma,
                      const float* beta, void* y, float* stats, hipStream_t stream) {
  if (!p || bad(x) || bad(y) || !aligned(gamma) || !aligned(beta) || !aligned(stats))
    return HUGE2_ERR_INVALID_ARG;
  const huge2_norm_desc& d = p->desc;
  const size_t bytes = norm_bytes(d), params = (size_t)d.c * sizeof(float);
  const size_t groups = (size_t)d.n * d.groups * sizeof(float2);
  if (overlaps({{y, bytes}, {stats, groups}}, {{x, bytes}, {gamma, params}, {beta, params}}))
    return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  NormArgs a = p->args[0];
  a.x = x, a.gamma = gamma, a.beta = beta, a.out = y;
  if (stats) a.stats_out = stats;
  const int nhwc = d.layout == HUGE2_NHWC;
  if (p->form[0] == NormForm::kGeneral)
    return launched(launch_norm(a, d.dtype, nhwc, p->vec, stream));
  return launched((nhwc ? launch_norm_nhwc : launch_norm_nchw)(a, d.dtype, p->vec, stream));
}

huge2_status norm_grad_run(const huge2_norm_plan* p, const void* x, const void* dy,
                           const float* stats, const float* gamma, const float* beta, void* dx,
                           float* dgamma, float* dbeta, hipStream_t stream) {
  if (!p || bad(x) || bad(dy) || bad(dx) || bad(stats) || !aligned(gamma) || !aligned(beta) ||
      !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return HUGE2_ERR_INVALID_ARG;
  const huge2_norm_desc& d = p->desc;
  const size_t bytes = norm_bytes(d), params = (size_t)d.c * sizeof(float);
  const size_t groups = (size_t)d.n * d.groups * sizeof(float2);
  if (overlaps({{dx, bytes}, {dgamma, params}, {dbeta, params}},
               {{x, bytes}, {dy, bytes}, {stats, groups}, {gamma, params}, {beta, params}}))
    return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  NormArgs a = p->args[1];
  a.x = x, a.dy = dy, a.stats = stats, a.gamma = gamma, a.beta = beta, a.out = dx;
  a.dgamma = dgamma, a.dbeta = dbeta;
  const int nhwc = d.layout == HUGE2_NHWC;
  if (p->form[1] == NormForm::kGeneral)
    return launched(launch_norm_grad(a, d.dtype, nhwc, p->vec, stream));
  return launched(
      (nhwc ? launch_norm_grad_nhwc : launch_norm_grad_nchw)(a, d.dtype, p->vec, stream));
}

// ---- embedding --------------------------------------------------------------------

bool valid(const huge2_embedding_desc& d) {
  return d.rows >= 1 && d.dim >= 1 && is_dtype(d.dtype) && (d.id_bits == 32 || d.id_bits == 64);
}
// The widest load that divides a row.  (26813 rows of 1218 fp32, 4202 ids: by 8 bytes 55 us,
// by 4 70, the gradient 63 and 79; of 1220 bf16 29 and 34, 43 and 52.)
int embed_vector(int dtype, int dim) {
  int vec = 16 / elem_size(dtype);
  while (dim % vec) vec /= 2;
  return vec;
}
// Rows of lanes (up to a workgroup) side by side on a row of the table.
int embed_lanes_log2(const huge2_embedding_desc& d, int vec) {
  return std::min(8, log2_ceil(d.dim / vec));
}
bool embed_fits(const huge2_embedding_desc& d) {
  return (long long)d.dim * elem_size(d.dtype) < (1ll << 31) && d.rows < INT_MAX;
}

huge2_status embed_run(const huge2_embedding_desc* desc, const void* ids, int64_t tokens,
                       const void* table, void* y, hipStream_t stream) {
  if (!desc || !valid(*desc) || tokens < 0) return HUGE2_ERR_INVALID_ARG;
  const huge2_embedding_desc& d = *desc;
  if (!embed_fits(d) || tokens >= (1ll << 31)) return HUGE2_ERR_UNSUPPORTED;
  if (tokens == 0) return HUGE2_OK;
  if (bad(ids, d.id_bits / 8) || bad(table) || bad(y)) return HUGE2_ERR_INVALID_ARG;
  const size_t row_b = (size_t)d.dim * elem_size(d.dtype);
  if (overlaps({{y, row_b * tokens}},
               {{table, row_b * d.rows}, {ids, (size_t)tokens * (d.id_bits / 8)}}))
    return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  const int vec = embed_vector(d.dtype, d.dim);
  EmbedArgs a;
  a.ids = ids, a.table = table, a.y = y, a.tokens = tokens;
  a.rows = d.rows, a.dim = d.dim, a.id64 = d.id_bits == 64, a.scale = d.scale;
  a.lanes_log2 = embed_lanes_log2(d, vec);
  // Results of 16 MiB and more are stored past the caches, by 4 bytes and more a lane (26813
  // rows of 1217 fp32 70 -> 48 us).  65536 rows of bf16, the table and the last result in the
  // caches, and out of them: of 128 (16 MiB) 6.2 -> 5.0 and 7.4 -> 6.0 us, of 256 10.4 -> 8.1
  // and 10.6 -> 9.9, of 512 19.3 -> 16.7 and 19.7 -> 17.9; together with a kernel that reads
  // them 18.9 -> 18.6, 25.5 -> 25.5, 40.6 -> 40.0; of 64 no difference.
  a.stream = row_b * tokens >= (size_t)16 << 20;
  return launched(launch_embedding(a, d.dtype, vec, stream));
}

// Sorted tokens of a chunk: 16, or where tokens abound and the parts would take
// much memory 64.
int embed_chunk_len(int64_t max_tokens) { return max_tokens > (1 << 17) ? 4 * kChunk : kChunk; }

// Counts of digits: those of the placed sorts' tiles, or of the long sorts'.
size_t embed_hist_bytes(int64_t max_tokens) {
  const size_t placed = (std::min<int64_t>(max_tokens, kMostPlaced) + kPlaceTile - 1) / kPlaceTile;
  const size_t tiles = max_tokens > kMostPlaced ? (max_tokens + kSortTile - 1) / kSortTile : 0;
  return std::max(placed * kMostDigits, (tiles + 1) * kDigits) * 4;
}

huge2_status embed_grad_create(huge2_embedding_grad_plan** out, const huge2_embedding_desc* desc,
                               int64_t max_tokens) {
  if (!out) return HUGE2_ERR_INVALID_ARG;
  *out = nullptr;
  if (!desc || !valid(*desc) || max_tokens < 0) return HUGE2_ERR_INVALID_ARG;
  if (!embed_fits(*desc) || max_tokens >= (1ll << 30)) return HUGE2_ERR_UNSUPPORTED;
  huge2_embedding_grad_plan* p = new (std::nothrow) huge2_embedding_grad_plan();
  if (!p) return HUGE2_ERR_ALLOC;
  p->desc = *desc;
  p->max_tokens = max_tokens;
  p->vec = embed_vector(desc->dtype, desc->dim);
  p->lanes_log2 = std::min(6, log2_ceil(desc->dim / p->vec));
  const int chunk = embed_chunk_len(max_tokens);
  const long long chunks = (max_tokens + chunk - 1) / chunk, vecs = desc->dim / p->vec;
  const int per = 256 >> p->lanes_log2;
  if (!launchable((chunks + per - 1) / per * ((vecs + 63) / 64) + desc->rows / 64 + 1, 256) ||
      !launchable((chunks + 15) / 16 * ((desc->dim / std::min(p->vec, 4) + 63) / 64), 1024) ||
      !launchable(desc->rows / kFewRows + 1 + kMostFew, kFewThreads)) {
    delete p;
    return HUGE2_ERR_UNSUPPORTED;
  }
  const size_t bytes = max_tokens == 0
                           ? 0
                           : 4 * round256(max_tokens * 4) + round256(embed_hist_bytes(max_tokens)) +
                                 (max_tokens + chunk - 1) / chunk * 2 * (size_t)desc->dim * 4;
  const huge2_status st = device_alloc(&p->ws, bytes);
  if (st != HUGE2_OK) {
    delete p;
    return st;
  }
  for (int many = 0; many < 2; ++many)
    std::snprintf(p->kernel_name[many], sizeof(p->kernel_name[many]), "embedding_%s_kernel v%d",
                  many ? "sum" : "few", p->vec);
  *out = p;
  return HUGE2_OK;
}

huge2_status embed_grad_run(const huge2_embedding_grad_plan* p, const void* ids, int64_t tokens,
                            const void* dy, void* dtable, hipStream_t stream) {
  if (!p || tokens < 0 || tokens > p->max_tokens || bad(dtable)) return HUGE2_ERR_INVALID_ARG;
  const huge2_embedding_desc& d = p->desc;
  const size_t row_b = (size_t)d.dim * elem_size(d.dtype);
  if (tokens && (bad(ids, d.id_bits / 8) || bad(dy) ||
                 overlaps({{dtable, row_b * d.rows}},
                          {{dy, row_b * tokens}, {ids, (size_t)tokens * (d.id_bits / 8)}})))
    return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  EmbedGradArgs a;
  std::memset(&a, 0, sizeof(a));
  a.ids = ids, a.dy = dy, a.dtable = dtable;
  a.tokens = (int)tokens, a.rows = d.rows, a.dim = d.dim, a.id64 = d.id_bits == 64;
  a.scale = d.scale;
  a.lanes_log2 = p->lanes_log2;
  // dy is read once, and the table's gradient finds more room in the caches.  bf16, inputs
  // out of the caches, and with dy written before and an AdamW step behind: 65536 tokens of
  // 512 (64 MiB), 30000 ids 51.8 -> 47.1 and 136 -> 134 us; 32768 of 1024, 40000 ids
  // 60 -> 50.4 and 250 -> 245; 131072 of 1024, 30000 ids 120 -> 110 and 334 -> 322; 32 MiB
  // and 16 MiB no difference.
  a.past_caches = streams(row_b * tokens);
  const int bits = std::max(2, log2_ceil((long long)d.rows + 1));  // keys are ids, and `rows`
  const int tile = tokens <= kMostPlaced ? kPlaceTile : kSortTile;
  a.tiles = (int)((tokens + tile - 1) / tile);
  if (tokens <= kMostPlaced) {
    a.passes = (bits + kMostDigitBits - 1) / kMostDigitBits;
    a.digit_bits = (bits + a.passes - 1) / a.passes;
  } else {
    a.passes = (bits + kDigitBits - 1) / kDigitBits;
  }
  a.chunk_len = embed_chunk_len(p->max_tokens);
  a.chunks = (int)((tokens + a.chunk_len - 1) / a.chunk_len);
  char* at = (char*)p->ws;
  const size_t list = round256(p->max_tokens * 4);
  for (int k = 0; k < 2; ++k) {
    a.key[k] = (int*)(at + 2 * k * list);
    a.token[k] = (int*)(at + (2 * k + 1) * list);
  }
  a.hist = (int*)(at + 4 * list);
  a.part = (float*)(at + 4 * list + round256(embed_hist_bytes(p->max_tokens)));
  return launched(launch_embedding_grad(a, d.dtype, p->vec, stream));
}

// ---- AdamW --------------------------------------------------------------------------

bool valid(const huge2_adamw_tensor& t, int bits) {
  if (t.count < 0 || !is_dtype(t.dtype) || !is_dtype(t.grad_dtype) ||
      !std::isfinite(t.weight_decay) || t.weight_decay < 0.f)
    return false;
  if (bits == 32 ? t.m_scale || t.v_scale : !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))
    return false;
  if (!aligned(t.param) || !aligned(t.m) || !aligned(t.v) || !aligned(t.copy)) return false;
  if (t.count == 0) return true;
  return t.param && t.m && t.v && (bits == 32 || (t.m_scale && t.v_scale));
}

// What a step writes, in order of address; false where two of them overlap (each must be one
// tensor's own: two workgroups would update it at once).
bool adamw_spans(const huge2_adamw_tensor* tensors, int count, int bits,
                 std::vector<uintptr_t>* begins, std::vector<uintptr_t>* ends) {
  std::vector<Span> spans;
  for (int i = 0; i < count; ++i) {
    const huge2_adamw_tensor& t = tensors[i];
    const size_t n = t.count, state = bits == 32 ? n * sizeof(float) : n;
    const size_t scales = (n + kAdamBlock - 1) / kAdamBlock * sizeof(float);
    for (const Span& s : {Span{t.param, n * elem_size(t.dtype)}, Span{t.m, state}, Span{t.v, state},
                          Span{t.m_scale, scales}, Span{t.v_scale, scales}, Span{t.copy, n * 2}})
      if (s.p && s.bytes) spans.push_back(s);
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.p < b.p; });
  for (const Span& s : spans) {
    const uintptr_t begin = (uintptr_t)s.p;
    if (!ends->empty() && begin < ends->back()) return false;
    begins->push_back(begin);
    ends->push_back(begin + s.bytes);
  }
  return true;
}
// Whether any of them overlaps.  (A search without branches: 160 gradients among 960 spans
// take 1.6 us.)
bool adamw_writes(const huge2_adamw_plan& p, const void* at, size_t bytes) {
  const uintptr_t begin = (uintptr_t)at, end = begin + bytes;
  if (!at || !bytes || p.begins.empty()) return false;
  const uintptr_t* base = p.begins.data();  // comes to the last that begins before `end`
  for (size_t n = p.begins.size(); n > 1;) {
    const size_t half = n / 2;
    base += base[half] < end ? half : 0;
    n -= half;
  }
  return *base < end && p.ends[base - p.begins.data()] > begin;
}

huge2_status adamw_create(huge2_adamw_plan** out, const huge2_adamw_tensor* tensors, int count,
                          int state_bits, hipStream_t stream) {
  if (!out) return HUGE2_ERR_INVALID_ARG;
  *out = nullptr;
  if (count < 0 || (count && !tensors) || (state_bits != 32 && state_bits != 8))
    return HUGE2_ERR_INVALID_ARG;
  int64_t total = 0, bytes = 0;  // bytes: of fp32 parameters and moments
  for (int i = 0; i < count; ++i) {
    if (!valid(tensors[i], state_bits)) return HUGE2_ERR_INVALID_ARG;
    if (tensors[i].count >= (1ll << 40) || (total += tensors[i].count) >= (1ll << 40))
      return HUGE2_ERR_UNSUPPORTED;
    bytes += tensors[i].count *
             ((state_bits == 32 ? 8 : 0) + (tensors[i].dtype == HUGE2_F32 ? 4 : 0));
  }
  std::vector<uintptr_t> begins, ends;
  if (!adamw_spans(tensors, count, state_bits, &begins, &ends)) return HUGE2_ERR_INVALID_ARG;
  std::vector<size_t> grad_bytes(count);
  std::vector<AdamTensorDev> table(count);
  std::vector<uint2> works;
  std::vector<huge2_adamw_plan::Launch> launches;
  for (int i = 0; i < count; ++i) {
    const huge2_adamw_tensor& t = tensors[i];
    table[i] = {t.param,    t.m,       t.v,
                t.m_scale,  t.v_scale, t.copy,
                t.count,    t.dtype == HUGE2_BF16, t.grad_dtype == HUGE2_BF16,
                t.weight_decay, 0};
    grad_bytes[i] = (size_t)t.count * elem_size(t.grad_dtype);
    if (i % kAdamTensors == 0)
      launches.push_back({i, std::min(kAdamTensors, count - i), works.size(), 0});
    for (int64_t k = 0; k * adam_work(state_bits) < t.count; ++k)
      works.push_back(make_uint2(i % kAdamTensors, (unsigned)k));
    launches.back().works = works.size() - launches.back().work;
  }
  auto* p = new huge2_adamw_plan();
  p->state_bits = state_bits;
  p->count = count;
  // fp32 parameters, moments and gradients, within the caches and past them: 4 M (46 MiB)
  // 18.8 and 20.7 us, 6 M (69 MiB) 30.2 and 29.3, 8 M 42.8 and 37.7, 134 M 675 and 645
  p->past_caches = streams(bytes);
  p->launches = std::move(launches);
  p->grad_bytes = std::move(grad_bytes);
  p->begins = std::move(begins);
  p->ends = std::move(ends);
  p->works_at = round256(table.size() * sizeof(AdamTensorDev));
  std::vector<char> image(works.empty() ? 0 : p->works_at + works.size() * sizeof(uint2));
  if (!works.empty()) {
    std::memcpy(image.data(), table.data(), table.size() * sizeof(AdamTensorDev));
    std::memcpy(image.data() + p->works_at, works.data(), works.size() * sizeof(uint2));
  }
  huge2_status st = device_alloc(&p->table, image.size());
  if (st == HUGE2_OK && !image.empty() &&
      (hipMemcpyAsync(p->table, image.data(), image.size(), hipMemcpyHostToDevice, stream) !=
           hipSuccess ||
       hipStreamSynchronize(stream) != hipSuccess)) {
    (void)hipGetLastError();
    st = HUGE2_ERR_HIP;
  }
  if (st != HUGE2_OK) {
    (void)device_free(p->table);
    delete p;
    return st;
  }
  *out = p;
  return HUGE2_OK;
}

huge2_status adamw_run(const huge2_adamw_plan* p, const void* const* grads,
                       const huge2_adamw_options* o, const float* grad_scale, hipStream_t stream) {
  if (!p || !o || (p->count && !grads) || !aligned(grad_scale, 4)) return HUGE2_ERR_INVALID_ARG;
  const auto beta = [](double b) { return b >= 0 && b < 1 && (float)b < 1.f; };
  if (!std::isfinite((float)o->lr) || o->lr < 0 || !beta(o->beta1) || !beta(o->beta2) ||
      !std::isfinite((float)o->eps) || o->eps < 0x1p-126 || o->step < 1)
    return HUGE2_ERR_INVALID_ARG;
  for (int i = 0; i < p->count; ++i)
    if (!aligned(grads[i]) || adamw_writes(*p, grads[i], p->grad_bytes[i]))
      return HUGE2_ERR_INVALID_ARG;
  if (adamw_writes(*p, grad_scale, sizeof(float))) return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  AdamArgs a;
  std::memset(&a, 0, sizeof(a));
  a.grad_scale = grad_scale;
  a.beta1 = (float)o->beta1, a.beta2 = (float)o->beta2;
  a.rest1 = (float)(1 - o->beta1), a.rest2 = (float)(1 - o->beta2);
  a.lr = (float)o->lr, a.eps = (float)o->eps;
  a.step_size = (float)(o->lr / (1 - std::pow(o->beta1, (double)o->step)));
  a.root = (float)(1 / std::sqrt(1 - std::pow(o->beta2, (double)o->step)));
  for (const auto& l : p->launches) {
    if (l.works == 0) continue;
    std::memcpy(a.grads, grads + l.tensor, l.tensors * sizeof(void*));
    a.tensors = (const AdamTensorDev*)p->table + l.tensor;
    const size_t most = (1u << 24) - 1;  // of 256 threads: what a launch can have
    for (size_t w = 0; w < l.works; w += most) {
      a.works = (const uint2*)((const char*)p->table + p->works_at) + l.work + w;
      const huge2_status st =
          launched(launch_adamw(a, (unsigned)std::min(most, l.works - w), p->state_bits,
                                p->past_caches, stream));
      if (st != HUGE2_OK) return st;
    }
  }
  return HUGE2_OK;
}

}  // namespace

extern "C" {

huge2_status huge2_norm_plan_create(huge2_norm_plan** out, const huge2_norm_desc* desc) {
  try {
    return norm_create(out, desc);
  } catch (...) {
    return HUGE2_ERR_ALLOC;
  }
}

huge2_status huge2_norm_execute(const huge2_norm_plan* plan, const void* x, const float* gamma,
                                const float* beta, void* y, float* stats, void* hip_stream) {
  return norm_run(plan, x, gamma, beta, y, stats, (hipStream_t)hip_stream);
}

huge2_status huge2_norm_grad_execute(const huge2_norm_plan* plan, const void* x, const void* dy,
                                     const float* stats, const float* gamma, const float* beta,
                                     void* dx, float* dgamma, float* dbeta, void* hip_stream) {
  return norm_grad_run(plan, x, dy, stats, gamma, beta, dx, dgamma, dbeta,
                       (hipStream_t)hip_stream);
}

const char* huge2_norm_plan_kernel(const huge2_norm_plan* plan, int32_t grad) {
  return plan ? plan->kernel_name[grad != 0] : "";
}

huge2_status huge2_norm_plan_destroy(huge2_norm_plan* plan) {
  if (!plan) return HUGE2_OK;
  const huge2_status st = device_free(plan->ws);
  delete plan;
  return st;
}

huge2_status huge2_embedding(const huge2_embedding_desc* desc, const void* ids, int64_t tokens,
                             const void* table, void* y, void* hip_stream) {
  return embed_run(desc, ids, tokens, table, y, (hipStream_t)hip_stream);
}

huge2_status huge2_embedding_grad_plan_create(huge2_embedding_grad_plan** out,
                                              const huge2_embedding_desc* desc,
                                              int64_t max_tokens) {
  try {
    return embed_grad_create(out, desc, max_tokens);
  } catch (...) {
    return HUGE2_ERR_ALLOC;
  }
}

huge2_status huge2_embedding_grad_execute(const huge2_embedding_grad_plan* plan, const void* ids,
                                          int64_t tokens, const void* dy, void* dtable,
                                          void* hip_stream) {
  return embed_grad_run(plan, ids, tokens, dy, dtable, (hipStream_t)hip_stream);
}

const char* huge2_embedding_grad_plan_kernel(const huge2_embedding_grad_plan* plan,
                                             int64_t tokens) {
  return plan ? plan->kernel_name[tokens > kMostFew] : "";
}

huge2_status huge2_embedding_grad_plan_destroy(huge2_embedding_grad_plan* plan) {
  if (!plan) return HUGE2_OK;
  const huge2_status st = device_free(plan->ws);
  delete plan;
  return st;
}

huge2_status huge2_adamw_plan_create(huge2_adamw_plan** out, const huge2_adamw_tensor* tensors,
                                     int32_t count, int32_t state_bits, void* hip_stream) {
  try {
    return adamw_create(out, tensors, count, state_bits, (hipStream_t)hip_stream);
  } catch (...) {
    if (out) *out = nullptr;
    return HUGE2_ERR_ALLOC;
  }
}

huge2_status huge2_adamw_step(const huge2_adamw_plan* plan, const void* const* grads,
                              const huge2_adamw_options* options, const float* grad_scale,
                              void* hip_stream) {
  return adamw_run(plan, grads, options, grad_scale, (hipStream_t)hip_stream);
}

huge2_status huge2_adamw_plan_destroy(huge2_adamw_plan* plan) {
  if (!plan) return HUGE2_OK;
  const huge2_status st = device_free(plan->table);
  delete plan;
  return st;
}

}  // extern "C"
