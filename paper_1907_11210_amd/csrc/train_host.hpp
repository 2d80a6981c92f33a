// train_host.hpp -- what the C entry points of huge2_train.h share: checks, allocations.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <initializer_list>
#include <vector>

#include "huge2.h"

namespace huge2 {

// HUGE2_FAULT=alloc, launch: as in capi.cpp (tests of the error paths).
inline bool fault(const char* what) {
  const char* f = std::getenv("HUGE2_FAULT");
  return f && std::strcmp(f, what) == 0;
}

inline bool aligned(const void* p, size_t to = 16) { return ((uintptr_t)p & (to - 1)) == 0; }
inline bool bad(const void* p, size_t to = 16) { return !p || !aligned(p, to); }
struct Span {
  const void* p;
  size_t bytes;
};
inline bool overlap(const Span& a, const Span& b) {
  return a.p && b.p && (uintptr_t)a.p < (uintptr_t)b.p + b.bytes &&
         (uintptr_t)b.p < (uintptr_t)a.p + a.bytes;
}
// Whether what a call writes overlaps what it reads, or another thing that it writes.
inline bool overlaps(std::initializer_list<Span> writes, std::initializer_list<Span> reads) {
  for (const Span* w = writes.begin(); w != writes.end(); ++w) {
    for (const Span* o = writes.begin(); o != w; ++o)
      if (overlap(*w, *o)) return true;
    for (const Span& r : reads)
      if (overlap(*w, r)) return true;
  }
  return false;
}

// What a step over many tensors writes, in order of address.
class Written {
 public:
  // False where two of the spans overlap.
  bool set(std::vector<Span> spans) {
    spans.erase(std::remove_if(spans.begin(), spans.end(),
                               [](const Span& s) { return !s.p || !s.bytes; }),
                spans.end());
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.p < b.p; });
    for (const Span& s : spans) {
      const uintptr_t begin = (uintptr_t)s.p;
      if (!ends_.empty() && begin < ends_.back()) return false;
      begins_.push_back(begin);
      ends_.push_back(begin + s.bytes);
    }
    return true;
  }
  // Whether any of them overlaps.  (A search without branches: 160 gradients among 960 spans
  // take 1.6 us.)
  bool touches(const void* at, size_t bytes) const {
    const uintptr_t begin = (uintptr_t)at, end = begin + bytes;
    if (!at || !bytes || begins_.empty()) return false;
    const uintptr_t* base = begins_.data();  // comes to the last that begins before `end`
    for (size_t n = begins_.size(); n > 1;) {
      const size_t half = n / 2;
      base += base[half] < end ? half : 0;
      n -= half;
    }
    return *base < end && ends_[base - begins_.data()] > begin;
  }

 private:
  std::vector<uintptr_t> begins_, ends_;
};

inline bool is_dtype(int d) { return d == HUGE2_F32 || d == HUGE2_BF16; }
inline int elem_size(int dtype) { return dtype == HUGE2_BF16 ? 2 : 4; }
inline size_t round256(size_t v) { return (v + 255) / 256 * 256; }
inline int log2_ceil(long long v) {
  int l = 0;
  while ((1ll << l) < v) ++l;
  return l;
}

// The widest load of the type that divides a run of `len` elements: 16 bytes, 4
// or one element.
inline int vector_width(int dtype, long long len) {
  const int full = 16 / elem_size(dtype);
  if (len % full == 0) return full;
  return dtype == HUGE2_BF16 && len % 2 == 0 ? 2 : 1;
}

// A result that fills much of the 256 MB Infinity Cache is stored past it; a smaller
// one stays there for the layer that reads it.
inline bool streams(size_t bytes) { return bytes >= (size_t)64 << 20; }

inline huge2_status device_alloc(void** out, size_t bytes) {
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

inline huge2_status device_free(void* p) {
  if (p && hipFree(p) != hipSuccess) {
    (void)hipGetLastError();
    return HUGE2_ERR_HIP;
  }
  return HUGE2_OK;
}

inline huge2_status launched(hipError_t e) {
  if (e == hipSuccess) return HUGE2_OK;
  (void)hipGetLastError();
  return HUGE2_ERR_HIP;
}

}  // namespace huge2
