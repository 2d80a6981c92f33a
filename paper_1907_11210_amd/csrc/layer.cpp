// layer.cpp -- the C ABI of layer norm (declared in include/huge2_train.h): checks, plans,
// workspaces.
#include "huge2_train.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <new>

#include "kernels.hpp"
#include "train.hpp"
#include "train_host.hpp"

using namespace huge2;

struct huge2_layer_norm_plan {
  huge2_layer_norm_desc desc;
  bool rows;
  int vec;
  LayerArgs args[2];  // forward, gradient
  void* ws;
  char kernel_name[2][64];
};

namespace {

bool valid(const huge2_layer_norm_desc& d) {
  return d.n >= 1 && d.c >= 1 && d.h >= 1 && d.w >= 1 &&
         (d.layout == HUGE2_NCHW || d.layout == HUGE2_NHWC) && is_dtype(d.dtype) &&
         d.activation >= HUGE2_NORM_NONE && d.activation <= HUGE2_NORM_SILU &&
         std::isfinite(d.eps) && d.eps > 0.f;
}
size_t bytes_of(const huge2_layer_norm_desc& d) {
  return (size_t)d.n * d.c * d.h * d.w * elem_size(d.dtype);
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Rows: as many lanes as a row has vectors, up to a wave; more vectors a lane, up to what its
// registers hold; then more waves, up to a workgroup.
void choose_rows(LayerArgs* a, int vec, int esz, bool grad) {
  const long long vecs = ceil_div(a->c, vec);
  const auto most = [&] {
    const int channels = a->lanes_log2 > 6 ? kLayerWideChannels
                         : grad            ? kLayerGradChannels
                                           : kLayerChannels;
    return std::max(1, channels / vec);
  };
  a->lanes_log2 = std::min(6, log2_ceil(vecs));
  while (a->lanes_log2 < 10 && vecs > (long long)most() << a->lanes_log2) ++a->lanes_log2;
  const long long slots =
      a->lanes_log2 > 6 ? most() : 1ll << log2_ceil(ceil_div(vecs, 1ll << a->lanes_log2));
  a->slots = vecs > (long long)most() << a->lanes_log2 ? 0 : (int)slots;
  // (lanes of more than a wave are a whole workgroup)
  a->threads = !a->slots ? 1024 : a->lanes_log2 > 6 ? 1 << a->lanes_log2 : 256;
  const int teams = a->slots ? a->threads >> a->lanes_log2 : 1;
  const long long all = ceil_div(a->rows, teams);
  const long long most_groups = (grad ? 1024 : 2048) * 256 / a->threads;
  // The gradient's sums of a workgroup's rows, 8 bytes a channel written and read, are 4% of its
  // bytes from 17000 rows of bf16 on (8500 of fp32): 32768 rows of 1024 bf16 with 512 workgroups
  // 47.7 us, with 1024 52.5; 65536 of 128 with 512 and 1024 22.5 and 20.7.  Fewer rows have 256
  // workgroups, a unit's one, whatever their sums take: 1024 of 512, where they are 67%, with 256
  // and 1024 10.6 and 12.9.
  const long long want = grad ? std::max(256ll, a->rows * esz * 3 / 400) : all;
  a->groups = (int)std::min({all, want, most_groups});
  a->parts = a->groups;
  if (!a->slots) {
    const long long blocks = ceil_div(a->c, 256ll * vec);
    a->parts = (int)std::min(a->rows, std::max(1ll, 1024 / blocks));
  }
}

// Planes: tiles of 128 bytes of each plane, or less where the channels then fit the registers
// (or where there would be a few workgroups alone), and four vectors a thread.  64 images of
// 256x16x16 bf16, 8, 4 and 2 lanes on a tile: 9.8, 10.5 and 13.3 us, the gradient 14.7, 17.0 and
// 20.2; 64 of 128x64x64 35, 43 and 67, 55, 69 and 114.  With 8, 4, 2 and 1 vectors a thread 36.9,
// 36.0, 38.7 and 88, the gradient 70, 55, 56 and 93.
// False where there are too many tiles.
bool choose_planes(LayerArgs* a, int vec, int esz, bool grad) {
  const long long vecs = ceil_div(a->hw, vec);
  a->lanes_log2 = std::min(3, log2_ceil(vecs));
  // (a thread of 1024 holds 128 registers, of 512 twice as many)
  const auto most = [&](int threads) {
    return !grad           ? kLayerPlanes
           : threads <= 512 ? kLayerGradPlanes
                            : std::min(kLayerGradPlanes, kLayerWideChannels / vec);
  };
  const long long most_held = std::max(1024 * most(1024), 512 * most(512));  // of a tile
  while (a->lanes_log2 > 1 && a->c > most_held >> a->lanes_log2) --a->lanes_log2;
  const auto tiles = [&] { return ceil_div(vecs, 1ll << a->lanes_log2) * a->n; };
  while (a->lanes_log2 > 1 && tiles() < 64) --a->lanes_log2;
  const auto slots = [&] { return ceil_div(a->c, a->threads >> a->lanes_log2); };
  a->threads = 64;
  while (a->threads < 512 && slots() > 4) a->threads *= 2;
  if (slots() > 8) a->threads = 1024;  // (1000 channels: 8 vectors 17.3 us, 16 21.2)
  // (offsets of held channels are 32 bits of bytes)
  const bool held = slots() <= most(a->threads) && (long long)a->c * a->hw * esz < (1ll << 32);
  a->slots = held ? 1 << log2_ceil(slots()) : 0;
  if (tiles() >= (1ll << 31)) return false;
  a->tiles = (uint32_t)tiles();
  a->tiles_per_image = (int)(a->tiles / a->n);
  division_magic((uint32_t)a->tiles_per_image, &a->tile_mul, &a->tile_shift);
  a->groups = (int)std::min<long long>(a->tiles, (grad ? 1024 : 2048) * 256 / a->threads);
  a->parts = a->slots ? a->groups : (int)std::min<long long>(a->n, std::max(1, 2048 / a->c));
  return true;
}

huge2_status layer_create(huge2_layer_norm_plan** out, const huge2_layer_norm_desc* desc) {
  if (!out) return HUGE2_ERR_INVALID_ARG;
  *out = nullptr;
  if (!desc || !valid(*desc)) return HUGE2_ERR_INVALID_ARG;
  const huge2_layer_norm_desc& d = *desc;
  const long long hw = (long long)d.h * d.w;
  if (hw >= (1ll << 31) || hw * d.c >= (1ll << 31) || hw * d.c * d.n >= (1ll << 40))
    return HUGE2_ERR_UNSUPPORTED;
  const bool rows = d.layout == HUGE2_NHWC || hw == 1;
  // (a workgroup of 256 for a channel of planes, of 1024 for 16 channels' sums)
  if (!launchable(rows ? d.c / 16 + 1 : d.c, rows ? 1024 : 256)) return HUGE2_ERR_UNSUPPORTED;
  huge2_layer_norm_plan* p = new (std::nothrow) huge2_layer_norm_plan();
  if (!p) return HUGE2_ERR_ALLOC;
  p->desc = d;
  p->rows = rows;
  const int full = 16 / elem_size(d.dtype);
  p->vec = (p->rows ? d.c : hw) >= full ? full : 1;
  size_t part_b = 0;
  for (int g = 0; g < 2; ++g) {
    LayerArgs& a = p->args[g];
    a = {};
    a.n = d.n, a.c = d.c, a.hw = (int)hw, a.rows = hw * d.n;
    a.act = d.activation;
    a.eps = d.eps;
    a.stream = streams(bytes_of(d));
    if (p->rows) {
      choose_rows(&a, p->vec, elem_size(d.dtype), g != 0);
    } else if (!choose_planes(&a, p->vec, elem_size(d.dtype), g != 0)) {
      delete p;
      return HUGE2_ERR_UNSUPPORTED;
    }
    if (g) part_b = (size_t)a.parts * a.c * sizeof(float2);
    std::snprintf(p->kernel_name[g], sizeof(p->kernel_name[g]), "layer_%s%s_kernel v%d t%d r%d",
                  p->rows && !a.slots ? "" : g ? "grad_" : "",
                  !p->rows ? "planes" : a.slots ? "rows" : "long", p->vec, a.threads, a.slots);
  }
  const huge2_status st = device_alloc(&p->ws, part_b);
  if (st != HUGE2_OK) {
    delete p;
    return st;
  }
  *out = p;
  return HUGE2_OK;
}

huge2_status layer_run(const huge2_layer_norm_plan* p, const void* x, const float* gamma,
                       const float* beta, void* y, float* stats, hipStream_t stream) {
  if (!p || bad(x) || bad(y) || !aligned(gamma) || !aligned(beta) || !aligned(stats))
    return HUGE2_ERR_INVALID_ARG;
  const size_t bytes = bytes_of(p->desc), params = (size_t)p->desc.c * sizeof(float);
  const size_t pixels = (size_t)p->args[0].rows * sizeof(float2);
  if (overlaps({{y, bytes}, {stats, pixels}}, {{x, bytes}, {gamma, params}, {beta, params}}))
    return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  LayerArgs a = p->args[0];
  a.x = x, a.gamma = gamma, a.beta = beta, a.out = y, a.stats_out = stats;
  return launched((p->rows ? launch_layer_rows : launch_layer_planes)(a, p->desc.dtype, p->vec,
                                                                      false, stream));
}

huge2_status layer_grad_run(const huge2_layer_norm_plan* p, const void* x, const void* dy,
                            const float* stats, const float* gamma, const float* beta, void* dx,
                            float* dgamma, float* dbeta, hipStream_t stream) {
  if (!p || bad(x) || bad(dy) || bad(dx) || bad(stats) || !aligned(gamma) || !aligned(beta) ||
      !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return HUGE2_ERR_INVALID_ARG;
  const size_t bytes = bytes_of(p->desc), params = (size_t)p->desc.c * sizeof(float);
  const size_t pixels = (size_t)p->args[1].rows * sizeof(float2);
  if (overlaps({{dx, bytes}, {dgamma, params}, {dbeta, params}},
               {{x, bytes}, {dy, bytes}, {stats, pixels}, {gamma, params}, {beta, params}}))
    return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  LayerArgs a = p->args[1];
  a.x = x, a.dy = dy, a.stats = stats, a.gamma = gamma, a.beta = beta, a.out = dx;
  a.dgamma = dgamma, a.dbeta = dbeta;
  a.part = dgamma || dbeta ? (float2*)p->ws : nullptr;
  return launched((p->rows ? launch_layer_rows : launch_layer_planes)(a, p->desc.dtype, p->vec,
                                                                      true, stream));
}

}  // namespace

extern "C" {

huge2_status huge2_layer_norm_plan_create(huge2_layer_norm_plan** out,
                                          const huge2_layer_norm_desc* desc) {
  try {
    return layer_create(out, desc);
  } catch (...) {
    return HUGE2_ERR_ALLOC;
  }
}

huge2_status huge2_layer_norm_execute(const huge2_layer_norm_plan* plan, const void* x,
                                      const float* gamma, const float* beta, void* y, float* stats,
                                      void* hip_stream) {
  return layer_run(plan, x, gamma, beta, y, stats, (hipStream_t)hip_stream);
}

huge2_status huge2_layer_norm_grad_execute(const huge2_layer_norm_plan* plan, const void* x,
                                           const void* dy, const float* stats, const float* gamma,
                                           const float* beta, void* dx, float* dgamma,
                                           float* dbeta, void* hip_stream) {
  return layer_grad_run(plan, x, dy, stats, gamma, beta, dx, dgamma, dbeta,
                        (hipStream_t)hip_stream);
}

const char* huge2_layer_norm_plan_kernel(const huge2_layer_norm_plan* plan, int32_t grad) {
  return plan ? plan->kernel_name[grad != 0] : "";
}

huge2_status huge2_layer_norm_plan_destroy(huge2_layer_norm_plan* plan) {
  if (!plan) return HUGE2_OK;
  const huge2_status st = device_free(plan->ws);
  delete plan;
  return st;
}

}  // extern "C"
