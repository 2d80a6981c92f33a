// muon.cpp -- the C ABI of orthogonalised matrices and the Muon step (declared in
// include/huge2_train.h): checks, plans, workspaces.
#include "huge2_train.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <vector>

#include "newton.hpp"
#include "train.hpp"
#include "train_host.hpp"

using namespace huge2;

namespace {

// A list of works in the plan's table.
struct Works {
  size_t at = 0;  // bytes
  unsigned count = 0;
};
// Matrices whose products share launches.
struct Group {
  int first, count;
  int size[4];  // of each product's tiles
  Works norm, pack, product[4], join[4];
};

// The polynomial and the powers of two that a step's operands are stored times: their
// magnitudes stay below 2^15 (fp16 ends at 65504).
struct Step {
  float a, b, c;
  int x, gram, poly;  // exponents of X, A and B
};

int exponent(double bound) { return 14 - (int)std::ceil(std::log2(std::max(bound, 0x1p-30))); }

}  // namespace

// What both plans have.
struct NsEngine {
  NsEngine() = default;
  NsEngine(const NsEngine&) = delete;
  ~NsEngine() { (void)release(); }
  huge2_status release() {
    const huge2_status a = device_free(ws), b = device_free(table);
    ws = table = nullptr;
    return a != HUGE2_OK ? a : b;
  }

  int parts = 2;
  double eps = 0;
  std::vector<Step> steps;
  std::vector<NsMatrix> mats;
  std::vector<Group> groups;
  void* table = nullptr;  // NsMatrix [], then the works
  void* ws = nullptr;
};

struct huge2_orthogonalize_plan {
  huge2_orthogonalize_desc desc;
  NsEngine ns;
};

struct huge2_muon_plan {
  int count;
  NsEngine ns;
  std::vector<size_t> grad_bytes;  // [count]
  Written written;                 // by a step
};

namespace {

// False where the singular values could leave what 16 bits hold.
bool steps_of(const huge2_newton_schulz& ns, NsEngine* e) {
  double s = 1;  // no singular value is larger: the norm is 1 at most
  for (int k = 0; k < ns.steps; ++k) {
    const double a = ns.coefficients[3 * k], b = ns.coefficients[3 * k + 1],
                 c = ns.coefficients[3 * k + 2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    const double q = s * s;
    Step step = {(float)a, (float)b, (float)c, exponent(s), exponent(q),
                 exponent(std::fabs(c) * q * q + (std::fabs(b) + 2 * std::fabs(c) * q) * q)};
    e->steps.push_back(step);
    // the largest |a x + b x^3 + c x^5| up to s: there, or where a + 3 b y + 5 c y^2 = 0, y = x^2
    const auto value = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
    double most = value(s);
    const double disc = 9 * b * b - 20 * a * c;
    for (const double y : {c != 0 && disc >= 0 ? (-3 * b + std::sqrt(disc)) / (10 * c) : -1.0,
                           c != 0 && disc >= 0 ? (-3 * b - std::sqrt(disc)) / (10 * c) : -1.0,
                           c == 0 && b != 0 ? -a / (3 * b) : -1.0})
      if (y > 0 && y < q) most = std::max(most, value(std::sqrt(y)));
    s = most * 1.002;  // (with what the roundings add)
    if (!(s <= 0x1p10) || step.poly < -10) return false;
  }
  return true;
}

bool valid(const huge2_newton_schulz* ns) {
  return ns && ns->steps >= 1 && ns->steps <= 32 && ns->coefficients && std::isfinite(ns->eps) &&
         ns->eps >= 0x1p-126 &&
         (ns->products == HUGE2_PRODUCTS_F32 || ns->products == HUGE2_PRODUCTS_F16);
}

int pad(int v) { return (v + kNsPad - 1) / kNsPad * kNsPad; }
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Sums of squares by blocks of tiles of any size.
size_t squares_room(const NsMatrix& t) {
  size_t most = 0;
  for (const NsTile& tile : kNsTiles)
    most = std::max<size_t>(
        most, ceil_div(t.mp, tile.rows) * ceil_div(t.np, tile.cols) * tile.blocks());
  return most;
}
size_t workspace(const NsMatrix& t, int parts) {
  const size_t whole = (size_t)t.mp * t.np * sizeof(half_bits);
  const size_t square = (size_t)t.mp * t.mp * sizeof(half_bits);
  return 3 * round256(2 * whole) + round256(2 * square) +
         round256(parts * square) + round256(squares_room(t) * sizeof(float)) +
         round256(t.norm_count * sizeof(double)) + 256;
}
void place(NsMatrix* t, int parts, char* at) {
  const size_t whole = (size_t)t->mp * t->np * sizeof(half_bits);
  const size_t square = (size_t)t->mp * t->mp * sizeof(half_bits);
  const auto take = [&](size_t bytes) {
    char* const p = at;
    at += round256(bytes);
    return p;
  };
  t->x = (half_bits*)take(2 * whole);
  t->t0 = (half_bits*)take(2 * whole);
  t->t1 = (half_bits*)take(2 * whole);
  t->a = (half_bits*)take(2 * square);
  t->b = (half_bits*)take(parts * square);
  t->squares = (float*)take(squares_room(*t) * sizeof(float));
  t->norm = (double*)take(t->norm_count * sizeof(double));
  t->mu = (float*)take(sizeof(float));
}

void shape(NsMatrix* t, long long rows, long long cols) {
  t->tall = rows > cols;
  t->m = (int)std::min(rows, cols);
  t->n = (int)std::max(rows, cols);
  t->mp = pad(t->m), t->np = pad(t->n);
  t->count = rows * cols;
  t->norm_chunk = (int)(ceil_div(std::max(4096ll, ceil_div(t->count, 1024)), 256) * 256);
  t->norm_count = (int)ceil_div(t->count, t->norm_chunk);
}

// Tiles of a product, of the given size; f(row, column) of each if wanted.
template <typename F>
void each_tile(const NsMatrix& t, int kind, int size, F&& f) {
  const NsTile& tile = kNsTiles[size];
  const bool symmetric = kind == kNsGram || kind == kNsSquare, turned = kind == kNsLast && t.tall;
  const long long rows = ceil_div(turned ? t.np : t.mp, tile.rows);
  const long long cols = ceil_div(symmetric || turned ? t.mp : t.np, tile.cols);
  for (long long r = 0; r < rows; ++r)
    for (long long c = symmetric ? r * tile.rows / tile.cols : 0; c < cols; ++c)
      f((int)r, (int)c);
}

constexpr int kUnits = 256;  // compute units

// The size of a product's tiles.  Large ones need the least of LDS and the caches, and enough
// columns to be worth their long prologue and epilogue; small ones start and end sooner.  Whole
// passes in us with the small, middle and large tiles alone:
//   1 of 4096x8192, two parts                     10980  6430  6130
//     one part                                     4960  2910  2730
//   6 of 4096x4096 and the like, two parts        24820 14900 13670
//     one part                                    11440  7530  6430
//   5 of 100x16384 to 128x48, two parts             869   816   899
//     one part                                      524   505   565
//   48 of 33x700 to 644x89, two parts               371   412   501
//     one part                                      260   254   340
//   6 of 1000x333, two parts                        200   220   304
// So large ones where there are three for four units, with 2048 columns each, and middle ones
// from 512 columns a unit on; of the last product, whose results leave by single elements and
// hide behind other tiles' products, from 1024 on.  (It takes 6150, 2730, 13670, 6460, 793, 474,
// 378, 260 and 197.)
int tile_size(const NsEngine& e, const Group& g, int kind) {
  if (const char* f = std::getenv("HUGE2_NS_TILE")) return (unsigned)std::atoi(f) % kNsSizes;
  long long tiles[kNsSizes] = {}, columns[kNsSizes] = {};
  for (int i = 0; i < g.count; ++i)
    for (int size = 0; size < kNsSizes; ++size)
      each_tile(e.mats[g.first + i], kind, size, [&](int, int) {
        ++tiles[size];
        const NsMatrix& t = e.mats[g.first + i];
        columns[size] += (kind == kNsGram ? t.np : t.mp) * e.parts;
      });
  if (tiles[2] >= kUnits * 3 / 4 && columns[2] >= tiles[2] * 2048) return 2;
  return columns[1] >= kUnits * (kind == kNsLast ? 1024ll : 512ll) ? 1 : 0;
}

// A product's tiles.  Where they do not fill the compute units, or leave some over that would
// run alone, those are cut along their sum: `slots` counts partial tiles.  (4096x8192: 272 large
// tiles of the first product are 256 and 16 in 16 pieces each.  Uncut, 16 units have
// two tiles and the others wait for them.)
void product_works(NsEngine& e, Group& g, int kind, std::vector<NsWork>* works,
                   std::vector<NsWork>* joins, int* slots) {
  const int size = g.size[kind] = tile_size(e, g, kind);
  std::vector<NsWork> all;
  double cost = 0;  // stages of all
  for (int i = 0; i < g.count; ++i) {
    NsMatrix& t = e.mats[g.first + i];
    if (kind == kNsApply) t.squares_count = 0;
    const int stages = (kind == kNsGram ? t.np : t.mp) / (kNsTiles[size].stage / e.parts);
    each_tile(t, kind, size, [&](int r, int c) {
      all.push_back({i, r, c, 0, stages, -1, 0});
      cost += stages;
      if (kind == kNsApply) t.squares_count += kNsTiles[size].blocks();
    });
  }
  std::stable_sort(all.begin(), all.end(),
                   [](const NsWork& a, const NsWork& b) { return a.k1 > b.k1; });
  // whole tiles, as many as all units take alike, and the rest in pieces of a unit's share
  const size_t whole = all.size() / kUnits * kUnits;
  double left = 0;
  for (size_t k = whole; k < all.size(); ++k) left += all[k].k1;
  *slots = 0;
  for (size_t k = 0; k < all.size(); ++k) {
    NsWork w = all[k];
    const int stages = w.k1;
    // (pieces of 32 stages of small tiles: shorter ones lose more to the join than they gain,
    // with half as many 207 us for 203 of 6 of 1000x333, 830 for 816 of 100x16384 to 128x48)
    const double piece = std::max(size == 0 ? 32.0 : 16.0, (k < whole ? cost : left) / kUnits);
    // (rounded down behind whole tiles, which hide an uneven end)
    const int cuts = std::max(1, std::min(stages / 8, (int)(stages / piece + (whole ? 0.0 : 0.6))));
    if (cuts > 1) {
      NsWork join = w;
      join.slot = *slots, join.slots = cuts;
      joins->push_back(join);
      for (int c = 0; c < cuts; ++c) {
        w.k0 = (int)((long long)stages * c / cuts);
        w.k1 = (int)((long long)stages * (c + 1) / cuts);
        w.slot = (*slots)++;
        works->push_back(w);
      }
    } else {
      works->push_back(w);
    }
  }
}

constexpr size_t kGroupBytes = (size_t)4 << 30;  // matrices beyond start another group

huge2_status engine_create(NsEngine* e, const huge2_newton_schulz& ns, hipStream_t stream) {
  e->parts = ns.products == HUGE2_PRODUCTS_F32 ? 2 : 1;
  e->eps = ns.eps;
  if (!steps_of(ns, e)) return HUGE2_ERR_INVALID_ARG;
  size_t ws_b = 0, bytes = 0;
  for (int i = 0; i < (int)e->mats.size(); ++i) {
    const size_t own = workspace(e->mats[i], e->parts);
    if (i == 0 || e->groups.back().count == kNsMatrices || bytes + own > kGroupBytes) {
      e->groups.push_back({i, 0, {}, {}, {}, {}, {}});
      bytes = 0;
    }
    ++e->groups.back().count;
    bytes += own;
    ws_b = std::max(ws_b, bytes);
  }
  std::vector<char> image(round256(e->mats.size() * sizeof(NsMatrix)));
  const auto append = [&](Works* list, const auto& works) {
    list->at = image.size();
    list->count = (unsigned)works.size();
    const size_t bytes = works.size() * sizeof(works[0]);
    image.resize(list->at + round256(bytes));
    if (bytes) std::memcpy(image.data() + list->at, works.data(), bytes);
  };
  size_t parts_b = 0;
  for (Group& g : e->groups) {
    std::vector<uint2> norm, pack;
    for (int i = 0; i < g.count; ++i) {
      const NsMatrix& t = e->mats[g.first + i];
      for (int k = 0; k < t.norm_count; ++k) norm.push_back(make_uint2(i, k));
      const unsigned blocks = (unsigned)(t.mp / kNsBlock) * (unsigned)(t.np / kNsBlock);
      for (unsigned k = 0; k < blocks; ++k) pack.push_back(make_uint2(i, k));
    }
    append(&g.norm, norm);
    append(&g.pack, pack);
    for (int kind = 0; kind < 4; ++kind) {
      std::vector<NsWork> works, joins;
      int slots;
      product_works(*e, g, kind, &works, &joins, &slots);
      parts_b = std::max(parts_b, slots * kNsTiles[g.size[kind]].slot() * sizeof(float));
      append(&g.product[kind], works);
      append(&g.join[kind], joins);
    }
  }
  huge2_status st = device_alloc(&e->ws, parts_b + ws_b);
  if (st == HUGE2_OK && !e->mats.empty()) st = device_alloc(&e->table, image.size());
  if (st != HUGE2_OK) return st;
  for (const Group& g : e->groups) {
    char* at = (char*)e->ws + parts_b;
    for (int i = 0; i < g.count; ++i) {
      NsMatrix& t = e->mats[g.first + i];
      place(&t, e->parts, at);
      at += workspace(t, e->parts);
    }
  }
  if (e->mats.empty()) return HUGE2_OK;
  std::memcpy(image.data(), e->mats.data(), e->mats.size() * sizeof(NsMatrix));
  if (hipMemcpyAsync(e->table, image.data(), image.size(), hipMemcpyHostToDevice, stream) !=
          hipSuccess ||
      hipStreamSynchronize(stream) != hipSuccess) {
    (void)hipGetLastError();
    return HUGE2_ERR_HIP;
  }
  return HUGE2_OK;
}

// One pass: src are the group's inputs, call what all launches share.
huge2_status engine_run(const NsEngine& e, const Group& g, NsInput in, NsArgs call,
                        hipStream_t stream) {
  const char* const table = (const char*)e.table;
  in.mats = call.mats = (const NsMatrix*)table + g.first;
  in.eps = e.eps;
  in.out_scale = (float)std::ldexp(1.0, e.steps[0].x);
  in.keep_lo = e.steps.size() == 1;
  for (int i = 0; i < g.count; ++i)
    if (!in.src[i]) call.skip[i >> 6] |= 1ull << (i & 63);
  in.works = (const uint2*)(table + g.norm.at);
  huge2_status st = launched(launch_ns_norm(in, g.norm.count, stream));
  in.works = (const uint2*)(table + g.pack.at);
  if (st == HUGE2_OK) st = launched(launch_ns_pack(in, g.pack.count, e.parts, stream));
  call.part = (float*)e.ws;
  const auto power = [](int k) { return (float)std::ldexp(1.0, k); };
  for (size_t k = 0; k < e.steps.size(); ++k) {
    const Step& s = e.steps[k];
    call.step = (int)k;
    call.from = (int)k & 1;
    const bool last = k + 1 == e.steps.size();
    call.a = s.a, call.b = s.b, call.c = s.c;
    call.keep_lo = k + 2 == e.steps.size();
    for (const int kind : {(int)kNsGram, (int)kNsSquare, last ? (int)kNsLast : (int)kNsApply}) {
      const bool apply = kind == kNsApply || kind == kNsLast;
      call.kind = kind;
      call.in_scale = power(apply ? -s.poly - s.x : kind == kNsGram ? -2 * s.x : -2 * s.gram);
      call.own_scale = power(kind == kNsSquare ? -s.gram : -s.x);
      call.out_scale = power(kind == kNsGram     ? s.gram
                             : kind == kNsSquare ? s.poly
                             : last              ? 0
                                                 : e.steps[k + 1].x);
      for (const bool join : {false, true}) {
        const Works& works = join ? g.join[kind] : g.product[kind];
        call.works = (const NsWork*)(table + works.at);
        if (st == HUGE2_OK && works.count)
          st = launched(launch_ns_product(call, works.count, g.size[kind], join, e.parts, stream));
      }
    }
  }
  return st;
}

// ---- orthogonalised matrices ------------------------------------------------------------

bool valid(const huge2_orthogonalize_desc& d) {
  return d.batch >= 1 && d.rows >= 1 && d.cols >= 1 && is_dtype(d.dtype);
}
constexpr long long kMostElements = 1ll << 31;  // of a matrix, below
constexpr int kMostSide = 1 << 28;
constexpr int kMostMatrices = 1 << 20;

size_t bytes_of(const huge2_orthogonalize_desc& d) {
  return (size_t)d.batch * d.rows * d.cols * elem_size(d.dtype);
}

huge2_status orthogonalize_create(huge2_orthogonalize_plan** out,
                                  const huge2_orthogonalize_desc* desc,
                                  const huge2_newton_schulz* ns, hipStream_t stream) {
  if (!out) return HUGE2_ERR_INVALID_ARG;
  *out = nullptr;
  if (!desc || !valid(*desc) || !valid(ns)) return HUGE2_ERR_INVALID_ARG;
  const long long count = (long long)desc->rows * desc->cols;
  if (count >= kMostElements || std::max(desc->rows, desc->cols) > kMostSide ||
      desc->batch > kMostMatrices ||
      count * desc->batch >= (1ll << 40))
    return HUGE2_ERR_UNSUPPORTED;
  std::unique_ptr<huge2_orthogonalize_plan> p(new huge2_orthogonalize_plan());
  p->desc = *desc;
  NsMatrix t = {};
  shape(&t, desc->rows, desc->cols);
  t.bf16 = t.grad_bf16 = desc->dtype == HUGE2_BF16;
  p->ns.mats.assign(desc->batch, t);
  for (int i = 0; i < desc->batch; ++i) p->ns.mats[i].out_at = i * count;
  const huge2_status st = engine_create(&p->ns, *ns, stream);
  if (st == HUGE2_OK) *out = p.release();
  return st;
}

huge2_status orthogonalize_run(const huge2_orthogonalize_plan* p, const void* x, void* y,
                               hipStream_t stream) {
  if (!p || bad(x) || bad(y)) return HUGE2_ERR_INVALID_ARG;
  const size_t bytes = bytes_of(p->desc), one = bytes / p->desc.batch;
  if (overlaps({{y, bytes}}, {{x, bytes}})) return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  for (const Group& g : p->ns.groups) {
    NsInput in;
    std::memset(&in, 0, sizeof(in));
    NsArgs call;
    std::memset(&call, 0, sizeof(call));
    for (int i = 0; i < g.count; ++i) in.src[i] = (const char*)x + one * (g.first + i);
    call.out = y;
    const huge2_status st = engine_run(p->ns, g, in, call, stream);
    if (st != HUGE2_OK) return st;
  }
  return HUGE2_OK;
}

// ---- the Muon step -----------------------------------------------------------------------

bool valid(const huge2_muon_tensor& t) {
  return t.rows >= 1 && t.cols >= 1 && is_dtype(t.dtype) && is_dtype(t.grad_dtype) &&
         std::isfinite(t.weight_decay) && t.weight_decay >= 0.f && std::isfinite(t.scale) &&
         !bad(t.param) && !bad(t.m) && aligned(t.copy);
}

huge2_status muon_create(huge2_muon_plan** out, const huge2_muon_tensor* tensors, int count,
                         const huge2_newton_schulz* ns, hipStream_t stream) {
  if (!out) return HUGE2_ERR_INVALID_ARG;
  *out = nullptr;
  if (count < 0 || (count && !tensors) || !valid(ns)) return HUGE2_ERR_INVALID_ARG;
  long long total = 0;
  std::vector<Span> spans;
  for (int i = 0; i < count; ++i) {
    const huge2_muon_tensor& t = tensors[i];
    if (!valid(t)) return HUGE2_ERR_INVALID_ARG;
    const long long n = (long long)t.rows * t.cols;
    if (n >= kMostElements || std::max(t.rows, t.cols) > kMostSide || (total += n) >= (1ll << 40))
      return HUGE2_ERR_UNSUPPORTED;
    for (const Span& s : {Span{t.param, (size_t)n * elem_size(t.dtype)},
                          Span{t.m, (size_t)n * sizeof(float)}, Span{t.copy, (size_t)n * 2}})
      spans.push_back(s);
  }
  if (count > kMostMatrices) return HUGE2_ERR_UNSUPPORTED;
  Written written;
  if (!written.set(std::move(spans))) return HUGE2_ERR_INVALID_ARG;
  std::unique_ptr<huge2_muon_plan> p(new huge2_muon_plan());
  p->count = count;
  p->written = std::move(written);
  for (int i = 0; i < count; ++i) {
    const huge2_muon_tensor& t = tensors[i];
    NsMatrix m = {};
    shape(&m, t.rows, t.cols);
    m.param = t.param, m.copy = t.copy, m.momentum = t.m;
    m.bf16 = t.dtype == HUGE2_BF16, m.grad_bf16 = t.grad_dtype == HUGE2_BF16;
    m.decay = t.weight_decay, m.scale = t.scale;
    p->ns.mats.push_back(m);
    p->grad_bytes.push_back((size_t)m.count * elem_size(t.grad_dtype));
  }
  const huge2_status st = engine_create(&p->ns, *ns, stream);
  if (st == HUGE2_OK) *out = p.release();
  return st;
}

huge2_status muon_run(const huge2_muon_plan* p, const void* const* grads,
                      const huge2_muon_options* o, const float* grad_scale, hipStream_t stream) {
  if (!p || !o || (p->count && !grads) || !aligned(grad_scale, 4)) return HUGE2_ERR_INVALID_ARG;
  if (!std::isfinite((float)o->lr) || o->lr < 0 || !(o->momentum >= 0) || o->momentum >= 1 ||
      (float)o->momentum >= 1.f)
    return HUGE2_ERR_INVALID_ARG;
  for (int i = 0; i < p->count; ++i)
    if (!aligned(grads[i]) || p->written.touches(grads[i], p->grad_bytes[i]))
      return HUGE2_ERR_INVALID_ARG;
  if (p->written.touches(grad_scale, sizeof(float))) return HUGE2_ERR_INVALID_ARG;
  if (fault("launch")) return HUGE2_ERR_HIP;
  for (const Group& g : p->ns.groups) {
    NsInput in;
    std::memset(&in, 0, sizeof(in));
    NsArgs call;
    std::memset(&call, 0, sizeof(call));
    std::memcpy(in.src, grads + g.first, g.count * sizeof(void*));
    in.muon = 1;
    in.nesterov = o->nesterov != 0;
    in.momentum = (float)o->momentum, in.rest = (float)(1 - o->momentum);
    in.grad_scale = grad_scale;
    call.lr = (float)o->lr;
    const huge2_status st = engine_run(p->ns, g, in, call, stream);
    if (st != HUGE2_OK) return st;
  }
  return HUGE2_OK;
}

}  // namespace

extern "C" {

huge2_status huge2_orthogonalize_plan_create(huge2_orthogonalize_plan** out,
                                             const huge2_orthogonalize_desc* desc,
                                             const huge2_newton_schulz* ns, void* hip_stream) {
  try {
    return orthogonalize_create(out, desc, ns, (hipStream_t)hip_stream);
  } catch (...) {
    if (out) *out = nullptr;
    return HUGE2_ERR_ALLOC;
  }
}

huge2_status huge2_orthogonalize_execute(const huge2_orthogonalize_plan* plan, const void* x,
                                         void* y, void* hip_stream) {
  return orthogonalize_run(plan, x, y, (hipStream_t)hip_stream);
}

huge2_status huge2_orthogonalize_plan_destroy(huge2_orthogonalize_plan* plan) {
  if (!plan) return HUGE2_OK;
  const huge2_status st = plan->ns.release();
  delete plan;
  return st;
}

huge2_status huge2_muon_plan_create(huge2_muon_plan** out, const huge2_muon_tensor* tensors,
                                    int32_t count, const huge2_newton_schulz* ns,
                                    void* hip_stream) {
  try {
    return muon_create(out, tensors, count, ns, (hipStream_t)hip_stream);
  } catch (...) {
    if (out) *out = nullptr;
    return HUGE2_ERR_ALLOC;
  }
}

huge2_status huge2_muon_step(const huge2_muon_plan* plan, const void* const* grads,
                             const huge2_muon_options* options, const float* grad_scale,
                             void* hip_stream) {
  return muon_run(plan, grads, options, grad_scale, (hipStream_t)hip_stream);
}

huge2_status huge2_muon_plan_destroy(huge2_muon_plan* plan) {
  if (!plan) return HUGE2_OK;
  const huge2_status st = plan->ns.release();
  delete plan;
  return st;
}

}  // extern "C"
