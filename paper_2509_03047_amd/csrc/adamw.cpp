// The optimizer step's host side: validation of an optimizer against a plan's
// table, its device tables, and the C entry points' checks.
#include "adamw.h"

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "checks.h"
#include "fr_internal.h"

using namespace fr;

namespace {

struct Range {
  uint64_t first, last;
  bool operator<(const Range& o) const { return first < o.first; }
};

// Whether two sorted lists of disjoint ranges meet.
bool meet(const std::vector<Range>& a, const std::vector<Range>& b) {
  if (a.empty() || b.empty() || a.back().last <= b.front().first || b.back().last <= a.front().first) return false;
  for (size_t i = 0, j = 0; i < a.size() && j < b.size();) {
    if (a[i].last <= b[j].first) i++;
    else if (b[j].last <= a[i].first) j++;
    else return true;
  }
  return false;
}

// A walk on the host: one run of slots per tensor, as launch_expand_slots
// takes them.
struct Runs {
  uint32_t tile;  // elements
  std::vector<uint64_t> first{0}, base;
  explicit Runs(uint32_t t) : tile(t) {}
  uint64_t n() const { return first.back(); }
  uint64_t stride() const { return (n() + 7) / 8; }
  void add(uint32_t tensor, uint64_t numel) {
    if (!numel) return;
    base.push_back(uint64_t(tensor) << 32);
    first.push_back(first.back() + (numel + tile - 1) / tile);
  }
};

// What an optimizer is, before the device knows of it.
struct AdamwLayout {
  std::vector<AdamwRec> recs;
  std::vector<uint8_t> eight, counted;
  std::vector<uint32_t> chunk0;      // kKinds per tensor: its arrays' first chunks
  std::vector<uint32_t> n_chunks;    // and how many each has
  std::vector<Range> moments;        // sorted
  fr_adamw_info info{};
};

uint64_t blocks_of(uint64_t numel) { return (numel + FR_ADAMW_BLOCK - 1) / FR_ADAMW_BLOCK; }

int validate(const fr_tensor_desc* table, uint32_t n_entries, const Layout& L, uint64_t arena_bytes,
             const fr_adamw_tensor* t, uint32_t n, uint32_t n_groups, uint64_t grad_bytes, AdamwLayout* out) {
  if (n && !t) return FR_E_INVAL;
  std::vector<uint8_t> named(n_entries, 0);
  std::vector<Range> written;
  out->recs.resize(n);
  out->eight.resize(n);
  out->counted.resize(n);
  out->chunk0.assign(size_t(n) * kKinds, 0);
  out->n_chunks.assign(size_t(n) * kKinds, 0);
  fr_adamw_info& info = out->info;
  info.n_tensors = n;
  info.n_groups = n_groups;
  info.grad_arena_bytes = grad_bytes;
  info.arena_bytes = arena_bytes;
  info.device = -1;
  bool twice = false, strange = false;
  for (uint32_t k = 0; k < n; k++) {
    const fr_adamw_tensor& d = t[k];
    if (d.reserved || (d.flags & ~uint32_t(FR_GRAD_NOT_COUNTED)) || d.group >= n_groups) return FR_E_INVAL;
    if (d.grad_dtype != FR_F32 && d.grad_dtype != FR_BF16) return FR_E_INVAL;
    if (d.grad_offset % 16) return FR_E_ALIGN;
    if ((d.m_scale < 0) != (d.v_scale < 0)) return FR_E_INVAL;
    if (d.master < 0 || uint32_t(d.master) >= n_entries) return FR_E_INVAL;
    const uint64_t numel = table[d.master].numel;
    const bool eight = d.m_scale >= 0;
    const uint64_t mom = eight ? (numel + 3) / 4 : numel;
    const struct {
      int32_t entry;
      uint64_t numel;
      uint32_t dtype;
      bool may_miss;
    } want[kKinds] = {{d.param, numel, FR_BF16, true},          {d.master, numel, FR_F32, false},
                      {d.m, mom, FR_F32, false},                {d.v, mom, FR_F32, false},
                      {d.m_scale, blocks_of(numel), FR_F32, !eight}, {d.v_scale, blocks_of(numel), FR_F32, !eight}};
    AdamwRec& r = out->recs[k];
    std::memset(&r, 0, sizeof r);
    for (uint32_t j = 0; j < kKinds; j++) {
      r.at[j] = kNone;
      if (want[j].entry < 0) {
        if (want[j].entry != -1 || !want[j].may_miss) return FR_E_INVAL;
        continue;
      }
      const uint32_t e = uint32_t(want[j].entry);
      if (e >= n_entries || table[e].dtype != want[j].dtype || table[e].numel != want[j].numel) return FR_E_INVAL;
      // (a restore derives the parameter anew: from the master that a step writes
      // it from, or not at all; of none there is nothing that could differ)
      if (j == kParam) strange |= numel && table[e].derive_from != -1 && table[e].derive_from != d.master;
      twice |= named[e] != 0;
      named[e] = 1;
      r.at[j] = table[e].src_offset;
      const uint64_t bytes = table[e].numel * (want[j].dtype == FR_F32 ? 4 : 2);
      if (bytes) {
        written.push_back({r.at[j], r.at[j] + bytes});
        if (j >= kMom1) out->moments.push_back(written.back());
      }
      out->chunk0[size_t(k) * kKinds + j] = uint32_t(L.chunk_base[e]);
      out->n_chunks[size_t(k) * kKinds + j] = uint32_t(L.chunk_base[e + 1] - L.chunk_base[e]);
      if (L.C >= FR_ADAMW_MIN_SUM_CHUNK) info.sums_chunks += L.chunk_base[e + 1] - L.chunk_base[e];
    }
    const uint64_t gb = numel * (d.grad_dtype == FR_F32 ? 4 : 2);
    if (d.grad_offset > grad_bytes || gb > grad_bytes - d.grad_offset) return FR_E_RANGE;
    r.numel = numel;
    r.counter = info.n_counters;
    r.grad = d.grad_offset;
    r.grad_f32 = d.grad_dtype == FR_F32;
    r.group = d.group;
    out->eight[k] = eight;
    out->counted[k] = !(d.flags & FR_GRAD_NOT_COUNTED);
    info.n_elements += numel;
    if (eight) info.n_elements_8bit += numel;
    info.n_counters += (numel + FR_ADAMW_SPAN - 1) / FR_ADAMW_SPAN * FR_ADAMW_SPAN;
  }
  if (twice) return FR_E_OVERLAP;
  std::sort(written.begin(), written.end());
  for (size_t i = 1; i < written.size(); i++)
    if (written[i].first < written[i - 1].last) return FR_E_OVERLAP;
  if (strange) return FR_E_INVAL;
  std::sort(out->moments.begin(), out->moments.end());
  // a launch has fewer than 2^32 threads: a wave for each tile of 256 elements,
  // or a workgroup for each chunk of scales, of which a tensor has two
  if (info.n_counters / 256 + 8 * uint64_t(n) >= (uint64_t(1) << 26)) return FR_E_RANGE;
  return FR_OK;
}

}  // namespace

struct fr_adamw {
  int device = -1;
  AdamwLayout layout;
  uint64_t C = 0, plan_chunks = 0;
  void* mem = nullptr;  // everything below
  const AdamwRec* d_recs = nullptr;
  // By form (0: 32 bits, 1: 8): the walks of a step, of one that sums and of
  // a conversion; what the second leaves and how that is folded.
  struct Form {
    AdamwWalk step, sum, convert;
    fr_chunk_sum* parts = nullptr;
    const AdamwFold* folds = nullptr;
    const AdamwScales* scales = nullptr;
    uint32_t n_folds = 0, n_scales = 0;
  } form[2];
  const fr_grad_stats* no_stats = nullptr;  // scale 1: a step without statistics reads these
  AdamwWalk norm;
  double* norm_parts = nullptr;
  uint32_t* arrived = nullptr;
};

namespace {

// One allocation, filled from host arrays (NULL: zeros).
struct Carver {
  struct Piece {
    const void* src;
    uint64_t bytes, at;
  };
  std::vector<Piece> pieces;
  uint64_t total = 0;
  size_t add(const void* src, uint64_t bytes) {
    pieces.push_back({src, bytes, total});
    total += (bytes + 255) & ~uint64_t(255);
    return pieces.size() - 1;
  }
};

int build(fr_adamw* o) {
  const AdamwLayout& Y = o->layout;
  const uint32_t n = uint32_t(Y.recs.size());
  // the walks: norm, then by form step, sum, convert
  enum { kNorm, kStep, kSum = kStep + 2, kConvert = kSum + 2, kWalks = kConvert + 2 };
  Runs runs[kWalks] = {Runs(kNormBytes / 4),
                       Runs(kStepShape[0].tile()), Runs(kStepShape[1].tile()),
                       Runs(kSumShape[0].tile()), Runs(kSumShape[1].tile()),
                       Runs(kConvertShape[0].tile()), Runs(kConvertShape[1].tile())};
  std::vector<AdamwFold> folds[2];
  std::vector<AdamwScales> scales[2];
  const bool sums = o->C >= FR_ADAMW_MIN_SUM_CHUNK;
  for (uint32_t k = 0; k < n; k++) {
    const uint32_t f = Y.eight[k];
    const uint64_t numel = Y.recs[k].numel;
    // (a tile of the norm is so many bytes: of bf16 twice the elements)
    if (Y.counted[k]) runs[kNorm].add(k, Y.recs[k].grad_f32 ? numel : (numel + 1) / 2);
    runs[kStep + f].add(k, numel);
    runs[kConvert + f].add(k, numel);
    if (!sums || !numel) continue;
    Runs& w = runs[kSum + f];
    const uint64_t first = w.n();
    w.add(k, numel);
    const uint64_t tiles = w.n() - first;
    // chunk i of an array holds this many elements, and so these tiles
    const uint64_t per[kSummed] = {o->C / 2, o->C / 4, f ? o->C : o->C / 4, f ? o->C : o->C / 4};
    for (uint32_t j = 0; j < kKinds; j++) {
      if (Y.recs[k].at[j] == kNone) continue;
      const uint32_t chunk0 = Y.chunk0[size_t(k) * kKinds + j], n_chunks = Y.n_chunks[size_t(k) * kKinds + j];
      for (uint32_t i = 0; i < n_chunks; i++) {
        if (j < kSummed) {
          const uint64_t t = per[j] / w.tile;
          folds[f].push_back({chunk0 + i, uint32_t(first + i * t), uint32_t(std::min(t, tiles - i * t)), j});
        } else {
          const uint64_t words = o->C / 4, from = i * words;
          scales[f].push_back({Y.recs[k].at[j] + i * o->C, uint32_t(std::min(words, blocks_of(numel) - from)), chunk0 + i});
        }
      }
    }
  }
  // (a summing step of the same tiles walks the step's table)
  auto shares_step = [&](int w) { return (w == kSum || w == kSum + 1) && runs[w].tile == runs[w - 2].tile; };
  Carver c;
  const size_t recs = c.add(Y.recs.data(), n * sizeof(AdamwRec));
  const fr_grad_stats neutral = {0.0, 0.0f, 1.0f, 0};
  const size_t ns = c.add(&neutral, sizeof neutral);
  const size_t np = c.add(nullptr, (8 * runs[kNorm].stride() + kNormFold) * sizeof(double));
  const size_t ar = c.add(nullptr, kNormArriveBytes);
  size_t fi[kWalks], ba[kWalks], sl[kWalks], pt[2], fo[2], sc[2];
  for (int w = 0; w < kWalks; w++) {
    fi[w] = c.add(runs[w].first.data(), runs[w].first.size() * 8);
    ba[w] = c.add(runs[w].base.data(), runs[w].base.size() * 8);
    sl[w] = c.add(nullptr, shares_step(w) ? 0 : 8 * runs[w].stride() * 8);
  }
  for (int f = 0; f < 2; f++) {
    pt[f] = c.add(nullptr, 8 * runs[kSum + f].stride() * kSummed * sizeof(fr_chunk_sum));
    fo[f] = c.add(folds[f].data(), folds[f].size() * sizeof(AdamwFold));
    sc[f] = c.add(scales[f].data(), scales[f].size() * sizeof(AdamwScales));
  }
  o->layout.info.device_bytes = c.total;
  hipError_t e = hipMalloc(&o->mem, c.total);
  if (e != hipSuccess) {
    o->mem = nullptr;
    (void)hipGetLastError();
    return e == hipErrorOutOfMemory ? FR_E_NOMEM : device_error(e);
  }
  // a stream of its own, as for plans: work queued elsewhere is not waited for
  hipStream_t s = nullptr;
  e = hipStreamCreateWithFlags(&s, hipStreamNonBlocking);
  if (e != hipSuccess) return device_error(e);
  uint8_t* base = static_cast<uint8_t*>(o->mem);
  auto at = [&](size_t i) { return base + c.pieces[i].at; };
  for (const Carver::Piece& p : c.pieces)
    if (e == hipSuccess && p.src && p.bytes)
      e = hipMemcpyAsync(base + p.at, p.src, p.bytes, hipMemcpyHostToDevice, s);
  if (e == hipSuccess) e = hipMemsetAsync(at(ar), 0, kNormArriveBytes, s);
  AdamwWalk* walks[kWalks] = {&o->norm, &o->form[0].step, &o->form[1].step, &o->form[0].sum, &o->form[1].sum,
                              &o->form[0].convert, &o->form[1].convert};
  for (int w = 0; w < kWalks; w++) {
    if (shares_step(w)) {
      *walks[w] = *walks[w - 2];
      continue;
    }
    uint64_t* d = reinterpret_cast<uint64_t*>(at(sl[w]));
    *walks[w] = AdamwWalk{d, runs[w].n(), runs[w].stride()};
    if (e == hipSuccess && runs[w].n())
      e = hipError_t(launch_expand_slots(reinterpret_cast<const uint64_t*>(at(fi[w])),
                                         reinterpret_cast<const uint64_t*>(at(ba[w])), runs[w].base.size(), runs[w].n(),
                                         runs[w].stride(), d, s));
  }
  const hipError_t es = hipStreamSynchronize(s);
  (void)hipStreamDestroy(s);
  if (e != hipSuccess || es != hipSuccess) return device_error(e != hipSuccess ? e : es);
  o->d_recs = reinterpret_cast<const AdamwRec*>(at(recs));
  o->no_stats = reinterpret_cast<const fr_grad_stats*>(at(ns));
  o->norm_parts = reinterpret_cast<double*>(at(np));
  o->arrived = reinterpret_cast<uint32_t*>(at(ar));
  for (int f = 0; f < 2; f++) {
    o->form[f].parts = reinterpret_cast<fr_chunk_sum*>(at(pt[f]));
    o->form[f].folds = reinterpret_cast<const AdamwFold*>(at(fo[f]));
    o->form[f].scales = reinterpret_cast<const AdamwScales*>(at(sc[f]));
    o->form[f].n_folds = uint32_t(folds[f].size());
    o->form[f].n_scales = uint32_t(scales[f].size());
  }
  return FR_OK;
}

}  // namespace

extern "C" int fr_adamw_create(const fr_plan* plan, const fr_adamw_tensor* tensors, uint32_t n,
                               uint32_t n_groups, uint64_t grad_arena_bytes, fr_adamw** out) {
  if (!plan || !out) return FR_E_INVAL;
  fr_adamw* o = nullptr;
  try {
    o = new fr_adamw();
    int rc = validate(plan->table.data(), uint32_t(plan->table.size()), plan->layout, plan->src_arena_bytes,
                      tensors, n, n_groups, grad_arena_bytes, &o->layout);
    if (rc == FR_OK) rc = check_device_and_stream(plan->device, nullptr);
    if (rc == FR_OK) {
      o->device = plan->device;
      o->layout.info.device = plan->device;
      o->C = plan->layout.C;
      o->plan_chunks = plan->layout.n_chunks;
      rc = build(o);
    }
    if (rc != FR_OK) {
      fr_adamw_destroy(o);
      return rc;
    }
  } catch (const std::bad_alloc&) {
    fr_adamw_destroy(o);
    return FR_E_NOMEM;
  }
  *out = o;
  return FR_OK;
}

extern "C" int fr_adamw_get_info(const fr_adamw* opt, fr_adamw_info* out) {
  if (!opt || !out) return FR_E_INVAL;
  *out = opt->layout.info;
  return FR_OK;
}

extern "C" int fr_adamw_destroy(fr_adamw* o) {
  if (!o) return FR_OK;
  int prev = -1;
  bool switched = false;
  if (o->device >= 0 && hipGetDevice(&prev) == hipSuccess && prev != o->device)
    switched = hipSetDevice(o->device) == hipSuccess;
  if (o->mem) (void)hipFree(o->mem);
  if (switched) (void)hipSetDevice(prev);
  delete o;
  return FR_OK;
}

extern "C" int fr_adamw_query(const fr_tensor_desc* table, uint32_t n_entries, uint64_t chunk_bytes,
                              uint64_t arena_bytes, const fr_adamw_tensor* tensors, uint32_t n,
                              uint32_t n_groups, uint64_t grad_arena_bytes, fr_adamw_info* info) {
  if (!info) return FR_E_INVAL;
  try {
    Layout L;
    // (the receiver's side of the table is not the step's)
    FR_TRY(validate_and_layout(table, n_entries, chunk_bytes, kDefaultSegmentAlign, arena_bytes,
                               uint64_t(1) << 62, &L));
    AdamwLayout Y;
    FR_TRY(validate(table, n_entries, L, arena_bytes, tensors, n, n_groups, grad_arena_bytes, &Y));
    *info = Y.info;
  } catch (const std::bad_alloc&) {
    return FR_E_NOMEM;
  }
  return FR_OK;
}

extern "C" int fr_adamw_state_table(const uint64_t* numel, const uint8_t* bits, uint32_t n,
                                    uint32_t grad_dtype, fr_tensor_desc* table, uint32_t cap,
                                    uint32_t* n_entries, fr_adamw_tensor* tensors, uint64_t* arena_bytes,
                                    uint64_t* grad_bytes) {
  if (!n_entries || !arena_bytes || !grad_bytes || (n && !numel)) return FR_E_INVAL;
  if (grad_dtype != FR_F32 && grad_dtype != FR_BF16) return FR_E_INVAL;
  const uint64_t gsize = grad_dtype == FR_F32 ? 4 : 2;
  uint64_t want = 0, elements = 0, off = 0, goff = 0;
  for (uint32_t k = 0; k < n; k++) {
    if (bits && bits[k] != 32 && bits[k] != 8) return FR_E_INVAL;
    if (numel[k] > (uint64_t(1) << 48)) return FR_E_RANGE;
    want += bits && bits[k] == 8 ? 6 : 4;
    elements += numel[k];
    // (at most 14 bytes each, and 90 for a tensor's last ones: below 2^62)
    if (want > 0x7FFFFFFFu || elements > (uint64_t(1) << 58)) return FR_E_RANGE;
  }
  *n_entries = uint32_t(want);
  if (table && cap < want) return FR_E_RANGE;
  uint32_t e = 0;
  for (uint32_t k = 0; k < n; k++) {
    const bool eight = bits && bits[k] == 8;
    const uint64_t mom = eight ? (numel[k] + 3) / 4 : numel[k], bl = blocks_of(numel[k]);
    const uint64_t counts[6] = {numel[k], numel[k], mom, eight ? bl : mom, mom, bl};
    const uint32_t e0 = e;
    for (int j = 0; j < (eight ? 6 : 4); j++, e++) {
      if (table) {
        fr_tensor_desc& d = table[e];
        d.src_offset = d.dst_offset = off;
        d.numel = counts[j];
        d.dtype = j == 0 ? FR_BF16 : FR_F32;
        d.derive_from = j == 0 ? int32_t(e0 + 1) : -1;
      }
      off += (counts[j] * (j == 0 ? 2 : 4) + 15) & ~uint64_t(15);
    }
    if (tensors) {
      fr_adamw_tensor& t = tensors[k];
      std::memset(&t, 0, sizeof t);
      t.grad_offset = goff;
      t.grad_dtype = grad_dtype;
      t.param = int32_t(e0);
      t.master = int32_t(e0 + 1);
      t.m = int32_t(e0 + 2);
      t.v = int32_t(e0 + (eight ? 4 : 3));
      t.m_scale = eight ? int32_t(e0 + 3) : -1;
      t.v_scale = eight ? int32_t(e0 + 5) : -1;
    }
    goff += (numel[k] * gsize + 15) & ~uint64_t(15);
  }
  *arena_bytes = off;
  *grad_bytes = goff;
  return FR_OK;
}

// --------------------------------------------------------------- operations

extern "C" int fr_grad_norm(const fr_adamw* opt, const void* grads, float max_norm, fr_grad_stats* stats,
                            hipStream_t stream) {
  if (!opt || !stats || !(max_norm > 0)) return FR_E_INVAL;
  const uint64_t gb = opt->layout.info.grad_arena_bytes;
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_buffer(opt->device, grads, gb, 16));
  FR_TRY(check_buffer(opt->device, stats, sizeof(fr_grad_stats), 8));
  const Region outs[] = {{stats, sizeof(fr_grad_stats)}}, ins[] = {{grads, gb}};
  FR_TRY(check_disjoint(outs, 1, ins, 1));
  AdamwNormArgs a;
  a.recs = opt->d_recs;
  a.walk = opt->norm;
  a.grads = grads;
  a.max_norm = max_norm;
  a.stats = stats;
  a.parts = opt->norm_parts;
  a.arrived = opt->arrived;
  return launch_result(launch_adamw_norm(a, stream));
}

extern "C" int fr_grad_scale(const fr_adamw* opt, float max_norm, fr_grad_stats* stats, hipStream_t stream) {
  if (!opt || !stats || !(max_norm > 0)) return FR_E_INVAL;
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_buffer(opt->device, stats, sizeof(fr_grad_stats), 8));
  return launch_result(launch_adamw_scale(max_norm, stats, stream));
}

extern "C" int fr_adamw_step(const fr_adamw* opt, void* state, const void* grads, const fr_adamw_hyper* hyper,
                             const fr_grad_stats* stats, fr_chunk_sum* sums, hipStream_t stream) {
  if (!opt) return FR_E_INVAL;
  const fr_adamw_info& info = opt->layout.info;
  if (sums && opt->C < FR_ADAMW_MIN_SUM_CHUNK) return FR_E_INVAL;
  const uint64_t hb = info.n_groups * sizeof(fr_adamw_hyper);
  const uint64_t sb = sums ? opt->plan_chunks * sizeof(fr_chunk_sum) : 0;
  const uint64_t tb = stats ? sizeof(fr_grad_stats) : 0;
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_buffer(opt->device, state, info.arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, grads, info.grad_arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, hyper, hb, 16));
  FR_TRY(check_buffer(opt->device, stats, tb, 8));
  FR_TRY(check_buffer(opt->device, sums, sb, 16));
  const Region outs[] = {{state, info.arena_bytes}, {sums, sb}};
  const Region ins[] = {{grads, info.grad_arena_bytes}, {hyper, hb}, {stats, tb}};
  FR_TRY(check_disjoint(outs, 2, ins, 3));
  for (int f = 0; f < 2; f++) {
    const fr_adamw::Form& F = opt->form[f];
    AdamwStepArgs a;
    a.recs = opt->d_recs;
    a.walk = sums ? F.sum : F.step;
    if (a.walk.n == 0) continue;
    a.eight = f == 1;
    a.state = state;
    a.grads = grads;
    a.hyper = hyper;
    a.stats = stats ? stats : opt->no_stats;
    if (sums) {
      a.C = opt->C;
      a.parts = F.parts;
      a.folds = F.folds;
      a.scales = F.scales;
      a.n_folds = F.n_folds;
      a.n_scales = F.n_scales;
      a.sums = sums;
    }
    FR_TRY(launch_result(launch_adamw_step(a, stream)));
  }
  return FR_OK;
}

extern "C" int fr_adamw_convert(const fr_adamw* from, const void* from_state, const fr_adamw* to, void* to_state,
                                uint32_t seed, hipStream_t stream) {
  if (!from || !to || from == to) return FR_E_INVAL;
  const AdamwLayout &X = from->layout, &Y = to->layout;
  if (X.recs.size() != Y.recs.size()) return FR_E_INVAL;
  for (size_t k = 0; k < X.recs.size(); k++)
    if (X.recs[k].numel != Y.recs[k].numel) return FR_E_INVAL;
  if (from->device != to->device) return FR_E_DEVICE_MISMATCH;
  FR_TRY(check_device_and_stream(to->device, stream));
  FR_TRY(check_buffer(to->device, from_state, X.info.arena_bytes, 16));
  FR_TRY(check_buffer(to->device, to_state, Y.info.arena_bytes, 16));
  const Region in = {from_state, X.info.arena_bytes}, out = {to_state, Y.info.arena_bytes};
  if (from_state == to_state ? meet(X.moments, Y.moments) : overlap(in, out)) return FR_E_OVERLAP;
  for (int f = 0; f < 2; f++) {
    AdamwConvertArgs a;
    a.walk = to->form[f].convert;
    if (a.walk.n == 0) continue;
    a.from_recs = from->d_recs;
    a.to_recs = to->d_recs;
    a.eight = f == 1;
    a.from = from_state;
    a.to = to_state;
    a.seed = seed;
    FR_TRY(launch_result(launch_adamw_convert(a, stream)));
  }
  return FR_OK;
}
