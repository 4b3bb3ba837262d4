// The host side of the step by orthogonalised momentum: validation of its
// matrices against a plan's table, its device tables, and the C entry points'
// checks.
#include "muon.h"

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "checks.h"
#include "fr_internal.h"

using namespace fr;

namespace {

constexpr fr_muon_coeffs kCoeffs = {3.4445f, -4.7750f, 2.0315f};
constexpr uint64_t kMaxSide = 1u << 20, kMaxLess = 1u << 15, kMaxNumel = uint64_t(1) << 31;

struct Range {
  uint64_t first, last;
  bool operator<(const Range& o) const { return first < o.first; }
};

bool disjoint(std::vector<Range>& r) {
  std::sort(r.begin(), r.end());
  for (size_t i = 1; i < r.size(); i++)
    if (r[i].first < r[i - 1].last) return false;
  return true;
}

// What an optimizer is, before the device knows of it.
struct MuonLayout {
  std::vector<MuonRec> recs;
  // first chunks, and how many, of each matrix's param, master and momentum
  std::vector<uint32_t> chunk0, n_chunks;
  std::vector<fr_muon_coeffs> coeffs;
  bool pair = false;
  uint32_t side = kMuonSmall;
  uint64_t scratch = 0;  // bytes
  fr_muon_info info{};
};

uint64_t up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

int check_shape(uint64_t rows, uint64_t cols) {
  if (rows > kMaxSide || cols > kMaxSide || rows * cols >= kMaxNumel || std::min(rows, cols) > kMaxLess)
    return FR_E_RANGE;
  return FR_OK;
}

// What operands' roundings may do to a singular value in a step, of itself: as a
// unit half a step of fp16, and twice that where range is at stake.
constexpr double kUnit = 1.0 / 2048, kMargin = 2 * kUnit;

// Whether the steps keep every singular value that starts in [0, 1], and the
// polynomial's parts, inside what fp16 operands can hold with the powers of two
// that they are stored times; and so that it holds for the values that roundings
// leave, not for exact ones alone:
//   * up to 4 and 64 exactly, up to 8 and 128 where everything that a step may
//     leave is up to kMargin larger (of 16 and 256, where A and Q pass fp16's
//     range).  Steps made for [0, 1] and no further, with a slope of 12 at its end,
//     leave values of 1e21 so.
//   * errors of kUnit in each step come to 4 at most in the last X, by the slopes
//     of the steps behind them: to 0.014 with kCoeffs, 0.12 with steps that start
//     with a slope of 8, 2.1 with kCoeffs 16 times; 50,000 with 16 steps that each
//     tear neighbours apart.
// *pair: those of the first two steps taken as one as well.
int check_coeffs(const fr_muon_coeffs* c, uint32_t n, std::vector<fr_muon_coeffs>* out, bool* pair) {
  if (!c && n) return FR_E_INVAL;
  if (c && (n < 1 || n > FR_MUON_MAX_STEPS)) return FR_E_INVAL;
  if (c) out->assign(c, c + n);
  else out->assign(5, kCoeffs);
  for (const fr_muon_coeffs& k : *out)
    if (!std::isfinite(k.a) || !std::isfinite(k.b) || !std::isfinite(k.c)) return FR_E_INVAL;
  *pair = out->size() >= 2;
  constexpr int kGrid = 4096;
  // (compared so that an overflow is a refusal)
  for (int i = 0; i <= kGrid; i++) {
    double s = double(i) / kGrid, error = kUnit * s;
    if (*pair) {
      const fr_muon_coeffs &f = (*out)[0], &g = (*out)[1];
      const double q = s * s, one = f.b * q + f.c * q * q, p = q * (f.a + one) * (f.a + one), two = g.b * p + g.c * p * p;
      *pair = std::fabs(f.a * two) + std::fabs(g.a * one) + std::fabs(one * two) <= 64;
    }
    for (const fr_muon_coeffs& k : *out) {
      const double q = s * s;
      if (!(std::fabs(k.b) * q + std::fabs(k.c) * q * q <= 64)) return FR_E_INVAL;
      error *= std::fabs(k.a + 3 * k.b * q + 5 * k.c * q * q);
      s *= k.a + k.b * q + k.c * q * q;
      if (!(std::fabs(s) <= 4)) return FR_E_INVAL;
      error += kUnit * std::fabs(s);
    }
    if (!(error <= 4)) return FR_E_INVAL;
  }
  double top = 1 + kMargin;  // everything up to here may come
  for (const fr_muon_coeffs& k : *out) {
    if (!(std::fabs(k.b) * top * top + std::fabs(k.c) * top * top * top * top <= 128)) return FR_E_INVAL;
    double next = 0;
    for (int i = 1; i <= kGrid; i++) {
      const double s = top * i / kGrid, q = s * s;
      next = std::max(next, std::fabs(s * (k.a + k.b * q + k.c * q * q)));
    }
    top = next * (1 + kMargin);
    if (!(top <= 8)) return FR_E_INVAL;
  }
  return FR_OK;
}

// Multiplications of a step of all matrices in tiles of this side, symmetric
// products by tiles on and below the diagonal.
double in_tiles(const std::vector<MuonRec>& recs, uint32_t side) {
  double sum = 0;
  for (const MuonRec& r : recs) {
    if (!r.numel) continue;
    const double m = double(up(r.m, side)), n = double(up(r.n, side));
    sum += (m + side) * m / 2 * (m + n) + m * m * n;
  }
  return sum;
}

// Which tiles the products take, and where in the scratch their operands lie.
// Large ones where the matrices have the elements of 256, one for each compute unit,
// and rounding their sides up costs no more than half the multiplications again
// (which is what large tiles are faster by).  Large and small, us:
//   by elements, of 1024 x 1024 matrices those of 64 tiles 524 and 313, of 128 544
//     and 506, of 192 564 and 688, of 256 586 and 874, of 512 1,197 and 1,713; of 2048 x
//     4096 128 1,055 and 674, 256 1,121 and 1,129, 384 1,349 and 1,630; one of 4096 x
//     4096 1,623 and 2,642; 20 of 900 x 900 (247 tiles' elements in 320 tiles) 769 and
//     970; 40 of 200 to 1,400 (201 in 274) 764 and 595;
//   by multiplications, times those in small tiles: 1.3 256 of 256 x 256 399 and 514;
//     1.4 8 of 1100 x 2100 969 and 976; 1.45 90 of 700 x 700 1,809 and 2,064; 1.55 16 of
//     512 x 4096 with 32 of 128 x 4096 1,146 and 981; 1.6 30 of 1300 x 1300 2,979 and
//     3,443; 1.75 300 of 448 x 448 2,074 and 2,362, 4 of 2048 x 2048 with 100 of 16 x 4096
//     2,141 and 1,697; 1.9 100 of 600 x 600 1,836 and 1,787; 2.1 4 of 2048 x 2048 with 1,500
//     of 64 x 64 3,197 and 1,517; 2.7 600 of 384 x 384 4,016 and 3,369; 4.7 64 of 128 x 4096
//     1,012 and 458; 64 4,096 of 64 x 64 5,691 and 508.
void lay_out_scratch(MuonLayout* out) {
  uint64_t elements = 0;
  for (const MuonRec& r : out->recs) elements += r.numel;
  const bool large = elements >= uint64_t(256) * kMuonLarge * kMuonLarge &&
                     in_tiles(out->recs, kMuonLarge) <= 1.5 * in_tiles(out->recs, kMuonSmall);
  out->side = large ? kMuonLarge : kMuonSmall;
  for (MuonRec& r : out->recs) {
    r.paired = out->pair && r.m >= kMuonPairedLess && r.n >= kMuonPairedMore && r.n >= kMuonPairedRatio * r.m;
    r.mp = uint32_t(up(r.m, out->side));
    r.np = uint32_t(up(r.n, out->side));
    if (!r.numel) continue;
    const uint64_t wide = uint64_t(r.mp) * r.np, square = uint64_t(r.mp) * r.mp;
    const struct {
      uint64_t* where;
      uint64_t bytes;
    } parts[9] = {{&r.x[0], 2 * wide},          {&r.x[1], 2 * wide},          {&r.rest, wide},
                  {&r.square[0], 2 * square},   {&r.square[1], 2 * square},   {&r.square[2], 2 * square},
                  {&r.diagonal[0], 4ull * r.mp}, {&r.diagonal[1], 4ull * r.mp}, {&r.diagonal[2], 4ull * r.mp}};
    for (const auto& p : parts) {
      *p.where = out->scratch;
      out->scratch += p.bytes;
    }
  }
}

int validate(const fr_tensor_desc* table, uint32_t n_entries, const Layout& L, uint64_t arena_bytes,
             const fr_muon_tensor* t, uint32_t n, uint32_t n_groups, uint64_t grad_bytes, uint64_t update_bytes,
             const fr_muon_coeffs* coeffs, uint32_t n_steps, MuonLayout* out) {
  if (n && !t) return FR_E_INVAL;
  FR_TRY(check_coeffs(coeffs, n_steps, &out->coeffs, &out->pair));
  std::vector<uint8_t> named(n_entries, 0);
  std::vector<Range> written, updated;
  out->recs.resize(n);
  out->chunk0.assign(size_t(n) * 3, 0);
  out->n_chunks.assign(size_t(n) * 3, 0);
  fr_muon_info& info = out->info;
  info.n_tensors = n;
  info.n_groups = n_groups;
  info.n_steps = out->coeffs.size();
  info.grad_arena_bytes = grad_bytes;
  info.update_arena_bytes = update_bytes;
  info.arena_bytes = arena_bytes;
  info.device = -1;
  bool twice = false, strange = false;
  uint64_t tiles = 0, subs = 0;
  for (uint32_t k = 0; k < n; k++) {
    const fr_muon_tensor& d = t[k];
    if (d.reserved || d.flags || d.group >= n_groups || !std::isfinite(d.scale)) return FR_E_INVAL;
    if (d.grad_dtype != FR_F32 && d.grad_dtype != FR_BF16) return FR_E_INVAL;
    if (d.grad_offset % 16 || d.update_offset % 16) return FR_E_ALIGN;
    FR_TRY(check_shape(d.rows, d.cols));
    const uint64_t numel = uint64_t(d.rows) * d.cols;
    if (d.master < 0 || uint32_t(d.master) >= n_entries) return FR_E_INVAL;
    MuonRec& r = out->recs[k];
    std::memset(&r, 0, sizeof r);
    r.param = kNone;
    const struct {
      int32_t entry;
      uint32_t dtype;
      bool may_miss;
      uint64_t* at;
    } want[3] = {{d.param, FR_BF16, true, &r.param}, {d.master, FR_F32, false, &r.master}, {d.m, FR_F32, false, &r.mom}};
    for (uint32_t j = 0; j < 3; j++) {
      if (want[j].entry < 0) {
        if (want[j].entry != -1 || !want[j].may_miss) return FR_E_INVAL;
        continue;
      }
      const uint32_t e = uint32_t(want[j].entry);
      if (e >= n_entries || table[e].dtype != want[j].dtype || table[e].numel != numel) return FR_E_INVAL;
      if (j == 0) strange |= numel && table[e].derive_from != -1 && table[e].derive_from != d.master;
      twice |= named[e] != 0;
      named[e] = 1;
      *want[j].at = table[e].src_offset;
      const uint64_t bytes = numel * (want[j].dtype == FR_F32 ? 4 : 2);
      if (bytes) written.push_back({*want[j].at, *want[j].at + bytes});
      out->chunk0[size_t(k) * 3 + j] = uint32_t(L.chunk_base[e]);
      out->n_chunks[size_t(k) * 3 + j] = uint32_t(L.chunk_base[e + 1] - L.chunk_base[e]);
      if (L.C >= FR_ADAMW_MIN_SUM_CHUNK) info.sums_chunks += L.chunk_base[e + 1] - L.chunk_base[e];
    }
    const uint64_t gb = numel * (d.grad_dtype == FR_F32 ? 4 : 2);
    if (d.grad_offset > grad_bytes || gb > grad_bytes - d.grad_offset) return FR_E_RANGE;
    if (d.update_offset > update_bytes || 2 * numel > update_bytes - d.update_offset) return FR_E_RANGE;
    if (numel) updated.push_back({d.update_offset, d.update_offset + 2 * numel});
    r.numel = numel;
    r.grad = d.grad_offset;
    r.update = d.update_offset;
    r.grad_f32 = d.grad_dtype == FR_F32;
    r.group = d.group;
    r.scale = d.scale;
    r.cols = d.cols;
    r.wide = d.rows <= d.cols;
    r.m = std::min(d.rows, d.cols);
    r.n = std::max(d.rows, d.cols);
    // entries of X_0 are some 1 / sqrt(m n), of an orthogonal matrix 1 / sqrt(n)
    r.lift = float(std::ldexp(1.0, int(std::lround(0.5 * std::log2(double(std::max(r.n, 1u)))))));
    info.n_elements += numel;
    info.multiplications += info.n_steps * (numel * (r.m + 1) / 2 + uint64_t(r.m) * r.m * (r.m + 1) / 2 + numel * r.m);
    r.slot0 = tiles;
    r.slots = (numel + kMuonTile - 1) / kMuonTile;
    tiles += r.slots;
    r.sub0 = subs;
    subs += (numel + kMuonSub - 1) / kMuonSub;
  }
  lay_out_scratch(out);
  if (twice) return FR_E_OVERLAP;
  if (!disjoint(written) || !disjoint(updated)) return FR_E_OVERLAP;
  if (strange) return FR_E_INVAL;
  // a launch has fewer than 2^32 threads, 256 or 512 a tile
  uint64_t spread = 0, products = 0;
  for (const MuonRec& r : out->recs) {
    if (!r.numel) continue;
    spread += uint64_t(r.mp) * r.np / 4096;
    products += uint64_t(r.mp / out->side) * (r.np / out->side);
  }
  if (tiles >= (uint64_t(1) << 22) - 8 || spread >= (uint64_t(1) << 24) || products >= (uint64_t(1) << 23))
    return FR_E_RANGE;
  return FR_OK;
}

}  // namespace

struct fr_muon {
  int device = -1;
  MuonLayout layout;
  uint64_t C = 0, plan_chunks = 0;
  void* mem = nullptr;  // everything below
  MuonArgs args;        // but for a call's buffers
  const AdamwFold* mom_folds = nullptr;   // of the momenta's chunks, which direction writes,
  const AdamwFold* step_folds = nullptr;  // and of the parameters' and masters', which apply does
  uint32_t n_mom_folds = 0, n_step_folds = 0;
  fr_chunk_sum* sum_parts = nullptr;
  const fr_grad_stats* no_stats = nullptr;
  AdamwNormArgs norm;  // but for a call's buffers
};

namespace {

struct Carver {
  struct Piece {
    const void* src;
    uint64_t bytes, at;
  };
  std::vector<Piece> pieces;
  uint64_t total = 0;
  size_t add(const void* src, uint64_t bytes) {
    pieces.push_back({src, bytes, total});
    total += up(bytes, 256);
    return pieces.size() - 1;
  }
};

// The tiles of a product over all matrices, those of the longest sums first, so
// that no workgroup starts a long one last.  Workgroup b runs on die b mod 8, and
// each die takes runs of kRun tiles in order, which share most of their operands'
// rows, from its own L2.
struct TileList {
  static constexpr size_t kRun = 16;
  struct Item {
    uint64_t tile;  // (matrix << 32) | (row << 16) | column
    uint32_t k;
  };
  std::vector<Item> items;
  std::vector<MuonTile> dealt(const std::vector<MuonRec>& recs, uint32_t side) {
    std::stable_sort(items.begin(), items.end(), [](const Item& a, const Item& b) { return a.k > b.k; });
    const size_t n = items.size(), whole = n / (8 * kRun) * (8 * kRun);
    std::vector<MuonTile> d(n);
    for (size_t b = 0; b < n; b++) {
      const size_t i = b % (8 * kRun);
      const uint64_t t = items[b < whole ? b - i + i % 8 * kRun + i / 8 : b].tile;
      d[b] = MuonTile{recs[t >> 32], uint32_t(t >> 16 & 0xFFFF) * side, uint32_t(t & 0xFFFF) * side, 0};
    }
    return d;
  }
};

int build(fr_muon* o) {
  const MuonLayout& Y = o->layout;
  const uint32_t n = uint32_t(Y.recs.size());
  std::vector<uint64_t> walk;
  std::vector<uint64_t> spread;
  TileList gram[3], whole[3];
  std::vector<AdamwFold> mom, step;
  const bool sums = o->C >= FR_ADAMW_MIN_SUM_CHUNK;
  uint64_t slots = 0, subs = 0;
  for (const MuonRec& r : Y.recs) {
    slots += r.slots;
    subs += (r.numel + kMuonSub - 1) / kMuonSub;
  }
  const uint64_t stride = (slots + 7) / 8, sub_stride = (subs + 7) / 8;
  walk.assign(8 * stride, 0);
  for (uint32_t k = 0; k < n; k++) {
    const MuonRec& r = Y.recs[k];
    const uint64_t id = uint64_t(k) << 32;
    for (uint64_t i = 0; i < r.slots; i++) {
      const uint64_t g = r.slot0 + i;
      walk[(g & 7) * stride + (g >> 3)] = id | i;
    }
    if (!r.numel) continue;
    const uint32_t tm = r.mp / Y.side, tn = r.np / Y.side;
    for (uint32_t of : {r.paired, 2u}) {
      for (uint32_t i = 0; i < tm; i++)
        for (uint32_t j = 0; j <= i; j++) gram[of].items.push_back({id | uint64_t(i) << 16 | j, r.np});
      for (uint32_t j = 0; j < tn; j++)
        for (uint32_t i = 0; i < tm; i++) whole[of].items.push_back({id | uint64_t(i) << 16 | j, r.mp});
    }
    for (uint64_t i = 0; i < uint64_t(r.mp) * r.np / 4096; i++) spread.push_back(id | i);
    if (!sums) continue;
    // chunk i of an array holds this many elements, and so these tiles
    const uint64_t per[3] = {o->C / 2, o->C / 4, o->C / 4};
    for (uint32_t j = 0; j < 3; j++)
      for (uint32_t i = 0; i < Y.n_chunks[size_t(k) * 3 + j]; i++) {
        const uint64_t t = per[j] / kMuonSub, all = (r.numel + kMuonSub - 1) / kMuonSub;
        const AdamwFold f = {Y.chunk0[size_t(k) * 3 + j] + i, uint32_t(r.sub0 + i * t),
                             uint32_t(std::min(t, all - i * t)), j == 2 ? 0 : j};
        (j == 2 ? mom : step).push_back(f);
      }
  }
  std::vector<MuonTile> t_gram[3], t_whole[3];
  for (int i = 0; i < 3; i++) {
    t_gram[i] = gram[i].dealt(Y.recs, Y.side);
    t_whole[i] = whole[i].dealt(Y.recs, Y.side);
  }
  // the gradients' norm is AdamW's, over tiles of kNormBytes
  std::vector<AdamwRec> tensors(n);
  uint64_t norm_slots = 0;
  const auto norm_tiles = [](const MuonRec& r) { return (r.numel * (r.grad_f32 ? 4 : 2) + kNormBytes - 1) / kNormBytes; };
  for (uint32_t k = 0; k < n; k++) {
    std::memset(&tensors[k], 0, sizeof tensors[k]);
    tensors[k].numel = Y.recs[k].numel;
    tensors[k].grad = Y.recs[k].grad;
    tensors[k].grad_f32 = Y.recs[k].grad_f32;
    norm_slots += norm_tiles(Y.recs[k]);
  }
  const uint64_t norm_stride = (norm_slots + 7) / 8;
  std::vector<uint64_t> norm_walk(8 * norm_stride, 0);
  for (uint64_t k = 0, g = 0; k < n; k++)
    for (uint64_t i = 0; i < norm_tiles(Y.recs[k]); i++, g++) norm_walk[(g & 7) * norm_stride + (g >> 3)] = k << 32 | i;
  Carver c;
  const size_t nt = c.add(tensors.data(), n * sizeof(AdamwRec)), nw = c.add(norm_walk.data(), norm_walk.size() * 8);
  const size_t nn = c.add(nullptr, (8 * norm_stride + kNormFold) * sizeof(double)), na = c.add(nullptr, kNormArriveBytes);
  const size_t recs = c.add(Y.recs.data(), n * sizeof(MuonRec));
  const fr_grad_stats neutral = {0.0, 0.0f, 1.0f, 0};
  const size_t ns = c.add(&neutral, sizeof neutral);
  const size_t wa = c.add(walk.data(), walk.size() * 8);
  size_t tg[3], tw[3];
  for (int i = 0; i < 3; i++) {
    tg[i] = c.add(t_gram[i].data(), t_gram[i].size() * sizeof(MuonTile));
    tw[i] = c.add(t_whole[i].data(), t_whole[i].size() * sizeof(MuonTile));
  }
  const size_t ts = c.add(spread.data(), spread.size() * 8);
  const size_t fm = c.add(mom.data(), mom.size() * sizeof(AdamwFold));
  const size_t fs = c.add(step.data(), step.size() * sizeof(AdamwFold));
  const size_t np = c.add(nullptr, 8 * stride * sizeof(double));
  const size_t nf = c.add(nullptr, n * sizeof(double));
  const size_t sp = c.add(nullptr, sums ? 2 * 8 * sub_stride * sizeof(fr_chunk_sum) : 0);
  const size_t sc = c.add(nullptr, Y.scratch);
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
  if (e == hipSuccess) e = hipMemsetAsync(at(na), 0, kNormArriveBytes, s);
  const hipError_t es = hipStreamSynchronize(s);
  (void)hipStreamDestroy(s);
  if (e != hipSuccess || es != hipSuccess) return device_error(e != hipSuccess ? e : es);
  o->norm.recs = reinterpret_cast<const AdamwRec*>(at(nt));
  o->norm.walk = AdamwWalk{reinterpret_cast<const uint64_t*>(at(nw)), norm_slots, norm_stride};
  o->norm.parts = reinterpret_cast<double*>(at(nn));
  o->norm.arrived = reinterpret_cast<uint32_t*>(at(na));
  int units = 0;
  e = hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, o->device);
  if (e != hipSuccess) return device_error(e);
  MuonArgs& a = o->args;
  a.units = uint32_t(units);
  a.recs = reinterpret_cast<const MuonRec*>(at(recs));
  a.n = n;
  a.side = Y.side;
  a.walk = AdamwWalk{reinterpret_cast<const uint64_t*>(at(wa)), slots, stride};
  a.scratch = at(sc);
  a.sub_stride = sub_stride;
  a.few_slots = true;
  for (const MuonRec& r : Y.recs) a.few_slots &= r.slots <= 256;
  a.parts = reinterpret_cast<double*>(at(np));
  a.factors = reinterpret_cast<double*>(at(nf));
  a.spread = reinterpret_cast<const uint64_t*>(at(ts));
  a.n_spread = spread.size();
  for (int i = 0; i < 3; i++) {
    a.gram[i] = MuonTiles{reinterpret_cast<const MuonTile*>(at(tg[i])), t_gram[i].size()};
    a.whole[i] = MuonTiles{reinterpret_cast<const MuonTile*>(at(tw[i])), t_whole[i].size()};
  }
  a.coeffs = Y.coeffs.data();
  a.n_steps = uint32_t(Y.coeffs.size());
  o->mom_folds = reinterpret_cast<const AdamwFold*>(at(fm));
  o->step_folds = reinterpret_cast<const AdamwFold*>(at(fs));
  o->n_mom_folds = uint32_t(mom.size());
  o->n_step_folds = uint32_t(step.size());
  o->sum_parts = reinterpret_cast<fr_chunk_sum*>(at(sp));
  o->no_stats = reinterpret_cast<const fr_grad_stats*>(at(ns));
  return FR_OK;
}

}  // namespace

extern "C" int fr_muon_create(const fr_plan* plan, const fr_muon_tensor* tensors, uint32_t n, uint32_t n_groups,
                              uint64_t grad_arena_bytes, uint64_t update_arena_bytes, const fr_muon_coeffs* coeffs,
                              uint32_t n_steps, fr_muon** out) {
  if (!plan || !out) return FR_E_INVAL;
  fr_muon* o = nullptr;
  try {
    o = new fr_muon();
    int rc = validate(plan->table.data(), uint32_t(plan->table.size()), plan->layout, plan->src_arena_bytes, tensors,
                      n, n_groups, grad_arena_bytes, update_arena_bytes, coeffs, n_steps, &o->layout);
    if (rc == FR_OK) rc = check_device_and_stream(plan->device, nullptr);
    if (rc == FR_OK) {
      o->device = plan->device;
      o->layout.info.device = plan->device;
      o->C = plan->layout.C;
      o->plan_chunks = plan->layout.n_chunks;
      rc = build(o);
    }
    if (rc != FR_OK) {
      fr_muon_destroy(o);
      return rc;
    }
  } catch (const std::bad_alloc&) {
    fr_muon_destroy(o);
    return FR_E_NOMEM;
  }
  *out = o;
  return FR_OK;
}

extern "C" int fr_muon_get_info(const fr_muon* opt, fr_muon_info* out) {
  if (!opt || !out) return FR_E_INVAL;
  *out = opt->layout.info;
  return FR_OK;
}

extern "C" int fr_muon_destroy(fr_muon* o) {
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

extern "C" int fr_muon_query(const fr_tensor_desc* table, uint32_t n_entries, uint64_t chunk_bytes,
                             uint64_t arena_bytes, const fr_muon_tensor* tensors, uint32_t n, uint32_t n_groups,
                             uint64_t grad_arena_bytes, uint64_t update_arena_bytes, const fr_muon_coeffs* coeffs,
                             uint32_t n_steps, fr_muon_info* info) {
  if (!info) return FR_E_INVAL;
  try {
    Layout L;
    // (the receiver's side of the table is not the step's)
    FR_TRY(validate_and_layout(table, n_entries, chunk_bytes, kDefaultSegmentAlign, arena_bytes, uint64_t(1) << 62,
                               &L));
    MuonLayout Y;
    FR_TRY(validate(table, n_entries, L, arena_bytes, tensors, n, n_groups, grad_arena_bytes, update_arena_bytes,
                    coeffs, n_steps, &Y));
    *info = Y.info;
  } catch (const std::bad_alloc&) {
    return FR_E_NOMEM;
  }
  return FR_OK;
}

extern "C" int fr_muon_state_table(const uint32_t* shapes, uint32_t n, uint32_t grad_dtype, uint32_t first_entry,
                                   fr_tensor_desc* table, uint32_t cap, uint32_t* n_entries, fr_muon_tensor* tensors,
                                   uint64_t* arena_bytes, uint64_t* grad_bytes, uint64_t* update_bytes) {
  if (!n_entries || !arena_bytes || !grad_bytes || !update_bytes || (n && !shapes)) return FR_E_INVAL;
  if (grad_dtype != FR_F32 && grad_dtype != FR_BF16) return FR_E_INVAL;
  constexpr uint64_t kMaxBytes = uint64_t(1) << 62;
  if (uint64_t(first_entry) + 3 * uint64_t(n) > 0x7FFFFFFFu || *arena_bytes > kMaxBytes || *grad_bytes > kMaxBytes)
    return FR_E_RANGE;
  for (uint32_t k = 0; k < n; k++) FR_TRY(check_shape(shapes[2 * k], shapes[2 * k + 1]));
  // (at most 2^30 matrices of 10 * 2^31 bytes)
  *n_entries = 3 * n;
  if (table && cap < 3 * n) return FR_E_RANGE;
  uint64_t off = up(*arena_bytes, 16), goff = up(*grad_bytes, 16), uoff = 0;
  for (uint32_t k = 0; k < n; k++) {
    const uint32_t rows = shapes[2 * k], cols = shapes[2 * k + 1], e0 = first_entry + 3 * k;
    const uint64_t numel = uint64_t(rows) * cols;
    for (uint32_t j = 0; j < 3; j++) {
      if (table) {
        fr_tensor_desc& d = table[3 * k + j];
        d.src_offset = d.dst_offset = off;
        d.numel = numel;
        d.dtype = j == 0 ? FR_BF16 : FR_F32;
        d.derive_from = j == 0 ? int32_t(e0 + 1) : -1;
      }
      off += up(numel * (j == 0 ? 2 : 4), 16);
    }
    if (tensors) {
      fr_muon_tensor& t = tensors[k];
      std::memset(&t, 0, sizeof t);
      t.grad_offset = goff;
      t.update_offset = uoff;
      t.rows = rows;
      t.cols = cols;
      t.grad_dtype = grad_dtype;
      t.param = int32_t(e0);
      t.master = int32_t(e0 + 1);
      t.m = int32_t(e0 + 2);
      t.scale = float(0.2 * std::sqrt(double(std::max(rows, cols))));
    }
    goff += up(numel * (grad_dtype == FR_F32 ? 4 : 2), 16);
    uoff += up(numel * 2, 16);
  }
  *arena_bytes = off;
  *grad_bytes = goff;
  *update_bytes = uoff;
  return FR_OK;
}

// --------------------------------------------------------------- operations

namespace {

// A call's sums, where asked for.
void take_sums(const fr_muon* o, fr_chunk_sum* sums, const AdamwFold* folds, uint32_t n, MuonArgs* a) {
  if (!sums) return;
  a->C = o->C;
  a->sum_parts = o->sum_parts;
  a->folds = folds;
  a->n_folds = n;
  a->sums = sums;
}

int check_sums(const fr_muon* o, const fr_chunk_sum* sums) {
  if (!sums) return FR_OK;
  return o->C < FR_ADAMW_MIN_SUM_CHUNK ? FR_E_INVAL : check_buffer(o->device, sums, o->plan_chunks * sizeof *sums, 16);
}

}  // namespace

extern "C" int fr_muon_grad_norm(const fr_muon* opt, const void* grads, float max_norm, fr_grad_stats* stats,
                                 hipStream_t stream) {
  if (!opt || !stats || !(max_norm > 0)) return FR_E_INVAL;
  const uint64_t gb = opt->layout.info.grad_arena_bytes;
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_buffer(opt->device, grads, gb, 16));
  FR_TRY(check_buffer(opt->device, stats, sizeof(fr_grad_stats), 8));
  const Region outs[] = {{stats, sizeof(fr_grad_stats)}}, ins[] = {{grads, gb}};
  FR_TRY(check_disjoint(outs, 1, ins, 1));
  AdamwNormArgs a = opt->norm;
  a.grads = grads;
  a.max_norm = max_norm;
  a.stats = stats;
  return launch_result(launch_adamw_norm(a, stream));
}

extern "C" int fr_muon_direction(const fr_muon* opt, void* state, const void* grads, const fr_muon_hyper* hyper,
                                 const fr_grad_stats* stats, void* updates, fr_chunk_sum* sums, hipStream_t stream) {
  if (!opt) return FR_E_INVAL;
  const fr_muon_info& info = opt->layout.info;
  const uint64_t hb = info.n_groups * sizeof(fr_muon_hyper), tb = stats ? sizeof(fr_grad_stats) : 0;
  const uint64_t sb = sums ? opt->plan_chunks * sizeof(fr_chunk_sum) : 0;
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_sums(opt, sums));
  FR_TRY(check_buffer(opt->device, state, info.arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, grads, info.grad_arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, hyper, hb, 16));
  FR_TRY(check_buffer(opt->device, stats, tb, 8));
  FR_TRY(check_buffer(opt->device, updates, info.update_arena_bytes, 16));
  const Region outs[] = {{state, info.arena_bytes}, {updates, info.update_arena_bytes}, {sums, sb}};
  const Region ins[] = {{grads, info.grad_arena_bytes}, {hyper, hb}, {stats, tb}};
  FR_TRY(check_disjoint(outs, 3, ins, 3));
  MuonArgs a = opt->args;
  a.hyper = hyper;
  a.stats = stats ? stats : opt->no_stats;
  a.state = state;
  a.grads = grads;
  a.updates = updates;
  a.momentum = true;
  take_sums(opt, sums, opt->mom_folds, opt->n_mom_folds, &a);
  return launch_result(launch_muon_direction(a, stream));
}

extern "C" int fr_muon_orthogonalize(const fr_muon* opt, const void* grads, const fr_muon_hyper* hyper, void* updates,
                                     hipStream_t stream) {
  if (!opt) return FR_E_INVAL;
  const fr_muon_info& info = opt->layout.info;
  const uint64_t hb = info.n_groups * sizeof(fr_muon_hyper);
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_buffer(opt->device, grads, info.grad_arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, hyper, hb, 16));
  FR_TRY(check_buffer(opt->device, updates, info.update_arena_bytes, 16));
  const Region outs[] = {{updates, info.update_arena_bytes}};
  const Region ins[] = {{grads, info.grad_arena_bytes}, {hyper, hb}};
  FR_TRY(check_disjoint(outs, 1, ins, 2));
  MuonArgs a = opt->args;
  a.hyper = hyper;
  a.stats = opt->no_stats;
  a.grads = grads;
  a.updates = updates;
  return launch_result(launch_muon_direction(a, stream));
}

extern "C" int fr_muon_apply(const fr_muon* opt, void* state, const void* updates, const fr_muon_hyper* hyper,
                             const fr_grad_stats* stats, fr_chunk_sum* sums, hipStream_t stream) {
  if (!opt) return FR_E_INVAL;
  const fr_muon_info& info = opt->layout.info;
  const uint64_t hb = info.n_groups * sizeof(fr_muon_hyper), tb = stats ? sizeof(fr_grad_stats) : 0;
  const uint64_t sb = sums ? opt->plan_chunks * sizeof(fr_chunk_sum) : 0;
  FR_TRY(check_device_and_stream(opt->device, stream));
  FR_TRY(check_sums(opt, sums));
  FR_TRY(check_buffer(opt->device, state, info.arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, updates, info.update_arena_bytes, 16));
  FR_TRY(check_buffer(opt->device, hyper, hb, 16));
  FR_TRY(check_buffer(opt->device, stats, tb, 8));
  const Region outs[] = {{state, info.arena_bytes}, {sums, sb}};
  const Region ins[] = {{updates, info.update_arena_bytes}, {hyper, hb}, {stats, tb}};
  FR_TRY(check_disjoint(outs, 2, ins, 3));
  MuonArgs a = opt->args;
  a.hyper = hyper;
  a.stats = stats ? stats : opt->no_stats;
  a.state = state;
  a.updates = const_cast<void*>(updates);
  take_sums(opt, sums, opt->step_folds, opt->n_step_folds, &a);
  return launch_result(launch_muon_apply(a, stream));
}
