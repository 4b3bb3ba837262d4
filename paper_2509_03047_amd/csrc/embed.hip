// gfx950 kernels of the embedding: rows of the state for a batch of tokens, and
// the gradient that they leave.
//
// The gradient's tokens are brought into the order of their rows by one launch:
// each workgroup owns some hundred rows at most, reads all ids (they stay in L2)
// and so counts the tokens of the rows in front of its own as well as its own's,
// by wave; a second pass puts each token at its place.  Its waves have
// consecutive tokens, so the order within a row is the tokens' own, and nothing
// depends on atomics' order.  A row of more than FR_EMBED_RUN tokens is cut into
// runs: the second launch sums those up and writes the shorter rows, the third adds
// up the runs of the long ones.
//
// What bounds them: HBM, and where there are few tokens the launches.  16,384
// tokens of 4,096 columns, a share of 16,032 rows of the vocabulary, bf16: a lookup
// takes 29 us when called again and again (168 MB, 5.8 TB/s, in part from the
// Infinity Cache; 47 with other rows in between), the order 17 us (two walks over the ids and what
// hangs on them in turn), rows and runs 33 us (177 MB, 5.4 TB/s), the long rows 5 us.
// 2,048 tokens of 256 columns: 9, 10 and 3 us, each of them a launch and a few
// loads that wait for each other.
#include <hip/hip_runtime.h>

#include "embed.h"
#include "elements.h"

#pragma clang fp contract(off)

namespace fr {
namespace {

constexpr uint32_t kRun = FR_EMBED_RUN;
constexpr uint32_t kVec = kEmbedVec;

// A launch's work is cut into units of `lanes` lanes, a power of two: a slice of
// 8 * lanes columns of a row, `slices` of which make up a row.
struct Units {
  uint32_t lanes_log, slices;
  __device__ __forceinline__ uint32_t unit() const { return (blockIdx.x * 256 + threadIdx.x) >> lanes_log; }
  __device__ __forceinline__ uint32_t lane() const { return threadIdx.x & ((1u << lanes_log) - 1); }
};

struct Cols {
  float x[kVec];
};

// The columns of a lane that starts with column c: kVec of them from `at` on, the
// first `skip` of which belong to the lane before it, at the end of a row.  So all
// loads are whole and without branches (a load within a branch is waited for
// before the branch ends).  kNarrow: a row has fewer than kVec, `n` of which count.
template <bool kNarrow>
struct Span {
  uint32_t at, skip, n;
  __device__ __forceinline__ Span(uint32_t c, uint32_t cols) {
    at = kNarrow ? 0 : c + kVec <= cols ? c : cols - kVec;
    skip = kNarrow ? 0 : c - at;
    n = kNarrow ? cols : kVec;
  }
};

template <bool kF32, bool kNarrow>
__device__ __forceinline__ Cols load_cols(const void* p, const Span<kNarrow>& s) {
  Cols v;
  if constexpr (kNarrow) {
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) {
      const uint32_t i = j < s.n ? j : s.n - 1;
      v.x[j] = kF32 ? static_cast<const float*>(p)[i] : as_f(uint32_t(static_cast<const uint16_t*>(p)[i]) << 16);
    }
  } else if constexpr (kF32) {
    const u32x4_at4* const q = reinterpret_cast<const u32x4_at4*>(static_cast<const float*>(p) + s.at);
    const u32x4 lo = q[0], hi = q[1];
#pragma unroll
    for (uint32_t j = 0; j < 4; j++) {
      v.x[j] = as_f(lo[j]);
      v.x[4 + j] = as_f(hi[j]);
    }
  } else {
    const u32x4 h = *reinterpret_cast<const u32x4_at2*>(static_cast<const uint16_t*>(p) + s.at);
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] = as_f(j % 2 ? h[j / 2] & 0xFFFF0000u : h[j / 2] << 16);
  }
  return v;
}

// The lane's own columns.
template <bool kF32, bool kNarrow>
__device__ __forceinline__ void store_cols(void* p, const Cols& v, const Span<kNarrow>& s) {
  const bool whole = !kNarrow && s.skip == 0;
  if constexpr (kF32) {
    float* const q = static_cast<float*>(p) + s.at;
    if (whole) {
      u32x4_at4* const w = reinterpret_cast<u32x4_at4*>(q);
      w[0] = u32x4{as_u(v.x[0]), as_u(v.x[1]), as_u(v.x[2]), as_u(v.x[3])};
      w[1] = u32x4{as_u(v.x[4]), as_u(v.x[5]), as_u(v.x[6]), as_u(v.x[7])};
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++)
      if (j >= s.skip && j < s.n) q[j] = v.x[j];
  } else {
    const u32x2 lo = to_bf16(f32x4{v.x[0], v.x[1], v.x[2], v.x[3]}), hi = to_bf16(f32x4{v.x[4], v.x[5], v.x[6], v.x[7]});
    const u32x4 w = {lo.x, lo.y, hi.x, hi.y};
    uint16_t* const q = static_cast<uint16_t*>(p) + s.at;
    if (whole) {
      *reinterpret_cast<u32x4_at2*>(q) = w;
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++)
      if (j >= s.skip && j < s.n) q[j] = uint16_t(w[j / 2] >> (16 * (j & 1)));
  }
}

// Token t's row, or `rows` and more if it has none.
__device__ __forceinline__ uint64_t row_at(const EmbedArgs& a, uint64_t t) {
  const int64_t id = a.id_bytes == 4 ? int64_t(static_cast<const int32_t*>(a.ids)[t]) : static_cast<const int64_t*>(a.ids)[t];
  return uint64_t(id) - a.first;
}

// ------------------------------------------------------------------- lookup

template <bool kTable32, bool kOut32, bool kNarrow>
__global__ __launch_bounds__(256) void k_embed_lookup(EmbedArgs a, Units units) {
  const uint32_t unit = units.unit(), t = unit / units.slices;
  const uint32_t c = (((unit - t * units.slices) << units.lanes_log) + units.lane()) * kVec;
  if (t >= a.n || c >= a.cols) return;
  const uint64_t row = row_at(a, t);
  const Span<kNarrow> s(c, a.cols);
  Cols v = {};
  if (row < a.rows) {
    v = load_cols<kTable32>(static_cast<const uint8_t*>(a.table) + row * a.cols * (kTable32 ? 4 : 2), s);
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] *= a.scale;
  }
  store_cols<kOut32>(static_cast<uint8_t*>(a.out) + uint64_t(t) * a.stride * (kOut32 ? 4 : 2), v, s);
}

// ----------------------------------------------------------------- gradient

// Tokens in the order of their rows, rows in the order of (row mod 2^log, row).
// Workgroup g owns the rows that are g mod 2^log, so that those of the frequent
// tokens, which vocabularies often have side by side, are spread.  kAhead ids of
// a lane are in flight at a time.
constexpr uint32_t kAhead = 16;

__global__ __launch_bounds__(64 * kEmbedWaves) void k_embed_order(EmbedArgs a, uint32_t log, uint32_t R, uint32_t bits) {
  __shared__ uint32_t count[kEmbedWaves * kEmbedRows];  // tokens, then the next place, by wave and row
  __shared__ uint32_t wave_rows[kEmbedRows / 64], below_of[kEmbedWaves];
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, group = blockIdx.x, mask = (1u << log) - 1;
  const uint32_t n = uint32_t(a.n), share = (n + 64 * kEmbedWaves - 1) / (64 * kEmbedWaves) * 64;
  const uint32_t from = wave * share < n ? wave * share : n, to = from + share < n ? from + share : n;
  for (uint32_t i = threadIdx.x; i < kEmbedWaves * R; i += 64 * kEmbedWaves) count[i] = 0;
  __syncthreads();
  constexpr uint32_t kNoRow = ~0u;
  const auto load_as = [&](auto* ids, uint32_t t0, uint32_t (&row)[kAhead]) {
    int64_t id[kAhead];
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      const uint32_t t = t0 + 64 * k + lane;
      id[k] = ids[t < to ? t : to - 1];
    }
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      const uint64_t x = uint64_t(id[k]) - a.first;
      row[k] = t0 + 64 * k + lane < to && x < a.rows ? uint32_t(x) : kNoRow;
    }
  };
  const auto load = [&](uint32_t t0, uint32_t (&row)[kAhead]) {
    if (a.id_bytes == 4) load_as(static_cast<const int32_t*>(a.ids), t0, row);
    else load_as(static_cast<const int64_t*>(a.ids), t0, row);
  };
  uint32_t row[kAhead];  // the last ones loaded: few tokens are loaded once
  const bool once = share <= 64 * kAhead;
  uint32_t below = 0;
  for (uint32_t t0 = from; t0 < to; t0 += 64 * kAhead) {
    load(t0, row);
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      below += row[k] != kNoRow && (row[k] & mask) < group;
      if (row[k] != kNoRow && (row[k] & mask) == group) atomicAdd(&count[wave * R + (row[k] >> log)], 1u);
    }
  }
  for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  // each row's tokens, and the sum of those of the rows before it
  uint32_t own = 0;
  if (threadIdx.x < R)
    for (uint32_t w = 0; w < kEmbedWaves; w++) own += count[w * R + threadIdx.x];
  uint32_t sum = own;
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t x = __shfl_up(sum, d);
    sum += int(lane) >= d ? x : 0;
  }
  if (lane == 63 && wave < kEmbedRows / 64) wave_rows[wave] = sum;
  __syncthreads();
  if (threadIdx.x < R) {
    const uint32_t row = threadIdx.x << log | group;
    uint32_t at = sum - own;
    for (uint32_t w = 0; w < wave; w++) at += wave_rows[w];
    for (uint32_t w = 0; w < kEmbedWaves; w++) at += below_of[w];
    if (row < a.rows) a.places[row] = Places{at, own};
    if (group == mask && threadIdx.x == R - 1) a.places[a.rows] = Places{at + own, 0};  // all
    for (uint32_t w = 0; w < kEmbedWaves; w++) {
      const uint32_t c = count[w * R + threadIdx.x];
      count[w * R + threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t t0 = from; t0 < to; t0 += 64 * kAhead) {
    if (!once) load(t0, row);
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      if (t0 + 64 * k >= to) break;
      const bool here = row[k] != kNoRow && (row[k] & mask) == group;
      const u64 any = __ballot(here);
      if (!any) continue;
      // the lanes whose tokens have this lane's row, by the bits of its number
      const uint32_t in = row[k] >> log;
      u64 same = any;
      for (uint32_t b = 0; b < bits; b++) {
        const u64 set = __ballot(in >> b & 1);
        same &= in >> b & 1 ? set : ~set;
      }
      // the first of them takes places for all, in order
      const uint32_t first = here ? uint32_t(__builtin_ctzll(same)) : lane;
      uint32_t at = 0;
      if (here && lane == first) at = atomicAdd(&count[wave * R + in], uint32_t(__builtin_popcountll(same)));
      at = __shfl(at, int(first));
      if (here) {
        const uint32_t place = at + uint32_t(__builtin_popcountll(same & ((u64(1) << lane) - 1)));
        a.order[place] = t0 + 64 * k + lane;
        a.row_of[place] = row[k];
      }
    }
  }
}

// Where the sum of the run that starts at place p of a row that starts at s is
// kept.  Of rows with more than kRun tokens one at most starts within kRun places,
// and one at most has a later run that starts there.
__device__ __forceinline__ uint64_t run_slot(uint32_t p, uint32_t s) { return uint64_t(p / kRun) * 2 + (p == s); }

// The sums of `n` <= kRun tokens from place p on, of U slices' columns.  kFlight
// tokens' rows are in flight at a time; past the end the last one again, not
// counted.
template <bool kF32, uint32_t U, uint32_t kFlight, bool kNarrow>
__device__ __forceinline__ void sum_run(const EmbedArgs& a, uint32_t p, uint32_t n, const Span<kNarrow> (&span)[U],
                                        Cols (&s)[U]) {
#pragma unroll
  for (uint32_t u = 0; u < U; u++) s[u] = Cols{};
  for (uint32_t i = 0; i < n; i += kFlight) {
    uint32_t t[kFlight];
#pragma unroll
    for (uint32_t k = 0; k < kFlight; k++) t[k] = a.order[p + (i + k < n ? i + k : n - 1)];
    Cols v[kFlight][U];
#pragma unroll
    for (uint32_t k = 0; k < kFlight; k++)
#pragma unroll
      for (uint32_t u = 0; u < U; u++)
        v[k][u] = load_cols<kF32>(static_cast<const uint8_t*>(a.dout) + uint64_t(t[k]) * a.stride * (kF32 ? 4 : 2),
                                  span[u]);
#pragma unroll
    for (uint32_t k = 0; k < kFlight; k++)
#pragma unroll
      for (uint32_t u = 0; u < U; u++)
#pragma unroll
        for (uint32_t j = 0; j < kVec; j++) s[u].x[j] = i + k < n ? s[u].x[j] + v[k][u].x[j] : s[u].x[j];
  }
}

// A row's gradient from its sum, in a span's columns.
template <bool kGrad32, bool kNarrow>
__device__ __forceinline__ void write_row(const EmbedArgs& a, uint32_t row, Cols v, const Span<kNarrow>& s) {
  uint8_t* const out = static_cast<uint8_t*>(a.grad) + uint64_t(row) * a.cols * (kGrad32 ? 4 : 2);
#pragma unroll
  for (uint32_t j = 0; j < kVec; j++) v.x[j] *= a.scale;
  if (a.add) {
    // (of columns that another lane may have written already, only what it does
    // not own: those are not stored)
    const Cols old = load_cols<kGrad32>(out, s);
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] = old.x[j] + v.x[j];
  }
  store_cols<kGrad32>(out, v, s);
}

// The row that starts among places b ... b + kRun - 1 and has more than kRun
// tokens, or `rows`.
__device__ __forceinline__ uint32_t long_row_at(const EmbedArgs& a, uint32_t b, uint32_t all) {
  if (b + kRun - 1 >= all) return a.rows;
  const uint32_t row = a.row_of[b + kRun - 1];
  const Places p = a.places[row];
  return p.first < b || p.n <= kRun ? a.rows : row;
}

// The first `run_units` units: sums of runs of long rows, by their places.  The
// others: the rows of up to kRun tokens, U slices a unit.
template <bool kF32, bool kGrad32, uint32_t U, bool kNarrow>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a, Units units, uint32_t run_units, uint32_t row_slices,
                                                    uint32_t all_units) {
  const uint32_t unit = units.unit();
  if (unit >= all_units) return;
  if (unit < run_units) {
    const uint32_t which = unit / units.slices;
    const uint32_t c = (((unit - which * units.slices) << units.lanes_log) + units.lane()) * kVec;
    const uint32_t all = a.places[a.rows].first, b = which / 2 * kRun;
    if (c >= a.cols || b >= all) return;
    uint32_t row = which & 1 ? long_row_at(a, b, all) : a.row_of[b];  // its first run, or of the row that holds b
    if (row == a.rows) return;
    const Places x = a.places[row];
    uint32_t p = x.first;
    if (!(which & 1)) {  // a later one
      if (x.first >= b || x.n <= kRun) return;
      p = b + x.first % kRun;
      if (p >= x.first + x.n) return;
    }
    const uint32_t left = x.first + x.n - p;
    const Span<kNarrow> span[1] = {{c, a.cols}};
    Cols s[1];
    sum_run<kF32, 1, 16>(a, p, left < kRun ? left : kRun, span, s);
    store_cols<true>(a.runs + uint64_t(which) * a.cols, s[0], span[0]);
  } else {
    const uint32_t k = unit - run_units, row = k / row_slices, step = kVec << units.lanes_log;
    const uint32_t c = (k - row * row_slices) * U * step + units.lane() * kVec;
    if (c >= a.cols) return;
    const Places x = a.places[row];
    if (x.n > kRun || (x.n == 0 && a.add)) return;
    // (a slice behind the row's end is the first one again, and not stored)
    const auto column = [&](uint32_t u) { return c + u * step < a.cols ? c + u * step : c; };
    Cols s[U];
    if constexpr (U == 1) {
      const Span<kNarrow> span[1] = {{c, a.cols}};
      sum_run<kF32, 1, 8>(a, x.first, x.n, span, s);
      write_row<kGrad32>(a, row, s[0], span[0]);
    } else {
      const Span<kNarrow> span[2] = {{c, a.cols}, {column(1), a.cols}};
      sum_run<kF32, 2, 4>(a, x.first, x.n, span, s);
      write_row<kGrad32>(a, row, s[0], span[0]);
      if (c + step < a.cols) write_row<kGrad32>(a, row, s[1], span[1]);
    }
  }
}

// The long rows, from the sums of their runs.
template <bool kGrad32, bool kNarrow>
__global__ __launch_bounds__(256) void k_embed_long(EmbedArgs a, Units units, uint32_t all_units) {
  const uint32_t unit = units.unit();
  if (unit >= all_units) return;
  const uint32_t which = unit / units.slices;
  const uint32_t c = (((unit - which * units.slices) << units.lanes_log) + units.lane()) * kVec;
  const uint32_t all = a.places[a.rows].first, b = which * kRun;
  if (c >= a.cols || b >= all) return;
  const uint32_t row = long_row_at(a, b, all);
  if (row == a.rows) return;
  constexpr uint32_t kFlight = 8;
  const Span<kNarrow> span(c, a.cols);
  const uint32_t s = a.places[row].first, runs = (a.places[row].n + kRun - 1) / kRun;
  Cols v = {};
  for (uint32_t g = 0; g < runs; g += kRun) {
    const uint32_t n = runs - g < kRun ? runs - g : kRun;
    Cols sum = {};
    for (uint32_t i = 0; i < n; i += kFlight) {
      Cols x[kFlight];
#pragma unroll
      for (uint32_t k = 0; k < kFlight; k++) {
        const uint32_t r = g + (i + k < n ? i + k : n - 1);
        x[k] = load_cols<true>(a.runs + run_slot(s + r * kRun, s) * a.cols, span);
      }
#pragma unroll
      for (uint32_t k = 0; k < kFlight; k++)
#pragma unroll
        for (uint32_t j = 0; j < kVec; j++) sum.x[j] = i + k < n ? sum.x[j] + x[k].x[j] : sum.x[j];
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] += sum.x[j];
  }
  write_row<kGrad32>(a, row, v, span);
}

// Above so many slices of rows, some four times the waves that the card holds, a unit
// of k_embed_rows takes two.  Two and one, us: 16,384 tokens, 16,032 rows of 1,024
// columns (32,064 slices) 40 and 37, of 1,536 41 and 43, of 2,048 44 and 48, of 4,096
// 67 and 75, 128,256 rows of 1,024 87 and 104; 4,096 tokens, 8,192 rows of 2,048
// (32,768) 30 and 26, of 4,096 both 34; 65,536 tokens, 2,000 rows of 2,048 (8,000)
// 119 and 111.
constexpr uint32_t kTwoSlices = 32768;

// Units of up to 64 lanes: one for up to 512 columns.
Units units_of(uint32_t cols) {
  Units u;
  u.lanes_log = 0;
  while (u.lanes_log < 6 && (kVec << u.lanes_log) < cols) u.lanes_log++;
  u.slices = (cols + (kVec << u.lanes_log) - 1) / (kVec << u.lanes_log);
  return u;
}
uint32_t blocks_of(uint64_t units, const Units& u) { return uint32_t(((units << u.lanes_log) + 255) / 256); }

}  // namespace

int launch_embed_lookup(const EmbedArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (!a.n) return 0;
  const Units u = units_of(a.cols);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks_of(a.n * u.slices, u)), dim3(256), 0, st, a, u);
  };
  const auto by_width = [&](auto wide, auto narrow) { a.cols < kVec ? launch(narrow) : launch(wide); };
  if (a.table_f32 && a.act_f32) by_width(k_embed_lookup<true, true, false>, k_embed_lookup<true, true, true>);
  else if (a.table_f32) by_width(k_embed_lookup<true, false, false>, k_embed_lookup<true, false, true>);
  else if (a.act_f32) by_width(k_embed_lookup<false, true, false>, k_embed_lookup<false, true, true>);
  else by_width(k_embed_lookup<false, false, false>, k_embed_lookup<false, false, true>);
  return int(hipGetLastError());
}

int launch_embed_grad(const EmbedArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (!a.n && a.add) return 0;
  uint32_t log = kEmbedGroupsLog, bits = 0;
  while ((a.rows >> log) + 1 > kEmbedRows) log++;
  const uint32_t R = (a.rows + (1u << log) - 1) >> log;
  while ((1u << bits) < R) bits++;
  hipLaunchKernelGGL(k_embed_order, dim3(1u << log), dim3(64 * kEmbedWaves), 0, st, a, log, R, bits);
  if (const int e = int(hipGetLastError())) return e;
  const Units u = units_of(a.cols);
  const uint32_t U = u.slices > 1 && uint64_t(a.rows) * u.slices > kTwoSlices ? 2 : 1, row_slices = (u.slices + U - 1) / U;
  const uint32_t runs = a.n > kRun ? uint32_t(embed_run_slots(a.n) * u.slices) : 0, all = runs + a.rows * row_slices;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks_of(all, u)), dim3(256), 0, st, a, u, runs, row_slices, all);
  };
  const auto by_width = [&](auto two, auto one, auto narrow) {
    a.cols < kVec ? launch(narrow) : U == 1 ? launch(one) : launch(two);
  };
#define FR_ROWS(f, g) k_embed_rows<f, g, 2, false>, k_embed_rows<f, g, 1, false>, k_embed_rows<f, g, 1, true>
  if (a.act_f32 && a.grad_f32) by_width(FR_ROWS(true, true));
  else if (a.act_f32) by_width(FR_ROWS(true, false));
  else if (a.grad_f32) by_width(FR_ROWS(false, true));
  else by_width(FR_ROWS(false, false));
#undef FR_ROWS
  if (const int e = int(hipGetLastError())) return e;
  if (!runs) return 0;
  const uint32_t places = runs / 2;  // of long rows' starts
  const auto launch_long = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks_of(places, u)), dim3(256), 0, st, a, u, places);
  };
  const bool narrow = a.cols < kVec;
  if (a.grad_f32) narrow ? launch_long(k_embed_long<true, true>) : launch_long(k_embed_long<true, false>);
  else narrow ? launch_long(k_embed_long<false, true>) : launch_long(k_embed_long<false, false>);
  return int(hipGetLastError());
}

}  // namespace fr
