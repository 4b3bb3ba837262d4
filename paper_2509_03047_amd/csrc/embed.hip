// gfx950 kernels of the embedding: rows of the state for a batch of tokens, and
// the gradient that they leave.
//
// The gradient's tokens are brought into the order of their rows by one launch:
// each workgroup owns some hundred rows at most, reads all ids (they stay in L2)
// and so counts the tokens of the rows in front of its own as well as its own's,
// by wave; a second pass puts each token at its place.  Its waves have
// consecutive tokens, so the order within a row is the tokens' own, and nothing
// depends on atomics' order.  A row of more than FR_EMBED_RUN tokens is cut into
// runs, which a launch of their own sums up; the last launch writes the rows.
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

// Eight elements from any element's address on (the compiler's own choice of
// loads for what alignment there is).
struct __attribute__((packed, aligned(2))) Half8 {
  uint16_t x[8];
};
struct __attribute__((packed, aligned(4))) Float8 {
  float x[8];
};

struct Cols {
  float x[kVec];
};

// Columns c ... c + 7 of a row of `cols` at p, zeros behind its end.
template <bool kF32>
__device__ __forceinline__ Cols load_cols(const void* p, uint32_t c, uint32_t cols) {
  Cols v;
  if (c + kVec <= cols) {
    if constexpr (kF32) {
      const Float8 f = *reinterpret_cast<const Float8*>(static_cast<const float*>(p) + c);
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) v.x[j] = f.x[j];
    } else {
      const Half8 h = *reinterpret_cast<const Half8*>(static_cast<const uint16_t*>(p) + c);
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) v.x[j] = as_f(uint32_t(h.x[j]) << 16);
    }
    return v;
  }
#pragma unroll
  for (uint32_t j = 0; j < kVec; j++) {
    v.x[j] = 0.0f;
    if (c + j < cols)
      v.x[j] = kF32 ? static_cast<const float*>(p)[c + j]
                    : as_f(uint32_t(static_cast<const uint16_t*>(p)[c + j]) << 16);
  }
  return v;
}

template <bool kF32>
__device__ __forceinline__ void store_cols(void* p, const Cols& v, uint32_t c, uint32_t cols) {
  if constexpr (kF32) {
    float* const q = static_cast<float*>(p) + c;
    if (c + kVec <= cols) {
      Float8 f;
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) f.x[j] = v.x[j];
      *reinterpret_cast<Float8*>(q) = f;
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++)
      if (c + j < cols) q[j] = v.x[j];
  } else {
    const u32x2 lo = to_bf16(f32x4{v.x[0], v.x[1], v.x[2], v.x[3]}), hi = to_bf16(f32x4{v.x[4], v.x[5], v.x[6], v.x[7]});
    const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
    uint16_t* const q = static_cast<uint16_t*>(p) + c;
    Half8 h;
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) h.x[j] = uint16_t(w[j / 2] >> (16 * (j & 1)));
    if (c + kVec <= cols) {
      *reinterpret_cast<Half8*>(q) = h;
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++)
      if (c + j < cols) q[j] = h.x[j];
  }
}

// Token t's row, or `rows` and more if it has none.
__device__ __forceinline__ uint64_t row_at(const EmbedArgs& a, uint64_t t) {
  const int64_t id = a.id_bytes == 4 ? int64_t(static_cast<const int32_t*>(a.ids)[t]) : static_cast<const int64_t*>(a.ids)[t];
  return uint64_t(id) - a.first;
}

// ------------------------------------------------------------------- lookup

// A unit takes U slices of a token's row, whose loads are in flight together.
template <bool kTable32, bool kOut32, uint32_t U>
__global__ __launch_bounds__(256) void k_embed_lookup(EmbedArgs a, Units units) {
  const uint32_t unit = units.unit(), t = unit / units.slices;
  if (t >= a.n) return;
  const uint32_t c0 = ((unit - t * units.slices) * U << units.lanes_log) + units.lane();
  const uint64_t row = row_at(a, t);
  Cols v[U] = {};
  if (row < a.rows) {
#pragma unroll
    for (uint32_t u = 0; u < U; u++) {
      const uint32_t c = (c0 + (u << units.lanes_log)) * kVec;
      if (c < a.cols)
        v[u] = load_cols<kTable32>(static_cast<const uint8_t*>(a.table) + row * a.cols * (kTable32 ? 4 : 2), c, a.cols);
    }
  }
#pragma unroll
  for (uint32_t u = 0; u < U; u++) {
    const uint32_t c = (c0 + (u << units.lanes_log)) * kVec;
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v[u].x[j] = row < a.rows ? v[u].x[j] * a.scale : 0.0f;
    if (c < a.cols)
      store_cols<kOut32>(static_cast<uint8_t*>(a.out) + uint64_t(t) * a.stride * (kOut32 ? 4 : 2), v[u], c, a.cols);
  }
}

// ----------------------------------------------------------------- gradient

// Tokens in the order of their rows.  Workgroup g owns rows [g R, (g + 1) R).
// kAhead ids of a lane are in flight at a time.
constexpr uint32_t kAhead = 8;

__global__ __launch_bounds__(64 * kEmbedWaves) void k_embed_order(EmbedArgs a, uint32_t R, uint32_t bits) {
  __shared__ uint32_t count[kEmbedWaves * kEmbedRows];  // tokens, then the next place, by wave and row
  __shared__ uint32_t wave_rows[kEmbedRows / 64], below_of[kEmbedWaves];
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const uint32_t r0 = blockIdx.x * R, mine = a.rows - r0 < R ? a.rows - r0 : R;
  const uint32_t n = uint32_t(a.n), share = (n + 64 * kEmbedWaves - 1) / (64 * kEmbedWaves) * 64;
  const uint32_t from = wave * share < n ? wave * share : n, to = from + share < n ? from + share : n;
  for (uint32_t i = threadIdx.x; i < kEmbedWaves * R; i += 64 * kEmbedWaves) count[i] = 0;
  __syncthreads();
  // rows that are not there count as behind all
  const auto load = [&](uint32_t t0, uint64_t (&row)[kAhead]) {
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      const uint32_t t = t0 + 64 * k + lane;
      row[k] = t < to ? row_at(a, t) : ~uint64_t(0);
    }
  };
  uint32_t below = 0;
  for (uint32_t t0 = from; t0 < to; t0 += 64 * kAhead) {
    uint64_t row[kAhead];
    load(t0, row);
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      below += row[k] < r0;
      if (row[k] - r0 < mine) atomicAdd(&count[wave * R + uint32_t(row[k] - r0)], 1u);
    }
  }
  for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  // each row's tokens, and the sum of those of the rows before it
  uint32_t own = 0;
  if (threadIdx.x < mine)
    for (uint32_t w = 0; w < kEmbedWaves; w++) own += count[w * R + threadIdx.x];
  uint32_t sum = own;
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t x = __shfl_up(sum, d);
    sum += int(lane) >= d ? x : 0;
  }
  if (lane == 63 && wave < kEmbedRows / 64) wave_rows[wave] = sum;
  __syncthreads();
  if (threadIdx.x < mine) {
    uint32_t at = sum - own;
    for (uint32_t w = 0; w < wave; w++) at += wave_rows[w];
    for (uint32_t w = 0; w < kEmbedWaves; w++) at += below_of[w];
    a.start[r0 + threadIdx.x] = at;
    if (r0 + threadIdx.x + 1 == a.rows) a.start[a.rows] = at + own;
    for (uint32_t w = 0; w < kEmbedWaves; w++) {
      const uint32_t c = count[w * R + threadIdx.x];
      count[w * R + threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t t0 = from; t0 < to; t0 += 64 * kAhead) {
    uint64_t row[kAhead];
    load(t0, row);
#pragma unroll
    for (uint32_t k = 0; k < kAhead; k++) {
      const bool here = row[k] - r0 < mine;
      const u64 any = __ballot(here);
      if (!any) continue;
      // the lanes whose tokens have this lane's row, by the bits of its number
      const uint32_t in = uint32_t(row[k] - r0);
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
        a.row_of[place] = r0 + in;
      }
    }
  }
}

// Where the sum of the run that starts at place p of a row that starts at s is
// kept.  Of rows with more than kRun tokens one at most starts within kRun places,
// and one at most has a later run that starts there.
__device__ __forceinline__ uint64_t run_slot(uint32_t p, uint32_t s) { return uint64_t(p / kRun) * 2 + (p == s); }

// The sum of `n` <= kRun tokens from place p on.  kFlight rows are in flight at a
// time; past the end the last one again, not counted.
constexpr uint32_t kFlight = 8;

template <bool kF32>
__device__ __forceinline__ Cols sum_run(const EmbedArgs& a, uint32_t p, uint32_t n, uint32_t c) {
  Cols s = {};
  for (uint32_t i = 0; i < n; i += kFlight) {
    uint32_t t[kFlight];
#pragma unroll
    for (uint32_t k = 0; k < kFlight; k++) t[k] = a.order[p + (i + k < n ? i + k : n - 1)];
    Cols v[kFlight];
#pragma unroll
    for (uint32_t k = 0; k < kFlight; k++)
      v[k] = load_cols<kF32>(static_cast<const uint8_t*>(a.dout) + uint64_t(t[k]) * a.stride * (kF32 ? 4 : 2), c, a.cols);
#pragma unroll
    for (uint32_t k = 0; k < kFlight; k++)
      if (i + k < n)
#pragma unroll
        for (uint32_t j = 0; j < kVec; j++) s.x[j] += v[k].x[j];
  }
  return s;
}

// Columns c ... of a row's gradient.
template <bool kGrad32>
__device__ __forceinline__ void write_row(const EmbedArgs& a, uint32_t row, Cols v, uint32_t c) {
  uint8_t* const out = static_cast<uint8_t*>(a.grad) + uint64_t(row) * a.cols * (kGrad32 ? 4 : 2);
#pragma unroll
  for (uint32_t j = 0; j < kVec; j++) v.x[j] *= a.scale;
  if (a.add) {
    const Cols old = load_cols<kGrad32>(out, c, a.cols);
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] = old.x[j] + v.x[j];
  }
  store_cols<kGrad32>(out, v, c, a.cols);
}

// The row that starts among places b ... b + kRun - 1 and has more than kRun
// tokens, or `rows`.
__device__ __forceinline__ uint32_t long_row_at(const EmbedArgs& a, uint32_t b, uint32_t all) {
  if (b + kRun - 1 >= all) return a.rows;
  const uint32_t row = a.row_of[b + kRun - 1], s = a.start[row];
  return s < b || a.start[row + 1] - s <= kRun ? a.rows : row;
}

// The first `run_units` units: sums of runs of long rows, by their places.  The
// others: the rows of up to kRun tokens.
template <bool kF32, bool kGrad32>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a, Units units, uint32_t run_units, uint32_t all_units) {
  const uint32_t unit = units.unit();
  if (unit >= all_units) return;
  const bool of_run = unit < run_units;
  const uint32_t k = of_run ? unit : unit - run_units, which = k / units.slices;
  const uint32_t c = ((k - which * units.slices << units.lanes_log) + units.lane()) * kVec;
  if (c >= a.cols) return;
  uint32_t p, n;
  if (of_run) {
    const uint32_t all = a.start[a.rows], b = which / 2 * kRun;
    if (b >= all) return;
    uint32_t row;
    if (which & 1) {  // its first one
      row = long_row_at(a, b, all);
      if (row == a.rows) return;
      p = a.start[row];
    } else {  // a later one, of the row that holds place b
      row = a.row_of[b];
      const uint32_t s = a.start[row];
      if (s >= b || a.start[row + 1] - s <= kRun) return;
      p = b + s % kRun;
    }
    const uint32_t e = a.start[row + 1];
    if (p >= e) return;
    n = e - p < kRun ? e - p : kRun;
  } else {
    p = a.start[which];
    n = a.start[which + 1] - p;
    if (n > kRun || (n == 0 && a.add)) return;
  }
  const Cols v = sum_run<kF32>(a, p, n, c);
  if (of_run) store_cols<true>(a.runs + uint64_t(which) * a.cols, v, c, a.cols);
  else write_row<kGrad32>(a, which, v, c);
}

// The long rows, from the sums of their runs.
template <bool kGrad32>
__global__ __launch_bounds__(256) void k_embed_long(EmbedArgs a, Units units, uint32_t all_units) {
  const uint32_t unit = units.unit();
  if (unit >= all_units) return;
  const uint32_t which = unit / units.slices;
  const uint32_t c = ((unit - which * units.slices << units.lanes_log) + units.lane()) * kVec;
  const uint32_t all = a.start[a.rows], b = which * kRun;
  if (c >= a.cols || b >= all) return;
  const uint32_t row = long_row_at(a, b, all);
  if (row == a.rows) return;
  const uint32_t s = a.start[row], runs = (a.start[row + 1] - s + kRun - 1) / kRun;
  Cols v = {};
  for (uint32_t g = 0; g < runs; g += kRun) {
    const uint32_t n = runs - g < kRun ? runs - g : kRun;
    Cols sum = {};
    for (uint32_t i = 0; i < n; i += kFlight) {
      Cols x[kFlight];
#pragma unroll
      for (uint32_t k = 0; k < kFlight; k++) {
        const uint32_t r = g + (i + k < n ? i + k : n - 1);
        x[k] = load_cols<true>(a.runs + run_slot(s + r * kRun, s) * a.cols, c, a.cols);
      }
#pragma unroll
      for (uint32_t k = 0; k < kFlight; k++)
        if (i + k < n)
#pragma unroll
          for (uint32_t j = 0; j < kVec; j++) sum.x[j] += x[k].x[j];
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] += sum.x[j];
  }
  write_row<kGrad32>(a, row, v, c);
}

// Units of up to 64 lanes: one for up to 512 columns.
Units units_of(uint32_t cols, uint32_t slices_each) {
  Units u;
  u.lanes_log = 0;
  while (u.lanes_log < 6 && (kVec << u.lanes_log) < cols) u.lanes_log++;
  const uint32_t columns = (kVec << u.lanes_log) * slices_each;
  u.slices = (cols + columns - 1) / columns;
  return u;
}
uint32_t blocks_of(uint64_t units, const Units& u) { return uint32_t(((units << u.lanes_log) + 255) / 256); }

}  // namespace

int launch_embed_lookup(const EmbedArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (!a.n) return 0;
  const auto launch = [&](auto kernel, uint32_t slices_each) {
    const Units u = units_of(a.cols, slices_each);
    hipLaunchKernelGGL(kernel, dim3(blocks_of(a.n * u.slices, u)), dim3(256), 0, st, a, u);
  };
  const bool many = a.cols > 512;
  if (a.table_f32 && a.act_f32) many ? launch(k_embed_lookup<true, true, 4>, 4) : launch(k_embed_lookup<true, true, 1>, 1);
  else if (a.table_f32) many ? launch(k_embed_lookup<true, false, 4>, 4) : launch(k_embed_lookup<true, false, 1>, 1);
  else if (a.act_f32) many ? launch(k_embed_lookup<false, true, 4>, 4) : launch(k_embed_lookup<false, true, 1>, 1);
  else many ? launch(k_embed_lookup<false, false, 4>, 4) : launch(k_embed_lookup<false, false, 1>, 1);
  return int(hipGetLastError());
}

int launch_embed_grad(const EmbedArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (!a.n && a.add) return 0;
  const uint32_t R = embed_group_rows(a.rows);
  uint32_t bits = 0;
  while ((1u << bits) < R) bits++;
  hipLaunchKernelGGL(k_embed_order, dim3((a.rows + R - 1) / R), dim3(64 * kEmbedWaves), 0, st, a, R, bits);
  if (const int e = int(hipGetLastError())) return e;
  const Units u = units_of(a.cols, 1);
  const uint32_t runs = a.n > kRun ? uint32_t(embed_run_slots(a.n) * u.slices) : 0, all = runs + a.rows * u.slices;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks_of(all, u)), dim3(256), 0, st, a, u, runs, all);
  };
  if (a.act_f32 && a.grad_f32) launch(k_embed_rows<true, true>);
  else if (a.act_f32) launch(k_embed_rows<true, false>);
  else if (a.grad_f32) launch(k_embed_rows<false, true>);
  else launch(k_embed_rows<false, false>);
  if (const int e = int(hipGetLastError())) return e;
  if (!runs) return 0;
  const uint32_t places = runs / 2;  // of long rows' starts
  if (a.grad_f32) hipLaunchKernelGGL(k_embed_long<true>, dim3(blocks_of(places, u)), dim3(256), 0, st, a, u, places);
  else hipLaunchKernelGGL(k_embed_long<false>, dim3(blocks_of(places, u)), dim3(256), 0, st, a, u, places);
  return int(hipGetLastError());
}

}  // namespace fr
