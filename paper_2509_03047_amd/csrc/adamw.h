// Internal declarations shared by the host and device sources of the
// optimizer step.
#pragma once

#include <cstdint>
#include <vector>

#include "flashrestore.h"

namespace fr {

// The arrays of a tensor.
enum AdamwKind : uint32_t { kParam, kMaster, kMom1, kMom2, kScale1, kScale2, kKinds };
constexpr uint32_t kSummed = kMom2 + 1;  // the first ones, which a step sums as it writes them

// One tensor, as the kernels read it (uniform loads).  Offsets from the state
// arena's base, `grad` from the gradients'.
struct alignas(16) AdamwRec {
  uint64_t numel;
  uint64_t counter;       // of its first element
  uint64_t grad;
  uint64_t at[kKinds];    // kNone: it has no such array
  uint32_t grad_f32;
  uint32_t group;
  uint64_t pad_;
};
static_assert(sizeof(AdamwRec) == 96, "AdamwRec is 96 bytes");
constexpr uint64_t kNone = ~uint64_t(0);

// Which tile of which tensor each workgroup of a launch takes: n slots
// (tensor << 32) | tile in order, stored XCD-major (slot g at
// (g mod 8) * stride + g / 8).
struct AdamwWalk {
  const uint64_t* d = nullptr;
  uint64_t n = 0, stride = 0;
};

// A chunk's sum: `n` consecutive slots of a walk from `slot` on, each of which
// left its part of the array `kind`.
struct alignas(16) AdamwFold {
  uint32_t chunk, slot, n, kind;
};
// A chunk of scales, which is summed from the state itself once the step has
// written it: a wave's two scales would take as much to leave and fold as their
// whole chunk to read, and a chunk of C bytes is fed by C / 8 waves.
struct alignas(16) AdamwScales {
  uint64_t at;  // in the state
  uint32_t words, chunk;
};

// What the kernels of one call need of its optimizer.
struct AdamwStepArgs {
  const AdamwRec* recs = nullptr;
  AdamwWalk walk;
  bool eight = false;      // of the tensors with 8-bit moments
  void* state = nullptr;
  const void* grads = nullptr;
  const fr_adamw_hyper* hyper = nullptr;
  const fr_grad_stats* stats = nullptr;
  // sums, or parts == NULL
  uint64_t C = 0;
  fr_chunk_sum* parts = nullptr;  // kSummed arrays of 8 * walk.stride places
  const AdamwFold* folds = nullptr;
  const AdamwScales* scales = nullptr;
  uint32_t n_folds = 0, n_scales = 0;
  fr_chunk_sum* sums = nullptr;
};

struct AdamwNormArgs {
  const AdamwRec* recs = nullptr;
  AdamwWalk walk;
  const void* grads = nullptr;
  float max_norm = 0;
  fr_grad_stats* stats = nullptr;
  double* parts = nullptr;     // a sum for each place of the walk, and kNormFold
  uint32_t* arrived = nullptr; // lines, zero between calls
};

struct AdamwConvertArgs {
  const AdamwRec* from_recs = nullptr;
  const AdamwRec* to_recs = nullptr;
  AdamwWalk walk;
  bool eight = false;  // the tensors of `to` in the walk have 8-bit moments
  const void* from = nullptr;
  void* to = nullptr;
  uint32_t seed = 0;
};

// How a kernel takes its work: workgroups of B threads with U groups of four
// elements each, the LDS a launch asks for to bound how many of them a compute
// unit holds (adamw.hip says why, and what a step's measured), and how many
// consecutive tiles one die takes.  A compute unit gives its 160 KB out in blocks
// of 1,280 bytes, so that a request for 14,800 of them leaves room for 10
// workgroups (so many of them sleep side by side; the runtime's occupancy query
// does not round up, and says 11).
struct AdamwShape {
  uint32_t B, U, lds, run;
  constexpr uint32_t tile() const { return B * U * 4; }
};
// Times are of an 8B model's share, 1.0e9 elements, in three allocations.
// By form, 32 bits and 8: 10 and 21 waves a compute unit.  (8 bits, U = 2: 12 waves
// 2.68-2.72 ms, 16 2.59-2.64, 21 2.62-2.69, no bound 2.66-2.72; U = 1: 21 2.64-2.66, 25
// 2.58-2.69; U = 4: 11 2.61-2.71.  One tile a run 2.55-2.76, two 2.62-2.69, four
// 2.67-2.69, eight 2.66-2.89, when the dies' windows drift apart; in 32 bits one
// 4.32-4.48, two 4.40-4.49.)
constexpr AdamwShape kStepShape[2] = {{64, 1, 14800, 1}, {64, 2, 6800, 2}};
// Steps that also sum: one wave, which folds its own sums; 16 and, as many as their
// registers allow, 24 waves.  (32 bits: 12 waves 4.78-4.85 ms, 14 4.61-4.66, 16
// 4.53-4.61, 21 4.57-4.69; U = 2: 10 waves 4.51-4.66, 12 4.48-4.72.  8 bits: U = 1
// 2.91-2.93; U = 2: 16 waves 3.03-3.07, 21 2.82-2.85, no bound 2.76-2.78, where the step
// and a checksum of the state take 3.8.)
constexpr AdamwShape kSumShape[2] = {{64, 1, 10200, 1}, {64, 2, 0, 1}};
// By the form written: 11 workgroups of two waves and 1,024 elements.  (To 8 bits:
// 64 x 2, 21 a compute unit 1.60-1.61 ms, 128 x 2, 11 1.59-1.61.  To 32: 64 x 2, 21
// 1.64-1.67, 12 1.59-1.61, 128 x 2, 11 1.63-1.68, 64 x 8, 5 1.59-1.64, but of 2,000 ragged
// tensors 69 us where the smaller tiles take 61.  One tile a run instead of two:
// to 8 bits 1.59-1.61, to 32 1.63-1.71.)
constexpr AdamwShape kConvertShape[2] = {{128, 2, 13500, 2}, {128, 2, 13500, 2}};
constexpr uint32_t kNormBytes = 16384;  // of gradients a workgroup of a norm takes (8 KiB: 374 us instead of 304)
// A norm of more workgroups than kNormOne adds up their sums by a second launch
// of kNormFold workgroups; these, or those of a smaller norm, arrive at lines of
// kNormPerLine each, whose last ones arrive at line 0 (up to kNormOneLine at line
// 0 themselves: arrivals at one line take 7 ns each, another line a round trip).
constexpr uint32_t kNormOne = 1024, kNormFold = 64, kNormPerLine = 32, kNormOneLine = 64, kNormLine = 128;
constexpr uint32_t kNormArriveBytes = (1 + kNormOne / kNormPerLine) * kNormLine;
static_assert(kSumShape[0].B == 64 && kSumShape[1].B == 64, "one wave");
static_assert(kSumShape[0].tile() * 4 <= FR_ADAMW_MIN_SUM_CHUNK && kSumShape[1].tile() * 4 <= FR_ADAMW_MIN_SUM_CHUNK,
              "a summed tile lies inside a chunk");

// Kernel launchers (adamw.hip): validated arguments, enqueue on `stream`,
// return the hipError_t as an int.
int launch_adamw_step(const AdamwStepArgs& a, void* stream);
int launch_adamw_norm(const AdamwNormArgs& a, void* stream);
int launch_adamw_scale(float max_norm, fr_grad_stats* stats, void* stream);
int launch_adamw_convert(const AdamwConvertArgs& a, void* stream);

}  // namespace fr
