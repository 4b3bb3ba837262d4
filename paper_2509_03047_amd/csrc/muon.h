// Internal declarations shared by the host and device sources of the step by
// orthogonalised momentum.
#pragma once

#include <cstdint>

#include "adamw.h"
#include "flashrestore.h"

namespace fr {

// One matrix, as the kernels read it (uniform loads).  m <= n are its sides, mp
// and np the same in whole tiles.  Offsets in bytes: of the state, the arenas
// and, for what the products read and write, the optimizer's scratch:
//   x     mp x np, fp16    X, twice: read and written in turn
//   rest  mp x np, 8 bits  what X is more than its fp16 number, in 2^-8 of its last place
//   square    mp x mp, fp16   X X^T and polynomials of it, three at a time
//   diagonal  mp, fp32        what their diagonals are more
struct alignas(16) MuonRec {
  uint64_t numel;
  uint64_t grad, update, param, master, mom;  // param: kNone if it has none
  uint64_t x[2], rest, square[3], diagonal[3];
  uint64_t slot0, slots;  // its tiles in the walk over elements
  uint64_t sub0;          // and its first sub-tile
  uint32_t cols, m, n, mp, np;
  uint32_t wide;      // rows <= cols: X has the matrix's own rows
  uint32_t grad_f32, group;
  float scale;
  float lift;         // the power of two that X is stored times
  uint32_t paired;    // its first two steps are taken as one
  uint32_t pad_;
};
static_assert(sizeof(MuonRec) == 192, "MuonRec is 192 bytes");

// Elements of a workgroup of the walk over elements, and of those that make one
// part of a chunk's sum.
constexpr uint32_t kMuonTile = 4096, kMuonSub = 1024;
static_assert(kMuonSub * 4 <= FR_ADAMW_MIN_SUM_CHUNK, "a sub-tile lies inside a chunk");
// Sides of the products' tiles, to which those of matrices are padded.
constexpr uint32_t kMuonLarge = 256, kMuonSmall = 64;
// Matrices whose first two steps are taken as one: 3 m^3 / 2 multiplications more
// and 3 m^2 n / 2 fewer, in three launches more.  As one and one by one, us: 8 of 128 x 1024 102 and 99, of 128 x 2048 132
// and 134, of 128 x 4096 181 and 201, 4 of 512 x 2048 182 and 190, 32 of 1024 x 2048
// 1,899 and 1,952, 3 of 2048 x 4096 1,350 and 1,377 (but 2 of them 1,121 and 1,101);
// one of 4096 x 4096 1,624 and 1,537, 32 of 2048 x 2048 6,660 and 6,370, of 1024 x
// 1024 1,303 and 1,198.  (8 of 64 x 4096 157 and 170, but fewer elements average out
// what the missing gram does not mend.)
constexpr uint32_t kMuonPairedLess = 128, kMuonPairedMore = 2048, kMuonPairedRatio = 2;
constexpr float kMuonLiftA = 256.0f;  // A and Q are stored times this

// A product's work, one entry for each workgroup: a tile of a matrix, of which it
// has a copy (a chain of loads less: of a few small matrices a product takes 5 to 9
// us, most of it such chains).
struct alignas(16) MuonTile {
  MuonRec rec;
  uint32_t i0, j0;
  uint64_t pad_;
};
struct MuonTiles {
  const MuonTile* d = nullptr;
  uint64_t n = 0;
};

struct MuonArgs {
  const MuonRec* recs = nullptr;
  uint32_t n = 0;
  uint32_t side = kMuonSmall;  // of the products' tiles
  uint32_t units = 1;          // compute units, each of which takes one workgroup of large tiles
  AdamwWalk walk;          // tiles of kMuonTile elements
  uint8_t* scratch = nullptr;
  bool few_slots = false;   // no matrix has more than 256 tiles in the walk
  double* parts = nullptr;  // a sum of squares for each place of the walk
  double* factors = nullptr; // of each matrix: lift / (|D| + eps)
  const fr_muon_hyper* hyper = nullptr;
  const fr_grad_stats* stats = nullptr;
  void* state = nullptr;
  const void* grads = nullptr;
  void* updates = nullptr;
  bool momentum = false;   // of the state; else the gradients as they are
  const uint64_t* spread = nullptr;  // (matrix << 32) | tile of 4,096 elements
  uint64_t n_spread = 0;
  // the products' of matrices whose first two steps are taken one by one, as one,
  // and of all
  MuonTiles gram[3], whole[3];
  const fr_muon_coeffs* coeffs = nullptr;
  uint32_t n_steps = 0;
  // sums, or sum_parts == NULL
  uint64_t C = 0;
  fr_chunk_sum* sum_parts = nullptr;  // by sub-tile, two arrays of 8 * sub_stride places
  uint64_t sub_stride = 0;
  const AdamwFold* folds = nullptr;
  uint32_t n_folds = 0;
  fr_chunk_sum* sums = nullptr;
};

int launch_muon_direction(const MuonArgs& a, void* stream);
int launch_muon_apply(const MuonArgs& a, void* stream);

}  // namespace fr
