// Internal declarations shared by the host and device sources of the embedding.
#pragma once

#include <cstdint>

#include "flashrestore.h"

namespace fr {

// The workgroups that order the tokens have 16 waves, and each up to
// kEmbedRows rows, whose counts by wave it keeps in LDS.
constexpr uint32_t kEmbedVec = 8;  // columns of a lane
constexpr uint32_t kEmbedWaves = 16, kEmbedRows = 512, kEmbedGroupsLog = 8;

// A row's tokens, by their places in the order.
struct Places {
  uint32_t first, n;
};

struct EmbedArgs {
  uint64_t first = 0;
  uint32_t rows = 0, cols = 0;
  const void* ids = nullptr;
  uint32_t id_bytes = 8;
  uint64_t n = 0;  // tokens
  float scale = 1;
  // a lookup's
  const void* table = nullptr;
  bool table_f32 = false;
  void* out = nullptr;
  // a gradient's
  const void* dout = nullptr;
  bool act_f32 = false;  // of out or dout
  uint64_t stride = 0;   // elements
  void* grad = nullptr;
  bool grad_f32 = false, add = false;
  uint32_t* order = nullptr;   // tokens by row, ascending
  uint32_t* row_of = nullptr;  // the row of each of these places
  Places* places = nullptr;    // of each row; behind them how many all have
  float* runs = nullptr;       // sums of runs of long rows
};

// Places of the sums of runs that n tokens can have.
inline uint64_t embed_run_slots(uint64_t n) { return 2 * ((n + FR_EMBED_RUN - 1) / FR_EMBED_RUN) + 2; }

// Whether the launches over so many rows, places or tokens have fewer than 2^32
// threads.
inline bool embed_waves_fit(uint64_t rows, uint32_t cols) {
  return rows * ((cols + 64 * kEmbedVec - 1) / (64 * kEmbedVec)) < (uint64_t(1) << 25);
}
inline bool embed_lanes_fit(uint64_t tokens, uint32_t cols) {
  return tokens * ((cols + 64 * kEmbedVec - 1) / (64 * kEmbedVec)) < (uint64_t(1) << 26) - 4;
}

int launch_embed_lookup(const EmbedArgs& a, void* stream);
int launch_embed_grad(const EmbedArgs& a, void* stream);

}  // namespace fr
