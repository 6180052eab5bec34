// Attention for many rows (prompts, chunks, and every token's rows over a shared
// prefix): launch descriptor of attend_tiles.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "step_common.hpp"

namespace fs {

constexpr int TILE_ROWS = 128;  // rows of a block

struct TilesPlan {
  int32_t prefix;    // 1: rows of all tokens over the prefix's keys; 0: of each request over its own
  int32_t min_rows;  // own keys: requests with at most this many rows are another kernel's
  int32_t tiles;     // tiles launched per key head (a bound)
  int32_t split;     // parts that a tile's keys are cut into
  int32_t parts;     // 1: write parts (always where split > 1)
  float* part_o;     // [split][n_tok * q_heads][head_dim]
  float2* part_ml;   // [split][n_tok * q_heads] (mu, l)
};

hipError_t launch_attend_tiles(const AttnArgs& a, const TilesPlan& p, int dtype, int head_dim,
                               hipStream_t s);

}  // namespace fs
