// Attention for requests with few rows (tokens times the query heads of one key
// head): launch descriptor of attend_rows.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "step_common.hpp"

namespace fs {

// A tile's parts: written by the block that begins the tile.
struct RowsTile {
  int32_t first;  // slot of its first part
  int32_t block;  // block that wrote it; the others are slots 2 (block + 1), 2 (block + 2), ..
  int32_t count;  // parts; 1: the block wrote the result itself
  int32_t pad;
};

struct RowsPlan {
  int32_t blocks;       // blocks of the launch
  int32_t row_tiles;    // 16-row tiles of a request and key head (1 or 2)
  int32_t keep_parts;   // 1: results join with those of the prefix, written as parts
  float* part_o;        // [2 * blocks][16 * row_tiles][head_dim]
  float2* part_ml;      // [2 * blocks][16 * row_tiles] (mu, l)
  RowsTile* tiles;      // [kv_heads][n_req]
};

int rows_blocks(int head_dim, int row_tiles, int n_cu);
hipError_t launch_attend_rows(const AttnArgs& a, const RowsPlan& p, int dtype, int head_dim,
                              hipStream_t s);

}  // namespace fs
