// Views into the plan that hgnn_pair_plan writes (internal).
#pragma once

#include <cstdint>

#include "common.h"

namespace hgnn {

constexpr int PAIR_T = 32;   // atoms of a tile: the edge of a matrix-core tile

struct PairPlan {
  int64_t* pair_off;      // [G+1] first byte of every graph's matrix
  int32_t* graph_off;     // [G+1] first atom of every graph (checked)
  int32_t* tile_off;      // [G+1] tiles of PAIR_T atoms before every graph; [G] = tiles in all, 0 if the offsets were refused
  int32_t* tile_graph;    // [max_tiles] graph of every tile
  int64_t max_tiles;      // what N atoms in G graphs can at most make
  size_t bytes;
};

inline PairPlan pair_plan_view(const void* plan, int32_t N, int32_t G) {
  Carver c(const_cast<void*>(plan));
  PairPlan v;
  v.max_tiles = (int64_t)N / PAIR_T + (G < N ? G : N);
  v.pair_off = c.take<int64_t>((size_t)G + 1);
  v.graph_off = c.take<int32_t>((size_t)G + 1);
  v.tile_off = c.take<int32_t>((size_t)G + 1);
  v.tile_graph = c.take<int32_t>((size_t)v.max_tiles);
  v.bytes = c.used();
  return v;
}

__host__ __device__ inline int64_t pair_pitch(int64_t n) { return (n + PAIR_T - 1) / PAIR_T * PAIR_T; }

}  // namespace hgnn
