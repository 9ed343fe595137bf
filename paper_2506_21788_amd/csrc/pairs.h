// Views into the plan that hgnn_pair_plan writes (internal).
#pragma once

#include <cstdint>

#include "common.h"

namespace hgnn {

constexpr int PAIR_T = 32;   // atoms of a tile: the edge of a matrix-core tile

// What a kernel has to know of a tile, in one load: with the graph's number alone its place took two more, each waiting for the one
// before, in each of the 13,000 wavefronts of attention over 390 graphs
struct alignas(32) PairTile {
  int64_t off;        // first byte of the graph's matrix
  int32_t lo, n;      // the graph's first atom, its atoms
  int32_t i0, g;      // first atom of the tile within the graph, the graph
  int32_t unused[2];
};

struct PairPlan {
  int32_t* count;         // [1] tiles in all; 0 if the offsets were refused
  PairTile* tile;         // [max_tiles] graph after graph
  int64_t max_tiles;      // what N atoms in G graphs can at most make
  size_t bytes;
};

inline PairPlan pair_plan_view(const void* plan, int32_t N, int32_t G) {
  Carver c(const_cast<void*>(plan));
  PairPlan v;
  v.max_tiles = (int64_t)N / PAIR_T + (G < N ? G : N);
  v.count = c.take<int32_t>(1);
  v.tile = c.take<PairTile>((size_t)v.max_tiles);
  v.bytes = c.used();
  return v;
}

__host__ __device__ inline int64_t pair_pitch(int64_t n) { return (n + PAIR_T - 1) / PAIR_T * PAIR_T; }

}  // namespace hgnn
