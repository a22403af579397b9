// How the tiles of a product are dealt out to persistent CTA pairs: whole tiles as long as they fill all pairs, and the rest, which would
// leave most pairs idle for the time of a tile, cut into narrower pieces.
#pragma once

#include <cstdint>

namespace falqon {

struct TileWalk {
  int block_n;      // width of a whole tile
  int full;         // whole tiles (a multiple of the number of pairs)
  int parts;        // pieces of each of the others,
  int part_n;       // of this width, a multiple of 32
  int items;        // full + others * parts
};

// Item -> the tile it belongs to, and which columns of it.
__host__ __device__ __forceinline__ int walk_tile(const TileWalk& w, int item, int* first_col, int* width) {
  if (item < w.full) {
    *first_col = 0, *width = w.block_n;
    return item;
  }
  const int rest = item - w.full, part = rest % w.parts;
  *first_col = part * w.part_n;
  *width = w.block_n - *first_col < w.part_n ? w.block_n - *first_col : w.part_n;
  return w.full + rest / w.parts;
}

// A tile's time goes with the bytes that its operands bring through L2: `constant` columns' worth of A and its own of B.
// *cost: the walk's time in these units.
inline TileWalk plan_walk(int64_t tiles, int64_t pairs, int block_n, int constant, int64_t* cost) {
  TileWalk w{block_n, 0, 1, block_n, 0};
  const int64_t rest = tiles % pairs;
  w.full = static_cast<int>(tiles - rest);
  *cost = tiles / pairs * (block_n + constant);
  if (rest > 0) {
    for (int parts = 4; parts >= 1; --parts) {
      const int n = (block_n / parts + 31) / 32 * 32;
      if (rest * parts > pairs || n * (parts - 1) >= block_n) continue;
      w.parts = parts, w.part_n = n;
      break;
    }
    *cost += (3 * w.part_n + block_n) / 4 + constant;      // (a piece's copies of B are a whole tile's)
  }
  w.items = static_cast<int>(w.full + rest * w.parts);
  return w;
}

}  // namespace falqon
