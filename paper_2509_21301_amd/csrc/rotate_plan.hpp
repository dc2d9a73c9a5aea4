// How the rotation of dense rows is split into workgroups (host code).
#pragma once
#include <algorithm>
#include <cstdint>

namespace nova {

// An item is 8 pairs of the half layout, or 8 elements of the interleaved one or that are not turned; a thread has
// ROT_AHEAD of them in flight.  A workgroup of 256 threads has at most ROT_ROWS rows of ROT_ITEMS items.
constexpr int ROT_AHEAD = 4, ROT_ITEMS = 4096, ROT_ROWS = 16;
constexpr int64_t ROT_MAX_GROUPS = (1 << 24) - 1;        // workgroups of 256 threads in a grid dimension, which has fewer than 2^32

// floor(n / d) is the high half of n m for n < 2^32 / d, m = 2^32 / d + 1; 0 stands for d = 1.
inline uint32_t reciprocal(uint32_t d) { return d == 1 ? 0u : (uint32_t)((1ull << 32) / d + 1); }

// Items of a head, heads and rows of a workgroup, reciprocals of the items of a head and of a row; the grid.
struct RotateSplit {
  int items, heads, rows;
  uint32_t per_item, per_row;
  unsigned row_groups, head_groups;
};
inline RotateSplit split_rotate(int rows, int heads, int head_dim, int rot, bool interleaved, int cus) {
  RotateSplit d;
  d.items = (interleaved ? rot / 8 : rot / 16) + (head_dim - rot) / 8;
  d.heads = std::min(heads, ROT_ITEMS / d.items);
  d.per_item = reciprocal(d.items);
  d.per_row = reciprocal(d.items * d.heads);
  const int64_t row = (int64_t)d.items * d.heads, groups = (heads + d.heads - 1) / d.heads;
  // Rows that give every thread ROT_AHEAD items, fewer while that leaves fewer than two workgroups for each compute unit,
  // and enough of them for the grid.
  const int64_t round = std::min<int64_t>({ROT_ROWS, 256 * ROT_AHEAD / row, rows * groups / (2 * (int64_t)cus)});
  d.rows = (int)std::max<int64_t>({1, round, (rows + ROT_MAX_GROUPS - 1) / ROT_MAX_GROUPS});
  d.row_groups = (unsigned)(((int64_t)rows + d.rows - 1) / d.rows);
  d.head_groups = (unsigned)groups;
  return d;
}

}  // namespace nova
