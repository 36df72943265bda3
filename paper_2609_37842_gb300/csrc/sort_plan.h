// How the embedding gradient's positions are sorted by token: host arithmetic only.
#pragma once

#include <algorithm>

constexpr int kSortItems = 8;  // positions a thread
constexpr int kSortThreads = 512;
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kMaxSortBlocks = 256;
constexpr int kMaxSortBits = 9;  // of a digit

struct SortPlan {
  int passes, bits, bins, blocks, per_block;  // per_block: positions of a block's range
};

// Keys 0..V of M positions; no blocks where there are no positions.
inline SortPlan sort_plan(int V, long long M) {
  SortPlan p;
  int key_bits = 1;
  while ((1ll << key_bits) <= V) ++key_bits;
  p.passes = (key_bits + kMaxSortBits - 1) / kMaxSortBits;
  p.bits = (key_bits + p.passes - 1) / p.passes;
  p.bins = 1 << p.bits;
  const long long tiles = (M + kSortTile - 1) / kSortTile;
  const long long each = std::max(1ll, (tiles + kMaxSortBlocks - 1) / kMaxSortBlocks);
  p.per_block = static_cast<int>(each * kSortTile);
  p.blocks = static_cast<int>((tiles + each - 1) / each);
  return p;
}
