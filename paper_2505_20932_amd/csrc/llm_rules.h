// How the attention over a paged cache is split.  Host arithmetic on sizes only, no HIP: the launcher, the workspace query
// and a CPU test share it.
#pragma once

#include <stdint.h>

namespace cwac {

constexpr int kPagedTile = 32;    // tokens that a wavefront takes at a time
constexpr int kPagedWaves = 4;    // wavefronts of a workgroup: they take turns over a split's tiles
constexpr int kPagedHeads = 16;   // query heads of one key head that share a workgroup: the columns of the matrix instruction
constexpr int kPagedMaxSplits = 128;

// Splits of `tokens` positions: as many as fill the chip four times with workgroups, none shorter than a turn of its wavefronts.
inline int paged_splits(int64_t batch, int q_heads, int kv_heads, int64_t tokens) {
  const int group = q_heads / kv_heads, tiles = (group + kPagedHeads - 1) / kPagedHeads;
  const int64_t rows = batch * kv_heads * tiles, turn = kPagedTile * kPagedWaves;
  int64_t most = (tokens + turn - 1) / turn, want = (2048 + rows - 1) / rows;
  if (want > kPagedMaxSplits) want = kPagedMaxSplits;
  if (want < most) most = want;
  return most < 1 ? 1 : (int)most;
}
// Tokens of one split: whole turns.
inline int64_t paged_chunk(int64_t tokens, int splits) {
  const int64_t turn = kPagedTile * kPagedWaves, each = (tokens + splits - 1) / splits;
  const int64_t c = (each + turn - 1) / turn * turn;
  return c < turn ? turn : c;
}

}  // namespace cwac
