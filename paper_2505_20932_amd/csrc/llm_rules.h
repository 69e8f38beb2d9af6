// How the attention over a paged cache is split, and the append's launches.  Host arithmetic on sizes only, no HIP: the launcher, the workspace query
// and a CPU test share it.
#pragma once

#include <stdint.h>

namespace cwac {

constexpr int kPagedTile = 32;    // tokens that a wavefront takes at a time
constexpr int kPagedWaves = 4;    // wavefronts of a workgroup: they take turns over a split's tiles
constexpr int kPagedWide = 8;     // of one that takes a short length whole
constexpr int kPagedHeads = 16;   // query heads of one key head that share a workgroup: the columns of the matrix instruction
constexpr int kPagedMaxSplits = 128;

// Positions that a request's visible tokens can take: a window's lie in at most one tile more than its own number.
inline int64_t paged_span(int64_t cap, int window) {
  const int64_t n = (int64_t)window + kPagedTile - 1;
  return window > 0 && n < cap ? n : cap;
}

// Splits of `tokens` positions.  A workgroup has a fixed cost of 1.6 us (its first loads, the join), so splits are long, 1024
// tokens, where there are enough of them - at most 4096 workgroups, for requests of uneven lengths - and shorter only to fill the chip
// with workgroups (two per compute unit, twice), down to a turn of the wavefronts.  Measured in us with at most 1024 / 2048 / 4096 workgroups and
// splits of 128 tokens or more: 61 requests of 1 to 8190 tokens, 8 key heads, bf16 192 / 189 / 189; 5 of 30011 to 131072, int8
// 187 / 170 / 164; 256 of 100 to 1900 190 / 190 / 207 (split in two); 8 of 2000, 32 key heads 51 / 52 / 60; 16 of 100 to 8000,
// heads of 256 101 / 107 / 116; 64 of 100 to 6000, int8 heads of 64 61 / 60 / 53; one of 131072, one key head 17.8 at 128 splits, 19.7 at 256.
// (The int8 ones take 1 to 3 % more since their weights' unit follows the largest product of weight and scale.)
// `tokens` is the capacity of a table row, not a request's length: short requests under a wide table get fewer workgroups (61 of up to 8190
// tokens, 8 key heads: 64 per request under a table of 8192 tokens, 8 under one of 131072).
inline int paged_splits(int64_t batch, int q_heads, int kv_heads, int64_t tokens) {
  const int group = q_heads / kv_heads, tiles = (group + kPagedHeads - 1) / kPagedHeads;
  const int64_t rows = batch * kv_heads * tiles, turn = kPagedTile * kPagedWaves;
  int64_t fill = (1024 + rows - 1) / rows, turns = (tokens + turn - 1) / turn;
  if (turns < fill) fill = turns;
  int64_t even = 4096 / rows;
  if (tokens / 1024 < even) even = tokens / 1024;
  const int64_t most = fill > even ? fill : even;
  return most < 1 ? 1 : (most > kPagedMaxSplits ? kPagedMaxSplits : (int)most);
}
// Whether a length that would be split goes to one workgroup of twice the wavefronts instead, which saves the join: up to two of its turns
// (one for heads of 256, whose turns take twice as long), or as many as rows fill the chip, a turn for each 20 of them, up to eight.
// Us without / with: one request of 256 tokens 7.3 / 5.1; 32 rows of 400 7.2 / 6.8, of 700 7.8 / 8.6; 64 rows of 700 10.4 / 9.3,
// int8 10.0 / 9.9, of 1000 12.1 / 10.6, int8 10.9 / 11.5; 128 rows of 1500 25.5 / 22.0; 256 rows of up to 2000 36.4 / 31.2; 512 rows, int8,
// of up to 2000 45.9 / 39.6, of up to 3500 64.1 / 63.1; 16 rows of heads of 256, int8, of 256 tokens 9.1 / 7.9, of 400 9.0 / 11.1.
inline bool paged_wide(int64_t batch, int q_heads, int kv_heads, int head_dim, int64_t tokens) {
  if (paged_splits(batch, q_heads, kv_heads, tokens) == 1) return false;
  const int group = q_heads / kv_heads, tiles = (group + kPagedHeads - 1) / kPagedHeads;
  const int64_t rows = batch * kv_heads * tiles, turn = kPagedTile * kPagedWide, least = head_dim == 256 ? 1 : 2;
  int64_t turns = rows / 20 > least ? rows / 20 : least;
  if (turns > 8) turns = 8;
  return tokens <= turns * turn;
}
// Wavefronts of a workgroup that takes a whole length: no more than it has tiles, so that more workgroups share a compute unit (201
// requests of 25 tokens, 32 key heads, int8, four wavefronts / one: 38 / 17 us; of 60, two: 46 / 31; of up to 4 x 8 rows the same).
inline int paged_waves(int64_t tokens) { return tokens <= kPagedTile ? 1 : tokens <= 2 * kPagedTile ? 2 : kPagedWaves; }
// Tokens of one split: whole turns.
inline int64_t paged_chunk(int64_t tokens, int splits) {
  const int64_t turn = kPagedTile * kPagedWaves, each = (tokens + splits - 1) / splits;
  const int64_t c = (each + turn - 1) / turn * turn;
  return c < turn ? turn : c;
}

// Workgroups of one launch of the append (256 threads each; a grid counts fewer than 2^32 threads); more take several.
constexpr int64_t kAppendBlocksPerLaunch = ((int64_t)1 << 31) / 256;

}  // namespace cwac
