// Which kernel takes a layer on microscaled 4-bit operands (mx4_linear.hip).  Host arithmetic on sizes only, no HIP: the
// launcher and a CPU test share it.
#pragma once

#include <stdint.h>

#include "fast_rules.h"

namespace cwac {

// Split-K kernel, channels x tokens; tiles of 128 x 128, one workgroup per compute unit with three stages or two with two; 256 x 256.
enum { kMx4Split16 = 1, kMx4Split32x16, kMx4Split32, kMx4Split64, kMx4Tile128Deep, kMx4Tile128Pair, kMx4Tile256 };

// Estimated microseconds, fitted to 200 layers of 96 to 8192 tokens (weights cold, P = panels of 256 values of K).  A round is what the
// chip holds at once: 512 tiles of 32 x 32 (256 of 64 x 64), 256 or 512 of 128 x 128, 256 of 256 x 256.
//   tokens x channels x K          split 32   split 64   128 deep   128 pair   256      (measured)
//   128 x 4096 x 4096                 6.1        8.6       10.7       14.5       -
//   256 x 4096 x 4096                 9.9        8.7       10.9       14.6      25.0
//   601 x 4096 x 4096                19.9       22.2       11.8       15.3      25.2
//   256 x 4096 x 11008               23.6       17.7       29.5       41.0      69.7
//   601 x 2304 x 768                  7.6        9.2        6.6        6.8      12.1
//   2048 x 4096 x 4096               67         62         28.8       25.4      35.5
//   4096 x 4096 x 4096              125        122         54.7       47.2      43.4
//   1500 x 11008 x 4096             120        119         57.9       55.7      63.5   (258 tiles of 256 x 256)
//   4096 x 11008 x 4096             324        327        150        134       111
//   8192 x 2304 x 768                70         72         28.7       22.7      28.4
inline double mx4_split32_us(int64_t m, int n, int k) {
  const double p = (double)((k + 255) / 256), x = (double)tiles_of(m, n, 32, 32) / 512.0;
  return 1.8 + (x < 1.0 ? (x < 0.5 ? 0.6 : 0.2 + 0.8 * x) : x) * (1.2 + 0.225 * p);
}
inline double mx4_split64_us(int64_t m, int n, int k) {
  const double p = (double)((k + 255) / 256);
  const int64_t rounds = (tiles_of(m, n, 64, 64) + 255) / 256;
  return 1.5 + (rounds == 1 ? 1.0 : (double)rounds - 0.1) * (3.4 + 0.25 * p);
}
inline double mx4_tile128_deep_us(int64_t m, int n, int k) {  // one round; more are the pair's
  const double p = (double)((k + 255) / 256);
  return tiles_of(m, n, 128, 128) <= 256 ? 5.2 + 0.3 * p + 0.006 * p * p : 1e30;
}
inline double mx4_tile128_pair_us(int64_t m, int n, int k) {
  const double p = (double)((k + 255) / 256), x = (double)tiles_of(m, n, 128, 128) / 512.0;
  if (x <= 0.5) return 5.0 + 0.7 * p;
  return (x + 0.07 < 0.95 ? 0.95 : x + 0.07) * (6.4 + 1.05 * p);
}
inline double mx4_tile256_us(int64_t m, int n, int k) {
  const double p = (double)((k + 255) / 256);
  const int64_t t = tiles_of(m, n, 256, 256), full = t / 256, rest = t % 256;
  return ((double)full * 1.1 + (rest ? 0.62 + 0.5 * (double)rest / 256.0 : 0.0)) * (9.0 + 1.75 * p);
}

inline int mx4_split_form(int64_t m, int n, int k) {
  // up to 16 tokens: 16 channels, so that there are tiles for all compute units; twice as many from where those are more than two
  // rounds (1 x 11008 x 4096: 7.0 / 6.7 us; 1 x 4096 x 4096 3.8 / 3.9, 16 x 4096 x 11008 6.9 / 8.3)
  if (m <= 16) return n > 8192 ? kMx4Split32x16 : kMx4Split16;
  // 17 to 32 tokens of a layer whose 32 x 32 tiles would leave compute units idle (32 x 4096 x 11008 9.6 / 8.2)
  if (m <= 32 && tiles_of(m, n, 32, 32) <= 192) return kMx4Split32x16;
  return mx4_split64_us(m, n, k) < mx4_split32_us(m, n, k) ? kMx4Split64 : kMx4Split32;
}

inline int mx4_form(int64_t m, int n, int k) {
  const int split = mx4_split_form(m, n, k);
  if (m < 128 || n < 128) return split;
  double best = split == kMx4Split64 ? mx4_split64_us(m, n, k) : mx4_split32_us(m, n, k);
  int form = split;
  const double deep = mx4_tile128_deep_us(m, n, k), pair = mx4_tile128_pair_us(m, n, k);
  if (deep < best) best = deep, form = kMx4Tile128Deep;
  if (pair < best) best = pair, form = kMx4Tile128Pair;
  if (m >= 256 && n >= 256 && mx4_tile256_us(m, n, k) < best) form = kMx4Tile256;
  return form;
}

}  // namespace cwac
