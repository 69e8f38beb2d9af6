// Which kernel takes a layer on microscaled 4-bit operands (mx4_linear.hip).  Host arithmetic on sizes only, no HIP: the
// launcher and a CPU test share it.
#pragma once

#include <stdint.h>

#include "fast_rules.h"

namespace cwac {

// Split-K kernel, channels x tokens; tiles of 128 x 128, one workgroup per compute unit with three stages or two with two; 256 x 256.
enum { kMx4Split16 = 1, kMx4Split32x16, kMx4Split32, kMx4Split64, kMx4Tile128Deep, kMx4Tile128Pair, kMx4Tile256 };

// Estimated microseconds, fitted to 147 layers of 96 to 8192 tokens (weights cold, P = panels of 256 values of K), the two last to 110
// layers of 400 to 16384 tokens and any width (off by 9 and 6 % in the mean, by 17 % at 16384 x 11008 x 4096, 407 for 348, where no
// other form is near; the choice costs 1 % over the best).  A round is what the
// chip holds at once: 512 tiles of 32 x 32 (256 of 64 x 64), 256 or 512 of 128 x 128, 256 of 256 x 256.
//   tokens x channels x K          split 32   split 64   128 deep   128 pair   256      (measured)
//   128 x 4096 x 4096                 6.1        8.6       11.2       14.5       -
//   256 x 4096 x 4096                 9.9        8.7       11.4       14.6      23.8
//   601 x 4096 x 4096                19.9       22.2       12.4       15.2      23.9
//   256 x 4096 x 11008               23.6       17.7       30.7       41.5      68.3
//   601 x 2304 x 768                  7.6        9.2        6.7        7.0      10.6
//   2048 x 4096 x 4096               67         62         29.0       25.5      26.7
//   4096 x 4096 x 4096              125        122         55.9       47.9      37.4
//   1500 x 11008 x 4096             120        119         57.5       55.4      54.8   (258 tiles of 256 x 256)
//   2721 x 4586 x 8288                -          -         96.2       91.4      61.3
//   12757 x 4565 x 1024               -          -         78.1       59.0      70.6
//   4096 x 11008 x 4096             324        327        148        131        94.3
//   8192 x 2304 x 768                70         72         29.5       23.2      23.2
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
  const double p = (double)((k + 255) / 256);
  const int64_t t = tiles_of(m, n, 128, 128), full = t / 512, rest = t % 512;
  return 5.8 + ((double)full + (rest ? 0.43 + 0.51 * (double)rest / 512.0 : 0.0)) * (3.2 + 1.14 * p + 0.0038 * p * p);
}
inline double mx4_tile256_us(int64_t m, int n, int k) {
  const double p = (double)((k + 255) / 256);
  const int64_t t = tiles_of(m, n, 256, 256), full = t / 256, rest = t % 256;
  return 1.1 + ((double)full + (rest ? 0.68 + 0.31 * (double)rest / 256.0 : 0.0)) * (11.4 + 1.59 * p + 0.00125 * p * p);
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

// Workgroups of one launch of the split-K forms (256 threads each; a grid counts fewer than 2^32 threads); more tiles take several.
constexpr int64_t kMx4TilesPerLaunch = ((int64_t)1 << 31) / 256;

}  // namespace cwac
