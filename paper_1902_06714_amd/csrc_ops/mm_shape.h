// Which tile a product of rows with rows takes (rows_mm.h), by its sizes: plain host code.
#pragma once

#include <cstdint>

namespace nf {

enum MmKind { MM_I8, MM_F16, MM_PARTS2 };

constexpr int MM_STAGE = 128;      // bytes of k of a stage

// The tile of a product: tiles(B) of B x B on a card of `units` compute units.
// Tiles of 32 by four groups of waves where each has a compute unit of its own, which takes
// in half the operands' bytes then (us, 64 by two groups and 32, launches included: X X^T of 203 x 3210 in pairs
// 20.2, 13.1, of 300 x 700 8.7, 6.4; a X + B X of 300 x 700 7.6, 6.7; 8-bit, 17 rows of 5000 to 700
// 11.0, 7.6, 200 of 2900 to 500 9.3, 6.3).  Larger tiles, measured (us; X' = a X + B X of m x m in pairs of parts, and in one f16 where two are given):
//   m       64, two groups   64, one     128         256
//   768     11.0 / 9.1       11.3 / 9.1  23.0 / 14.4 60.1 / 31.1    144 tiles of 64
//   1024    13.4 / 10.0      14.5 / 10.6 27.8 / 17.2 74.1 / 35.8    256
//   1400    31.6 / 19.3      28.6 / 16.0 36.5 / 21.7 94.9 / 43.0    484
//   2048    81.7 / 43.7      76.8 / 40.0 61.2 / 32.7 131 / 56.7     1024
//   4096                     471         389         348            (192: 427)
// and X X^T of 4096 with half the tiles: 128 262, 192 208, 256 245.  The larger three go by
// the rounds that their tiles make (two of 128 share a compute unit) times a tile's
// entries times its stages and 6 for its end; a stage of the smaller ones takes 1.1 and 1.2
// times as long for its entries, and the end of one of 128 runs beside another's stages
// (8-bit products of 10000 x 1024 over 7 stages: 128 25.3, 256 28.0; 8192 x 4096 over 32: 174, 143).
enum MmShape { MM_32_GROUPS, MM_64_GROUPS, MM_64, MM_128, MM_192, MM_256, MM_128_192 };
template <class F>
inline MmShape mm_shape(F&& tiles, int64_t units, int64_t stages) {
  if (tiles(32) <= units) return MM_32_GROUPS;
  const int64_t small = tiles(64);
  if (small <= units) return MM_64_GROUPS;
  if (small <= 3 * units) return MM_64;
  auto cost = [&](int64_t b, int64_t at_once, double stage, double end) {
    return (double)((tiles(b) + at_once - 1) / at_once) * (double)(at_once / units * b * b) * (stage * (double)stages + end);
  };
  const double c128 = cost(128, 2 * units, 1.2, 3.6), c192 = cost(192, units, 1.1, 6.0), c256 = cost(256, units, 1.0, 6.0);
  if (c256 <= c192 && c256 <= c128) return MM_256;
  return c192 < c128 ? MM_192 : MM_128;
}

// A product of i8, `bytes` of k.  128 x 192 where all tiles run at once then, two on a compute unit (us, 128 and
// 192 columns: 784 inputs 10000 x 1024 f32 25.3, 23.2, bf16 25.8, 24.8; 300, 16000 x 600 21.6, 21.2; 100,
// 14000 x 700 20.2, 19.7).
inline MmShape linear_shape(int64_t rows, int64_t outputs, int64_t bytes, int64_t units) {
  auto tiles = [&](int64_t b) { return ((rows + b - 1) / b) * ((outputs + b - 1) / b); };
  const MmShape s = mm_shape(tiles, units, (bytes + MM_STAGE - 1) / MM_STAGE);
  const bool once = ((rows + 127) / 128) * ((outputs + 191) / 192) <= 2 * units;
  return s == MM_128 && tiles(128) > 2 * units && once ? MM_128_192 : s;
}

// The products of an orthogonalisation of `count` matrices, m x n with m <= n, in f16 or
// pairs of f16 parts; a symmetric one's tiles are those on and below the diagonal.
enum OrthProduct { PROD_GRAM, PROD_POLY, PROD_STEP, PROD_LAST };

// bytes of a row of n, in whole stages, and of m, in whole tiles of 32 columns
inline int64_t orth_wide(bool parts, int64_t n) { return (n * (parts ? 4 : 2) + 127) / 128 * 128; }
inline int64_t orth_narrow(bool parts, int64_t m) {
  const int64_t a = parts ? 128 : 64;
  return (m * (parts ? 4 : 2) + a - 1) / a * a;
}
inline MmShape orth_shape(OrthProduct prod, bool parts, int64_t count, int64_t m, int64_t n, int64_t units) {
  auto tiles = [&](int64_t b) {
    const int64_t x = (m + b - 1) / b, y = (n + b - 1) / b;
    return count * (prod == PROD_GRAM || prod == PROD_POLY ? x * (x + 1) / 2 : x * y);
  };
  const int64_t bytes = prod == PROD_GRAM ? orth_wide(parts, n) : orth_narrow(parts, m);
  return mm_shape(tiles, units, (bytes + MM_STAGE - 1) / MM_STAGE);
}

}  // namespace nf
