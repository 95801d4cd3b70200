// Which tiles the product of 8-bit codes runs in.  Plain constexpr code: it
// compiles on the host alone, where the choices for given sizes are checked.
#pragma once

#include <cstdint>

// Tiles of `size` rows that m rows in ngroup groups can have (grouped: every
// group, and the empty rows behind them, may end in a tile of its own).
constexpr int64_t i8_most_tiles(int m, int ngroup, bool grouped, int size) {
  if (!grouped) return ((int64_t)m + size - 1) / size;
  const int64_t t = (int64_t)m / size + ngroup + 1;
  return t < m ? t : m;
}

// Whether few enough rows share an expert's weights for tiles of 16 rows: at most
// 16 for one layer; for experts, whose rows the host does not know one by one, by
// the rows in all and their average.  Device times, us, few rows and the kernels
// that take over, even choice and (in brackets) a share of 1 / e^2 for expert e:
//   bfloat16, 4,096 x 4,096      64 experts, 4 rows each 209 211 (78 78), 8 223 217 (144 143), 16 277 223
//                                (209 154), 64 552 317 (521 316); 256 experts, 8 rows 799 837 (371 275);
//                                3 experts, 48 rows in all 24.8 26.5, 64 24.5 26.6, 128 35.6 26.9
//   bfloat16, 1,024 x 1,024      256 experts, 4 rows 53 68 (26 21), 8 60 75 (36 28), 16 73 78 (53 42)
//   float32, 1,600 to 240        64 experts, 8 rows 14.2 16.9 (12.0 16.0), 16 19.5 17.3 (17.1 16.2), 64 35.9 20.6;
//                                256 experts, 2 rows 25.7 22.7, 8 32.7 25.1 (24.4 18.7), 16 38 26 (31 20)
// A busy expert's W is read again for each of its 16-row tiles: with few rows on
// average and most of them on one of many experts that still costs up to a half.
constexpr bool i8_few_rows(int m, int n, int ngroup, bool grouped) {
  if (!grouped) return m <= 16;
  if (n <= 256) return m <= 512 && m <= 16 * ngroup;
  return m <= 64 || m <= 8 * ngroup;
}

// Whether the rows of a layer of up to 256 channels are short enough to be held
// (a chunk of 16 bytes at least, and the codes of 32 rows twice in LDS), and one
// kernel faster than two.  Device times, us, 240 channels, one kernel and two:
//   float32, 1,600 columns     512 rows 13.4 13.6, 2,048 14.1 15.2, 8,192 17.6 25.3, 262,144 468 616
//   bfloat16, 1,600 columns    256 rows 13.7 12.9, 2,048 14.3 15.2, 8,192 16.0 23.0, 262,144 337 444
//   float64, 1,024 columns     512 rows 11.5 11.8, 2,048 12.9 13.3, 8,192 20.1 26.1, 262,144 512 675
//   float64, 1,600 columns     512 rows 20.2 13.7, 8,192 35.0 35.2, 16,000 61.1 58.1, 24,000 90.0 91.5,
//                              32,000 116 122, 524,288 1,771 1,855 (27 registers of its kernel spill)
//   bfloat16, 240 columns      512 rows 6.8 7.5, 8,192 7.7 9.4, 32,000 18.9 20.6, 50,000 33.0 29.7, 262,144 131 103
//   float32, 128 columns       512 rows 5.6 6.6, 8,192 6.9 8.5, 32,000 17.6 18.8, 50,000 30.8 26.7, 262,144 126 114
//   float32, 129 columns       512 rows 6.5 7.2, 8,192 7.9 11.1, 32,000 21.5 26.4, 50,000 38.3 40.0, 262,144 170 192
// Up to 32 chunks leave half of a wavefront without one while it codes.
constexpr int kI8OneKernelLd = 2048;
constexpr bool i8_one_kernel(int m, int k, int ld, int chunk_elems) {
  const int chunks = ld / chunk_elems;
  if (k < chunk_elems || ld > kI8OneKernelLd) return false;
  if (chunks <= 32) return m <= 32768;
  return chunks <= 64 * 8 || m >= 24000;
}

// A tile of bm rows times bn channels, and its times in us: a fixed part, for
// each step of K (128 columns) the larger of one tile's time alone and the time
// of the tiles of a CU one after the other, and each tile's start and stores.
// Measured on 256 CUs (us, bf16 results; 256x256, 128x128, 128x64, 64x64 tiles):
//   4096 x 4096 x 4096   73.8  84.5 103.4 121.6     1024 x 8192 x 4096  53.0 39.5 52.8 53.6
//   2048 x 2048 x 2048   29.2  15.8  14.0  16.9     32000 x 240 x 1600  27.9 23.5 25.9 27.6
//   512 x 4096 x 4096    47.4  22.7  20.1  16.8     16000 x 240 x 1600  25.6 14.7 13.7 15.0
//   256 x 4096 x 4096    46.6  20.8  14.1  11.1     4000 x 240 x 1600   24.7 12.1  8.5  6.9
//   8192 x 2048 x 512    17.6  20.2  20.6  23.3     32000 x 512 x 512   17.8 22.3 21.2 24.1
//   262144 x 1024 x 256   205   245   249   291     131072 x 1600 x 240  163  182  183  215
struct I8Tile {
  int bm, bn;
  double fixed, alone, each, stores;
};
constexpr I8Tile kI8Tiles[] = {{256, 256, 8.0, 1.35, 1.9, 4.0},
                               {128, 128, 5.0, 0.7, 0.64, 1.4},
                               {128, 64, 4.0, 0.5, 0.35, 0.95},
                               {64, 64, 3.3, 0.25, 0.22, 0.5}};
constexpr int kI8TileKinds = sizeof(kI8Tiles) / sizeof(kI8Tiles[0]);

constexpr double i8_tile_cost(const I8Tile& t, int m, int n, int ld, int ngroup, bool grouped) {
  const int64_t tiles = i8_most_tiles(m, ngroup, grouped, t.bm) * ((n + t.bn - 1) / t.bn);
  // more threads than a launch has: the largest tile, if any
  const double fixed = tiles >= 1 << 22 ? t.fixed + 1e30 / t.bm : t.fixed;
  const double turns = (double)((tiles + 255) / 256), cu = t.each * turns;
  return fixed + ld / 128 * (t.alone > cu ? t.alone : cu) + t.stores * turns;
}

// The kind of tile for m rows times n channels of codes of ld columns.
constexpr int i8_tile(int m, int n, int ld, int ngroup, bool grouped) {
  int best = 0;
  for (int i = 1; i < kI8TileKinds; ++i)
    if (i8_tile_cost(kI8Tiles[i], m, n, ld, ngroup, grouped) < i8_tile_cost(kI8Tiles[best], m, n, ld, ngroup, grouped))
      best = i;
  return best;
}
