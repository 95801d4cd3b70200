// Which kernel and which tiles the product of 4-bit codes runs in.  Plain constexpr
// code: it compiles on the host alone, where the choices for given sizes are checked.
#pragma once

#include <cstdint>

// Tiles of `size` rows that m rows in ngroup groups can have (grouped: every
// group, and the empty rows behind them, may end in a tile of its own).
constexpr int64_t mx4_most_tiles(int m, int ngroup, bool grouped, int size) {
  if (!grouped) return ((int64_t)m + size - 1) / size;
  const int64_t t = (int64_t)m / size + ngroup + 1;
  return t < m ? t : m;
}

// The number of them that is likely: every group ends in half a tile.
constexpr int64_t mx4_likely_tiles(int m, int ngroup, bool grouped, int size) {
  if (!grouped) return ((int64_t)m + size - 1) / size;
  const int64_t t = ((int64_t)m + size - 1) / size + ngroup / 2;
  return t < m ? t : m;
}

// Whether tiles of 16 rows and 16 channels, whose K several wavefronts share, are
// faster than those below.  They are while all of them run at once (1,024 of them,
// 256 where many rows share W), and for many experts of few rows, where either
// kernel is bound by the read of W.  Device times, us, few rows and the tiles that
// take over, even choice of the expert and (in brackets) a share of 1 / e^2 for expert e:
//   4,096 x 4,096     64 rows 6.6 7.6, 96 9.7 7.8;  8,192 x 8,192   32 rows 11.6 17.0, 48 18.0 17.1
//   1,024 x 1,024     64 rows 3.4 3.9, 96 4.0 4.0, 256 5.8 4.0;  240 x 1,600   256 rows 4.0 4.9
//   2,048 x 512       64 rows 3.4 3.4, 96 4.3 3.6
//   4,096 x 4,096     3 experts, 48 rows in all 7.8 9.7 (10.8 9.7), 96 11.8 10.0;
//                     16 experts, 64 rows 25.0 23.8 (20.3 18.2), 128 26.4 25.3, 256 34.7 25.6;
//                     64 experts, 128 rows 90 108 (28 26), 256 111 118 (37 27), 512 120 119 (60 43)
//   1,024 x 1,024     3 experts, 96 rows 5.2 6.1, 192 7.0 6.2; 16 experts, 128 rows 5.8 6.2, 256 6.6 6.3;
//                     64 experts, 256 rows 8.8 10.0 (6.5 7.0), 512 10.4 10.0 (8.1 7.3)
//   240 x 1,600       3 experts, 192 rows 5.1 7.0; 16 experts, 256 rows 6.5 7.1, 1,024 7.8 7.1;
//                     64 experts, 512 rows 7.5 7.3 (6.0 7.2), 2,048 13.9 7.4
constexpr bool mx4_few_rows(int m, int n, int ngroup, bool grouped) {
  const int64_t units = mx4_likely_tiles(m, ngroup, grouped, 16) * ((n + 15) / 16);
  if (!grouped) return m <= 16 || units <= 256 || (m <= 64 && units <= 1024);
  return m <= 48 || units <= 1024 || (ngroup >= 32 && m <= 4 * ngroup);
}

// A tile of bm rows times bn channels, and its times in us: a fixed part, for each
// step of K (256 columns) the larger of one tile's time alone and the time of the
// tiles of a CU one after the other, and each tile's start and stores.  A group's
// tiles share less: each takes at least its bytes at 39 KB a us, the rate of a CU
// when all of them read past L2.  Measured on 256 CUs (us, bf16 results; 256x256,
// 128x128, 128x64, 64x64 tiles):
//   8192 x 8192 x 8192   254 299 358 412         4096 x 4096 x 4096  39.3 44.4 50.2 58.8
//   2048 x 2048 x 2048   20.4 11.9 10.1 11.1     1024 x 8192 x 4096  34.6 24.0 28.3 31.5
//   512 x 4096 x 4096    30.4 16.7 11.9 10.6     256 x 4096 x 4096   29.9 16.1 11.3 8.3
//   32000 x 240 x 1600   20.5 15.1 17.7 17.5     16000 x 240 x 1600  18.2 11.0 9.5 9.8
//   4000 x 240 x 1600    17.2 10.1 7.2 5.4       8192 x 2048 x 512   14.2 15.5 15.1 16.7
//   262144 x 1024 x 256  143 157 167 184         131072 x 1600 x 240 118 135 126 142
// and of experts (rows, channels, columns, experts)
//   32768 4096 4096 16   355 485 559 583         4096 2048 2048 16   26.3 29.2 28.4 30.7
//   2048 4096 4096 8     39.4 42.9 40.8 46.4     1024 4096 4096 64   176 144 164 134
//   32000 240 1600 3     24.5 19.1 24.8 23.6
struct Mx4Tile {
  int bm, bn;
  double fixed, alone, each, stores;
};
constexpr Mx4Tile kMx4Tiles[] = {{256, 256, 8.0, 1.4, 1.9, 4.0},
                                 {128, 128, 5.0, 0.6, 0.53, 1.4},
                                 {128, 64, 4.0, 0.38, 0.316, 0.95},
                                 {64, 64, 3.3, 0.25, 0.184, 0.5}};
constexpr int kMx4TileKinds = sizeof(kMx4Tiles) / sizeof(kMx4Tiles[0]);

constexpr double mx4_tile_cost(const Mx4Tile& t, int m, int n, int steps, int ngroup, bool grouped) {
  const int64_t cols = (n + t.bn - 1) / t.bn, tiles = mx4_likely_tiles(m, ngroup, grouped, t.bm) * cols;
  // more threads than a launch has: the largest tile, if any
  const double fixed = mx4_most_tiles(m, ngroup, grouped, t.bm) * cols >= 1 << 22 ? t.fixed + 1e30 / t.bm : t.fixed;
  const double bytes = (t.bm + t.bn) * 136 / 39e3;
  const double each = grouped && bytes > t.each ? bytes : t.each;
  const double turns = (double)((tiles + 255) / 256), cu = each * turns;
  return fixed + steps * (t.alone > cu ? t.alone : cu) + t.stores * turns;
}

// The kind of tile for m rows times n channels of codes of 256 steps columns.
constexpr int mx4_tile(int m, int n, int steps, int ngroup, bool grouped) {
  int best = 0;
  for (int i = 1; i < kMx4TileKinds; ++i)
    if (mx4_tile_cost(kMx4Tiles[i], m, n, steps, ngroup, grouped) < mx4_tile_cost(kMx4Tiles[best], m, n, steps, ngroup, grouped))
      best = i;
  return best;
}
