// Which tiles a product of 8-bit rows takes (scaled_gemm.h): plain arithmetic on its sizes.
#pragma once
#include <algorithm>

namespace spark {

// Tiles: their size, and into how many parts k is cut.  All have eight waves along the outputs (a row block's codes go to
// one wave), of one or two row blocks each, and as many operands of 16 rows as there are rows or registers.
struct TilePlan { int shape, splits; };
struct TileShape { int nt, mt; float us_fp32, us_8bit; };   // us: of a k block, where the matrix instructions and conversions take the time
constexpr TileShape TILE_SHAPES[] = {{1, 2, 0.39f, 0.41f}, {1, 4, 0.61f, 0.41f}, {2, 1, 0.44f, 0.38f}, {2, 2, 0.62f, 0.58f}, {2, 4, 0.95f, 0.67f}, {2, 8, 1.66f, 0.92f}};
constexpr int PLAN_WAVES = 8;

// The plan whose estimate is shortest.  A tile's k block takes its arithmetic or its weights' way from memory, of which a CU
// gets 42 GB/s at most and all of them 6.3 TB/s (rows of tiles behind the first read them from L2); tiles go in rounds of one
// per CU; parts are written and read once more, by a launch of its own.  In us beyond a launch's own, fitted to sweeps of all
// shapes and cuts.  At 178 sizes (1 to 2048 rows, the projections of both backbones and 1000 x 1000, both types) the choice is
// 0.5 % above the fastest on average, 9 % at most (64 x 3584 x 3584 to bf16: 11.9 us, 10.9).
inline TilePlan tile_plan(int m, int row_blocks, int k, bool pair, bool fp32, int n_cu) {
  TilePlan best{0, 1};
  float best_us = 1e30f;
  const int blocks = (k + 127) / 128, groups = (blocks + 3) / 4;   // of 128, of four of them
  for (int i = 0; i < (int)(sizeof(TILE_SHAPES) / sizeof(TILE_SHAPES[0])); ++i) {
    const TileShape &t = TILE_SHAPES[i];
    if (pair ? t.nt != 2 : i == 2) continue;   // (gate and partner belong to one wave; single matrices gained nothing by the third shape)
    if (t.mt > 1 && 8 * t.mt >= m) continue;   // (half of the tile's rows would do)
    const long long tiles = (long long)((row_blocks + t.nt * PLAN_WAVES - 1) / (t.nt * PLAN_WAVES)) * ((m - 1) / (16 * t.mt) + 1);
    for (int splits = 1; splits <= groups && (splits == 1 || tiles * splits <= 2ll * n_cu); ++splits) {
      const long long wgs = tiles * splits;
      const float active = (float)std::min<long long>(wgs, n_cu), rounds = (float)((wgs + n_cu - 1) / n_cu);
      const float bytes = (float)(t.nt * PLAN_WAVES * 2048), weights = (float)row_blocks * blocks * 2048;
      const float way = std::max(bytes / 42.3e3f, bytes * active / 6.32e6f);
      const float kbs = (float)std::min(blocks, 4 * ((groups + splits - 1) / splits));
      float us = rounds * (0.11f + kbs * std::max(fp32 ? t.us_fp32 : t.us_8bit, std::min(way, weights * 1.52f / 6.32e6f / (rounds * kbs))));
      if (splits > 1) us += 2.4f + (splits + 1.1f) * (float)m * row_blocks * 64.0f / 3.83e6f;
      if (us < best_us) { best_us = us; best = TilePlan{i, splits}; }
    }
  }
  return best;
}

}  // namespace spark
