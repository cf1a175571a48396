// Which tile a matrix product of the projections takes, and how the weight gradient
// splits its tokens: rules on sizes and types alone, for the host.
#pragma once

#include <stdint.h>

namespace pk {

inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Tiles: 256 x 256 by eight waves; 128 x 128 by four, two workgroups a CU; the same
// with four waves more for the other half of k, one workgroup a CU; 64 x 64 by
// four waves, 32 x 32 by eight that share k.
enum { TILE_256, TILE_128, TILE_128_K2, TILE_64, TILE_32 };
constexpr int tile_size(int t) { return t == TILE_256 ? 256 : t == TILE_64 ? 64 : t == TILE_32 ? 32 : 128; }
inline int64_t tile_count(int t, int64_t M, int64_t N) { return (int64_t)ceil_div(M, tile_size(t)) * ceil_div(N, tile_size(t)); }
// The largest tiles that are enough to fill the chip; the smallest where one round
// of them does (two in fp32: 300 x 1024 x 1024 takes 14.8 us in them and 16.5 in
// tiles of 64).  2048 x 2048 bf16: 128 rows 7.2 us in tiles of 32 and 8.9 of 64, 256
// rows 12.8 and 9.6; 512 rows 12.1 in 64 and 15.1 in 128, 1024 rows 23.7 and 16.7,
// 2048 25 (K2), 4096 42 in 128 and 47.6 in 256, 8192 83 and 63.
// Rows that leave half of a 256-wide tile empty take narrower ones: 128 x 131072 x 256
// 35.7 us in 256 and 24.3 in 128, 65 x 51200 x 1024 24.4 and 23.3, fp32 137.9 and 78.
// Up to 64 rows the same holds of 128 until there are many tiles: 64 x 16384 x 2048
// 17.7 us in 64 and 20.5 in 128, 64 x 32768 x 2048 32.0 and 25.6; fp32 64 x 32768 x 2048
// 68 and 90, 64 x 51200 x 1024 70 and 78, 64 x 131072 x 256 64 and 49.
inline int pick_tile(bool f32, int64_t M, int64_t N) {
  if (tile_count(TILE_32, M, N) <= (f32 ? 512 : 256)) return TILE_32;
  if (M > 128 && tile_count(TILE_256, M, N) >= 200) return TILE_256;
  const int64_t mid = tile_count(TILE_128, M, N);
  if (mid < 128 || (M <= 64 && mid <= (f32 ? 512 : 192))) return TILE_64;
  return mid <= 256 ? TILE_128_K2 : TILE_128;
}

// grad_W [N, K] from T tokens: the tile and the number of splits of the tokens
// with the least time by these measured parts: a stage of 64 bytes of k takes a
// workgroup 0.85 us (256 wide), 0.35 (128, two groups), 0.1 (64, four groups) or
// 0.06 (32, eight groups) in bf16 and 2.3, 0.7, 0.2 and 0.09 in fp32, which takes
// six products for each; a workgroup's start and end 5 us; splitting a launch of
// 5 us, and writing and reading the parts at 5 TB/s.  4096 tokens of 1024 x 1024
// bf16: 18.1 us in tiles of 64, 21.4 in four splits of 128, 48.5 of 32; 4934 of
// 2048 x 1024 fp32: 127 us in eight splits of 256, 141 of 64.
struct GradPlan {
  int tile, splits;
  int64_t k_split;
};
inline GradPlan grad_plan(bool bf16, int64_t T, int N, int K) {
  constexpr int tiles[4] = {TILE_256, TILE_128_K2, TILE_64, TILE_32};
  constexpr double stage_us[2][4] = {{2.3, 0.7, 0.2, 0.09}, {0.85, 0.35, 0.1, 0.06}};
  const int64_t per_stage = bf16 ? 32 : 16;
  GradPlan best{TILE_64, 1, T};
  double least = 1e30;
  for (int c = 0; c < 4; ++c) {
    const int64_t count = tile_count(tiles[c], N, K);
    for (int s = 1; s <= 64; s *= 2) {
      const int64_t k_split = ((T + s - 1) / s + 63) / 64 * 64;
      const int splits = T > 0 ? ceil_div(T, k_split) : 1;
      if (splits < s && s > 1) break;
      const double rounds = (double)ceil_div(count * splits, 256);
      const double us = rounds * (5.0 + stage_us[bf16][c] * ceil_div(k_split, per_stage)) +
                        (splits > 1 ? 5.0 + 8e-6 * splits * N * K / 5.0 : 0.0);
      if (us < least) {
        least = us;
        best = GradPlan{tiles[c], splits, k_split};
      }
    }
  }
  return best;
}
}  // namespace pk
