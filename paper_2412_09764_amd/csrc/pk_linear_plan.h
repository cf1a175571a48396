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

// The products in blocks and the gated part (with 2 N columns) take their tiles by the same rule,
// which was measured on them too: codes with tiled scales of 2048 k, gated part in bf16 of 2048 k,
// gated part in codes of 2048 k, us in tiles of two steps 256 wide and 128 wide:
//   2000 x 8192 (256 taken) 34 / 38, 51 / 59, 29 / 34;   4096 x 4096 (256) 34 / 38, 50 / 59, 30 / 33;
//   6000 x 4096 (256) 56 / 55, 88 / 87, 50 / 48;         3000 x 4096 (128) 31 / 31, 48 / 51, 28 / 29;
//   2000 x 4096 (128) 29 / 21, 45 / 31, 26 / 18;         3000 x 2048 (128) 27 / 19, 44 / 27, 25 / 16.
// Where it takes TILE_128_K2, at 128 to 256 tiles, which is k_gemm's alone, the 128-wide tiles of
// two steps would be faster but for the gated part in bf16 of a long k: 2000 x 2048 of 2048 k in
// blocks 17.9 / 14.1 (a scale for each row 20.8 / 16.3), 1000 x 4096 16.9 / 14.0; gated 2000 x 4096
// of 1024 k in bf16 13.6 / 11.6, of 2048 k 24.5 / 25.3, in codes 17.3 / 11.8.  In codes the
// gated part's products are exact there and would not be in those tiles.

// Workgroups of the tiles of two steps (pk_gemm8.h) that 256 CUs hold at once, by LDS; of more tiles
// each takes one after another.
inline int step_tile_places(int tile) { return tile == TILE_256 ? 256 : 512; }

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

// Products of codes in blocks.  Exact ones (for fp32 results) take no tiles wider than 128, as
// they hold two sets of sums, and split k where these measured parts say so: a call of 5.5 us
// and for each k 0.0087 us in tiles of 128, 0.0033 of 64, 0.0014 of 32; a split one of 12 us and
// the writing and reading of its parts at 5 TB/s.  2048 x 1024 of 16384 k 101 us in two parts
// and 150 in one, 1024 x 1024 of 8192 k 34 in one of 64 and 37 in four of 128, 100 x 256 of
// 32768 k 19 in 32 parts and 45 in one.
struct BlocksPlan {
  int tile, splits;
  int64_t k_split;
};
inline BlocksPlan blocks_plan(bool exact, int64_t M, int64_t N, int64_t K) {
  int tile = pick_tile(false, M, N);
  if (!exact) return BlocksPlan{tile, 1, K};
  if (tile == TILE_256 || tile == TILE_128) tile = TILE_128_K2;
  const double per_k = tile == TILE_32 ? 0.0014 : tile == TILE_64 ? 0.0033 : 0.0087;
  const int64_t count = tile_count(TILE_128_K2, M, N);
  const int64_t most = count > 128 ? 1 : 256 / count < K / 1024 ? 256 / count : K / 1024;
  if (most > 1) {
    const int64_t k_split = ((K + most - 1) / most + 255) / 256 * 256;
    const int splits = ceil_div(K, k_split);
    const double one = 5.5 + per_k * K * ceil_div(tile_count(tile, M, N), 256);
    if (12.0 + 0.0087 * k_split + 1.6e-6 * splits * M * N < one) return BlocksPlan{TILE_128_K2, splits, k_split};
  }
  return BlocksPlan{tile, 1, K};
}
}  // namespace pk
