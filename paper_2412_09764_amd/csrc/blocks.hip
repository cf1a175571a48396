// Products in 8 bits with a scale for each 128 elements along k:
//   y = act(z + bias) + res,  z[t, n] = sum over blocks b of sx[b, t] sw[b, n] times the sum
//   over the block of the products of codes.
//
// The projections' kernel; a stage brings the scales of its rows into LDS beside the codes.  The
// sums of a stage (64 k) start from 0 and are added, times their scales, in fp32.
#include "pk_gemm8.h"

namespace pk {

namespace {

template <int MODE, int BM, int BN, int WM, int WN, int KG>
void blocks_tile(GemmArgs g, hipStream_t st) {
  g.tiles_m = ceil_div(g.M, BM);
  g.tiles_n = ceil_div(g.N, BN);
  hipLaunchKernelGGL((k_gemm<D_E4M3, false, false, false, BM, BN, WM, WN, KG, MODE>),
                     dim3((unsigned)(g.tiles_m * g.tiles_n)), dim3(WM * WN * KG * 64), 0, st, g);
}
template <int MODE>
void blocks_launch(const GemmArgs& g, hipStream_t st) {
  constexpr bool EIGHT = MODE >= G_BLOCKS8;
  switch (pick_tile(false, g.M, g.N)) {
    case TILE_256:
      if constexpr (EIGHT) gemm8_launch<256, 256, 2, 4, MODE>(g, st);
      else blocks_tile<MODE, 256, 256, 2, 4, 1>(g, st);
      break;
    case TILE_128:
      if constexpr (EIGHT) gemm8_launch<128, 128, 2, 2, MODE>(g, st);
      else blocks_tile<MODE, 128, 128, 2, 2, 1>(g, st);
      break;
    case TILE_128_K2: blocks_tile<MODE, 128, 128, 2, 2, 2>(g, st); break;
    case TILE_64: blocks_tile<MODE, 64, 64, 1, 1, 4>(g, st); break;
    default: blocks_tile<MODE, 32, 32, 1, 1, 8>(g, st);
  }
}

}  // namespace

hipError_t launch_linear_blocks(const LinearCall& c, bool tiled, hipStream_t st) {
  if (c.T <= 0) return hipSuccess;
  LaunchTimer lt("linear_blocks", st);
  GemmArgs g{};
  g.a = c.x;
  g.b = c.w;
  g.M = c.T;
  g.N = c.N;
  g.K = g.k_split = c.K;
  g.a_block = c.x_scale;
  g.b_block = c.w_scale;
  g.bias = c.bias;
  g.res = c.res;
  g.z = c.z;
  g.out = c.y;
  g.act = c.act;
  g.out_bf16 = c.out_bf16;
  if (g.M <= FEW_T) {
    const dim3 grid((unsigned)ceil_div(g.N, 16)), block(FEW_WAVES * 64);
    if (tiled) hipLaunchKernelGGL((k_gemm_few<D_E4M3, G_BLOCKS_TILED>), grid, block, 0, st, g);
    else hipLaunchKernelGGL((k_gemm_few<D_E4M3, G_BLOCKS>), grid, block, 0, st, g);
  } else if (c.out_bf16) {
    // what the 8-bit instruction cuts off is far below half a step of bf16 for all but sums that cancel
    if (tiled) blocks_launch<G_BLOCKS8_TILED>(g, st);
    else blocks_launch<G_BLOCKS8>(g, st);
  } else {
    if (tiled) blocks_launch<G_BLOCKS_TILED>(g, st);
    else blocks_launch<G_BLOCKS>(g, st);
  }
  return hipGetLastError();
}

}  // namespace pk
