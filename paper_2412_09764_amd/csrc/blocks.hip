// Products in 8 bits with a scale for each 128 elements along k:
//   y = act(z + bias) + res,  z[t, n] = sum over blocks b of sx[b, t] sw[b, n] times the sum
//   over the block of the products of codes.
//
// A step brings the scales of its rows into LDS beside the codes; its sums start from 0 and are
// added, times their scales, in fp32.  Results in bf16 take the tiles of two steps (256 and 128
// wide) or the projections' kernel with the 8-bit instruction, results in fp32 the latter with
// exact products.  Calls in a graph, on three cards: 32768 x 2048 x 2048 124-133 us (2.1-2.2
// PFLOP/s), with residual 153-158, a scale for each row of the weight 143-151 (two vector
// instructions for each sum of a block instead of one); 8192^3 422-442 (2.5-2.6), for each row
// 504-528; 2000 x 4096 x 2048 22, for each row 24; in fp32 for each row 2048 x 1024 x 16384 88-101
// with its residual, 8192^3 1270-1310 (0.85), tiled 1115-1166 (0.94-0.99).
#include "pk_gemm8.h"

namespace pk {

namespace {

template <int MODE, int BM, int BN, int WM, int WN, int KG>
void blocks_tile(GemmArgs g, int splits, hipStream_t st) {
  g.tiles_m = ceil_div(g.M, BM);
  g.tiles_n = ceil_div(g.N, BN);
  hipLaunchKernelGGL((k_gemm<D_E4M3, false, false, false, BM, BN, WM, WN, KG, MODE>),
                     dim3((unsigned)(g.tiles_m * g.tiles_n * splits)), dim3(WM * WN * KG * 64), 0, st, g);
}
template <int MODE>
void blocks_launch(const GemmArgs& g, const BlocksPlan& p, hipStream_t st) {
  if constexpr (MODE >= G_BLOCKS8) {
    if (p.tile == TILE_256) return gemm8_launch<D_E4M3, 256, 256, 2, 4, MODE>(g, st);
    if (p.tile == TILE_128) return gemm8_launch<D_E4M3, 128, 128, 2, 2, MODE>(g, st);
  }
  if (p.tile == TILE_128_K2) blocks_tile<MODE, 128, 128, 2, 2, 2>(g, p.splits, st);
  else if (p.tile == TILE_64) blocks_tile<MODE, 64, 64, 1, 1, 4>(g, p.splits, st);
  else blocks_tile<MODE, 32, 32, 1, 1, 8>(g, p.splits, st);
}

// y from the parts of a split product, added in order: 8 columns a thread.
__global__ __launch_bounds__(256) void k_join_blocks(const GemmArgs g, int splits) {
  const int along = g.N / 8;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = t / along;
  if (i >= g.M) return;
  const int j = (int)(t - i * along) * 8;
  const size_t at = (size_t)i * g.N + j, n = (size_t)g.M * g.N;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    Raw8 p;
    p.load(g.part, s * n + at, false);
    float u[8];
    p.unpack(false, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += u[e];
  }
  Epilogue epi;
  epi.init(g, j);
  Raw8 res;
  if (g.res) res.load(g.res, at, g.out_bf16);
  epi.store(g, at, 1.f, res, v);
}

}  // namespace

size_t linear_blocks_ws_bytes(bool out_bf16, int64_t T, int N, int K) {
  if (T <= FEW_T) return 0;
  const BlocksPlan p = blocks_plan(!out_bf16, T, N, K);
  return p.splits > 1 ? (size_t)p.splits * T * N * sizeof(float) : 0;
}

hipError_t launch_linear_blocks(const LinearCall& c, bool tiled, void* ws, hipStream_t st) {
  if (c.T <= 0) return hipSuccess;
  LaunchTimer lt("linear_blocks", st);
  const BlocksPlan plan = blocks_plan(!c.out_bf16, c.T, c.N, c.K);
  GemmArgs g{};
  g.a = c.x;
  g.b = c.w;
  g.M = c.T;
  g.N = c.N;
  g.K = c.K;
  g.k_split = plan.k_split;
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
    if (tiled) blocks_launch<G_BLOCKS8_TILED>(g, plan, st);
    else blocks_launch<G_BLOCKS8>(g, plan, st);
  } else {
    if (plan.splits > 1) g.part = (float*)ws;
    if (tiled) blocks_launch<G_BLOCKS_TILED>(g, plan, st);
    else blocks_launch<G_BLOCKS>(g, plan, st);
    if (plan.splits > 1)
      hipLaunchKernelGGL(k_join_blocks, dim3((unsigned)((g.M * (g.N / 8) + 255) / 256)), dim3(256), 0, st, g, plan.splits);
  }
  return hipGetLastError();
}

}  // namespace pk
