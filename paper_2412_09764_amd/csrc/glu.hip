// The gated feed-forward part of a block: both projections, the activation and their
// product in one kernel, and the element-wise part of its backward.
//   z = x W^T * scales + bias, W the gate's N rows and then the up projection's N;
//   y[t, j] = act(z[t, j]) z[t, N + j];
//   dz[t, j] = dy[t, j] z[t, N + j] act'(z[t, j]),  dz[t, N + j] = dy[t, j] act(z[t, j]).
//
// The product's tiles hold 32 columns of the gate and the same 32 of the up projection in
// turn, so that one lane has both numbers of a result in its registers: z is written only
// for a backward that asks for it.
//
// Calls in a graph, on three cards: 16384 x 4096 x 1024 bf16 230-234 us, with z 243-271 (403 MB
// written); 8192 x 4096 x 8192 bf16 745-769 (1.43-1.48 PFLOP/s), e4m3 369-387 (2.8-3.0); 2000 x
// 8192 x 2048 e4m3 55-58, to fp32 (exact products) 111-118, fp32 628-661 (0.20-0.21); 1 x 8192 x
// 2048 bf16 16 (weights apart, each read at 4.2 TB/s), e4m3 10.7 (3.1), fp32 33 (4.0).  The
// element-wise backward of 16384 x 4096 bf16 107-117 us (5.7-6.3 TB/s); its exponentials are
// the exact ones, so that dz is rounded as the definition's.
#include "pk_gemm8.h"

namespace pk {

namespace {

template <int DT, int BM, int BN, int WM, int WN, int KG>
void glu_tile(GemmArgs g, hipStream_t st) {
  g.tiles_m = ceil_div(g.M, BM);
  g.tiles_n = ceil_div(g.N, BN / 2);
  hipLaunchKernelGGL((k_gemm<DT, false, false, false, BM, BN, WM, WN, KG, G_GLU>),
                     dim3((unsigned)(g.tiles_m * g.tiles_n)), dim3(WM * WN * KG * 64), 0, st, g);
}
template <int DT>
void glu_launch(const GemmArgs& g, hipStream_t st) {
  if (g.M <= FEW_T) {
    hipLaunchKernelGGL((k_gemm_few<DT, G_GLU>), dim3((unsigned)ceil_div(g.N, 16)), dim3(FEW_WAVES * 64), 0, st, g);
    return;
  }
  // The tiles of a product with 2 N columns (pick_tile, where both widths of the tiles of two
  // steps are measured).  Tiles 64 high against 32 high at sizes where
  // the rule takes either: 200 x 1024 x 4096 bf16 14.8 against 16.9 us, 777 x 328 x 200 fp32
  // 8.6 against 12.0; the other way round 300 x 512 x 1024 bf16 6.9 against 6.2 and
  // 64 x 4096 x 2048 bf16 13.5 against 11.6, which no rule on the number of tiles alone parts.
  const int tile = pick_tile(DT == D_F32, g.M, 2 * (int64_t)g.N);
  if constexpr (DT != D_F32) {
    if (g.out_bf16 && tile == TILE_256) return gemm8_launch<DT, 256, 256, 2, 4, G_GLU>(g, st);
    if (g.out_bf16 && tile == TILE_128) return gemm8_launch<DT, 128, 128, 2, 2, G_GLU>(g, st);
  }
  switch (tile) {
    case TILE_256: glu_tile<DT, 256, 256, 2, 4, 1>(g, st); break;
    case TILE_128: glu_tile<DT, 128, 128, 2, 2, 1>(g, st); break;
    case TILE_128_K2: glu_tile<DT, 128, 128, 2, 2, 2>(g, st); break;
    case TILE_64: glu_tile<DT, 64, 64, 1, 1, 4>(g, st); break;
    default: glu_tile<DT, 32, 64, 1, 1, 4>(g, st);
  }
}

// dz from dy and z, 16 bytes of columns a thread; dz may be z.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_glu_bwd(const T* dy, const T* z, int64_t chunks, int row_chunks, T* dz) {
  using Ch = Chunk<T>;
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * 256) {
    const int64_t row = c / row_chunks;
    const size_t gate = (size_t)(c + row * row_chunks) * Ch::N, up = gate + (size_t)row_chunks * Ch::N;
    float d[Ch::N], g[Ch::N], u[Ch::N];
    Ch::unpack(ld16_nt(dy + c * Ch::N), d);
    Ch::unpack(ld16_nt(z + gate), g);
    Ch::unpack(ld16_nt(z + up), u);
#pragma unroll
    for (int e = 0; e < Ch::N; ++e) {
      u[e] *= d[e] * act_grad_of<false, ACT>(g[e]);
      d[e] *= act_of<false, ACT>(g[e]);
    }
    *reinterpret_cast<uint4*>(dz + gate) = Ch::pack(u);
    *reinterpret_cast<uint4*>(dz + up) = Ch::pack(d);
  }
}

}  // namespace

hipError_t launch_glu(const LinearCall& c, hipStream_t st) {
  if (c.T <= 0) return hipSuccess;
  LaunchTimer lt("glu", st);
  GemmArgs g{};
  g.a = c.x;
  g.b = c.w;
  g.M = c.T;
  g.N = c.N;
  g.K = g.k_split = c.K;
  g.a_scale = c.x_scale;
  g.b_scale = c.w_scale;
  g.bias = c.bias;
  g.z = c.z;
  g.out = c.y;
  g.act = c.act;
  g.out_bf16 = c.out_bf16;
  if (c.dt == PKMEM_BF16) glu_launch<D_BF16>(g, st);
  else if (c.dt == PKMEM_E4M3) glu_launch<D_E4M3>(g, st);
  else glu_launch<D_F32>(g, st);
  return hipGetLastError();
}

hipError_t launch_glu_backward(bool bf16, const void* dy, const void* z, int act, int64_t T, int N, void* dz,
                               hipStream_t st) {
  if (T <= 0) return hipSuccess;
  LaunchTimer lt("glu_backward", st);
  const int row_chunks = N / (bf16 ? 8 : 4);
  const int64_t chunks = T * row_chunks;
  int64_t blocks = (chunks + 255) / 256;
  if (blocks > 16384) blocks = 16384;
#define PK_ACT(A)                                                                                        \
  case A:                                                                                                \
    if (bf16)                                                                                            \
      hipLaunchKernelGGL((k_glu_bwd<uint16_t, A>), dim3((unsigned)blocks), dim3(256), 0, st,             \
                         (const uint16_t*)dy, (const uint16_t*)z, chunks, row_chunks, (uint16_t*)dz);    \
    else                                                                                                 \
      hipLaunchKernelGGL((k_glu_bwd<float, A>), dim3((unsigned)blocks), dim3(256), 0, st,                \
                         (const float*)dy, (const float*)z, chunks, row_chunks, (float*)dz);             \
    break;
  switch (act) {
    PK_ACT(PKMEM_ACT_RELU)
    PK_ACT(PKMEM_ACT_SILU)
    PK_ACT(PKMEM_ACT_GELU)
    PK_ACT(PKMEM_ACT_NONE)
  }
#undef PK_ACT
  return hipGetLastError();
}

}  // namespace pk
