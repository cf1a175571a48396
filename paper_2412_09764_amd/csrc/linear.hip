// Matrix products of the projections around the memory, with their epilogue:
//   forward   y = act(x W^T * scales + bias) + residual,
//   backward  dx = dz W + add,  grad_W += dz^T x,  grad_bias += sum_t dz.
//
// One kernel computes C[i, j] = sum_k A(i, k) B(j, k) for the three layouts: an
// operand lies either with k consecutive (x, W of the forward; dz of dx) or with
// its rows consecutive and k strided (W of dx; both of grad_W).  The latter is
// read from LDS by transposing reads (bf16) or element by element (fp32), so
// nothing is transposed in memory.
//
// All products are bf16 ones with fp32 sums: e4m3 codes are widened (exactly) as
// they leave LDS, fp32 operands are split into three bf16 parts of which six
// products count.
//
// Tiles of 256 x 256 by eight waves (128 x 64 each); where these are too few for
// the chip, smaller ones whose waves also share k.  A stage holds 64 bytes of k;
// four stages are in LDS, filled by direct loads that run three stages ahead.
// What bounds them: a 256-wide tile keeps the matrix cores busy 79% of its cycles,
// at a clock that the power limit holds near 1.6 GHz (8192^3 bf16 at 1.27
// PFLOP/s, fp32 0.211); a 128-wide one fetches its operands at the 12-14 TB/s
// that the L2s gave in large products (0.88 PFLOP/s); small products are bound by the
// latency of a few stages and the launch (64 x 2048 x 2048: 6.8 us).  Median of calls in
// a graph, bf16 unless said:
//   32768 x 2048 x 2048 forward 272 us (least 258), with residual 295 (290; memory
//     traffic of the epilogues, which all workgroups reach at once), fp32 1336;
//   16384 x 2048 x 1024 dx 62 us, grad_W with its bias 79;
//   2000 x 2048 x 2048 26 us, e4m3 19, fp32 100;  1 x 2048 x 2048 5.8.
#include "pk_gemm.h"

namespace pk {

namespace {

// out += part[0] + part[1] + ... in this order, 4 elements a thread; the last
// workgroups do the same for the bias (one column a thread, `rows` parts).
__global__ __launch_bounds__(256) void k_add_parts(const float* __restrict__ part, int splits,
                                                   size_t n, float* __restrict__ out,
                                                   unsigned blocks, const float* __restrict__ bias_part,
                                                   int rows, int cols, float* __restrict__ bias) {
  if (blockIdx.x >= blocks) {
    const int c = (blockIdx.x - blocks) * 256 + threadIdx.x;
    if (c >= cols) return;
    float s = 0.f;
#pragma unroll 8
    for (int p = 0; p < rows; ++p) s += bias_part[(size_t)p * cols + c];
    bias[c] += s;
    return;
  }
  const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= n) return;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < splits; ++p) {
    float v[4];
    load4(part, p * n + at, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += v[e];
  }
  float o[4];
  load4(out, at, o);
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] += s[e];
  store4(out, at, o);
}

// Sums over rows: part[b, c] for the rows of workgroup b (four at a time, one a
// wave, 4 gridDim.x apart), 64 chunks of columns a workgroup; the parts are
// added by launch_add_rows.
template <typename T>
__global__ __launch_bounds__(256) void k_column_sums(const T* __restrict__ x, int64_t rows, int N,
                                                     float* __restrict__ part) {
  constexpr int C = Chunk<T>::N, AHEAD = 8;
  __shared__ float sums[3][64][C + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.y * 64 + lane;
  const bool in = c < N / C;
  const int64_t step = 4 * (int64_t)gridDim.x;
  float s[C];
#pragma unroll
  for (int e = 0; e < C; ++e) s[e] = 0.f;
  if (in) {
    for (int64_t r = 4 * (int64_t)blockIdx.x + wave; r < rows; r += AHEAD * step) {
      uint4 v[AHEAD];
#pragma unroll
      for (int a = 0; a < AHEAD; ++a)
        v[a] = r + a * step < rows ? ld16(x + (size_t)(r + a * step) * N + (size_t)c * C) : uint4{0, 0, 0, 0};
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) {
        float f[C];
        Chunk<T>::unpack(v[a], f);
#pragma unroll
        for (int e = 0; e < C; ++e) s[e] += f[e];
      }
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < C; ++e) sums[wave - 1][lane][e] = s[e];
  }
  __syncthreads();
  if (wave == 0 && in) {
#pragma unroll
    for (int e = 0; e < C; ++e) {
      s[e] += sums[0][lane][e];
      s[e] += sums[1][lane][e];
      s[e] += sums[2][lane][e];
      part[(size_t)blockIdx.x * N + (size_t)c * C + e] = s[e];
    }
  }
}

// dz = dy act'(z), 16 bytes a thread.
template <typename T, bool FAST, int ACT>
__global__ __launch_bounds__(256) void k_act_bwd(const T* dy, const T* z, int64_t chunks, T* dz) {
  using Ch = Chunk<T>;
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < chunks; c += (int64_t)gridDim.x * 256) {
    float d[Ch::N], v[Ch::N];
    Ch::unpack(ld16_nt(dy + c * Ch::N), d);
    Ch::unpack(ld16_nt(z + c * Ch::N), v);
#pragma unroll
    for (int e = 0; e < Ch::N; ++e) d[e] *= act_grad_of<FAST, ACT>(v[e]);
    *reinterpret_cast<uint4*>(dz + c * Ch::N) = Ch::pack(d);
  }
}

template <int DT, bool AKS, bool BKS, bool GRAD>
void gemm_launch(GemmArgs g, int tile, int splits, hipStream_t st) {
  g.tiles_m = ceil_div(g.M, tile_size(tile));
  g.tiles_n = ceil_div(g.N, tile_size(tile));
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * splits));
  if (tile == TILE_256)
    hipLaunchKernelGGL((k_gemm<DT, AKS, BKS, GRAD, 256, 256, 2, 4, 1>), grid, dim3(512), 0, st, g);
  else if (tile == TILE_128_K2)
    hipLaunchKernelGGL((k_gemm<DT, AKS, BKS, GRAD, 128, 128, 2, 2, 2>), grid, dim3(512), 0, st, g);
  else if (tile == TILE_64)
    hipLaunchKernelGGL((k_gemm<DT, AKS, BKS, GRAD, 64, 64, 1, 1, 4>), grid, dim3(256), 0, st, g);
  else if (tile == TILE_32)
    hipLaunchKernelGGL((k_gemm<DT, AKS, BKS, GRAD, 32, 32, 1, 1, 8>), grid, dim3(512), 0, st, g);
  else if constexpr (!GRAD)  // the weight gradient splits k instead
    hipLaunchKernelGGL((k_gemm<DT, AKS, BKS, GRAD, 128, 128, 2, 2, 1>), grid, dim3(256), 0, st, g);
}
template <int DT>
void forward_launch(const GemmArgs& g, hipStream_t st) {
  if (g.M <= FEW_T)
    hipLaunchKernelGGL(k_gemm_few<DT>, dim3((unsigned)ceil_div(g.N, 16)), dim3(FEW_WAVES * 64), 0, st, g);
  else
    gemm_launch<DT, false, false, false>(g, pick_tile(DT == D_F32, g.M, g.N), 1, st);
}

// Workgroups along the tokens of the bias gradient.
int bias_parts(int64_t T) {
  const int64_t p = (T + 63) / 64;
  return (int)(p < 256 ? p : 256);
}

inline size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

hipError_t launch_linear(const LinearCall& c, hipStream_t st) {
  if (c.T <= 0) return hipSuccess;
  LaunchTimer lt("linear", st);
  GemmArgs g{};
  g.a = c.x;
  g.b = c.w;
  g.M = c.T;
  g.N = c.N;
  g.K = g.k_split = c.K;
  g.a_scale = c.x_scale;
  g.b_scale = c.w_scale;
  g.bias = c.bias;
  g.res = c.res;
  g.z = c.z;
  g.out = c.y;
  g.act = c.act;
  g.out_bf16 = c.out_bf16;
  if (c.dt == PKMEM_BF16) forward_launch<D_BF16>(g, st);
  else if (c.dt == PKMEM_E4M3) forward_launch<D_E4M3>(g, st);
  else forward_launch<D_F32>(g, st);
  return hipGetLastError();
}

hipError_t launch_act_backward(bool bf16, const void* dy, const void* z, int act, int64_t n, void* dz,
                               hipStream_t st) {
  if (n <= 0) return hipSuccess;
  LaunchTimer lt("act_backward", st);
  const int64_t chunks = n / (bf16 ? 8 : 4);
  int64_t blocks = (chunks + 255) / 256;
  if (blocks > 16384) blocks = 16384;
#define PK_ACT(A)                                                                                  \
  case A:                                                                                          \
    if (bf16)                                                                                      \
      hipLaunchKernelGGL((k_act_bwd<uint16_t, true, A>), dim3((unsigned)blocks), dim3(256), 0, st, \
                         (const uint16_t*)dy, (const uint16_t*)z, chunks, (uint16_t*)dz);          \
    else                                                                                           \
      hipLaunchKernelGGL((k_act_bwd<float, false, A>), dim3((unsigned)blocks), dim3(256), 0, st,   \
                         (const float*)dy, (const float*)z, chunks, (float*)dz);                   \
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

size_t linear_backward_ws_bytes(bool bf16, int64_t T, int N, int K) {
  const GradPlan p = grad_plan(bf16, T, N, K);
  const int64_t rows = (int64_t)p.splits * ceil_div(K, tile_size(p.tile));  // of the bias, beside the weights
  const int64_t alone = bias_parts(T);
  return (p.splits > 1 ? up256((size_t)p.splits * N * K * sizeof(float)) : 0) +
         up256((size_t)(rows > alone ? rows : alone) * N * sizeof(float));
}

hipError_t launch_linear_backward(bool bf16, const void* dz, const void* x, const void* w, int64_t T,
                                  int N, int K, const void* add, void* dx, float* grad_w,
                                  float* grad_bias, void* ws, hipStream_t st) {
  if (T <= 0) return hipSuccess;
  LaunchTimer lt("linear_backward", st);
  if (dx) {
    GemmArgs g{};
    g.a = dz;
    g.b = w;
    g.M = T;
    g.N = K;
    g.K = g.k_split = N;
    g.res = add;
    g.out = dx;
    g.out_bf16 = bf16;
    const int tile = pick_tile(!bf16, T, K);
    if (bf16) gemm_launch<D_BF16, false, true, false>(g, tile, 1, st);
    else gemm_launch<D_F32, false, true, false>(g, tile, 1, st);
  }
  if (grad_w) {
    const GradPlan plan = grad_plan(bf16, T, N, K);
    const size_t n = (size_t)N * K;
    GemmArgs g{};
    g.a = dz;
    g.b = x;
    g.M = N;
    g.N = K;
    g.K = T;
    g.k_split = plan.k_split;
    g.out = grad_w;
    g.bias_sum = grad_bias;
    if (plan.splits > 1) {
      g.part = (float*)ws;
      if (grad_bias) g.bias_sum = (float*)((char*)ws + up256((size_t)plan.splits * n * sizeof(float)));
    }
    if (bf16) gemm_launch<D_BF16, true, true, true>(g, plan.tile, plan.splits, st);
    else gemm_launch<D_F32, true, true, true>(g, plan.tile, plan.splits, st);
    if (plan.splits > 1) {
      const unsigned blocks = (unsigned)((n / 4 + 255) / 256);
      const unsigned more = grad_bias ? (unsigned)ceil_div(N, 256) : 0;
      hipLaunchKernelGGL(k_add_parts, dim3(blocks + more), dim3(256), 0, st, g.part, plan.splits, n, grad_w,
                         blocks, g.bias_sum, plan.splits * ceil_div(K, tile_size(plan.tile)), N, grad_bias);
    }
  } else if (grad_bias) {
    const int parts = bias_parts(T);
    const dim3 grid((unsigned)parts, (unsigned)ceil_div(N / (bf16 ? 8 : 4), 64));
    float* p = (float*)ws;
    if (bf16) hipLaunchKernelGGL(k_column_sums<uint16_t>, grid, dim3(256), 0, st, (const uint16_t*)dz, T, N, p);
    else hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(256), 0, st, (const float*)dz, T, N, p);
    launch_add_rows(p, parts, N, grad_bias, st);
  }
  return hipGetLastError();
}

}  // namespace pk
