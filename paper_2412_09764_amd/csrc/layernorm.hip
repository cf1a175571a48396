// Layer norm of rows with the residual's addition, and its backward.
//
//   h = x + res (stored in the row type; what is stored is normalised),
//   mean = sum h / D, var = sum (h - mean)^2 / D, rstd = 1 / sqrt(var + eps) (0 where
//   that sum is 0), y = (h - mean) rstd w + b;
//   backward, with xh = (h - mean) rstd and g = dy w:
//   dx = rstd (g - mean(g) - xh mean(g xh)) + dsum, grad_w += sum dy xh, grad_b += sum dy.
//
// A row is read once into registers.  Its mean is first summed from the differences to the
// row's first element (of a row far from zero these are exact); the second pass over the
// registers sums the deviations from that mean along with their squares, which corrects both
// mean and variance for the roundings of the first one.
//
// Memory bound: 32768 x 2048 bf16 with residual 84-86 us (6.3 TB/s), called in turn with its
// backward 96-100; backward 88-94 (dy, h, dsum read and dx written at 5.7-6.1); 16384 x 2048 fp32
// 79-81 and 88-91.  Below some 4000 rows a
// call is bound by its launch (777 x 200 fp32: 2.8 and 3.9 us of kernel, joining the parts 4.1).
#include "pk_internal.h"
#include "pk_norm.h"

namespace pk {

namespace {

template <typename T>
__device__ __forceinline__ float element(const T* p) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(*p);
  else return *p;
}

// (h - m) - d is the deviation from the mean.
struct RowStats {
  float m, d, rstd;
};
// From the sums of (h - m) / D and (h - m)^2.
__device__ __forceinline__ RowStats row_stats(float m, float d, float ss, int D, float eps) {
  const float v = ss / (float)D;  // infinity: rstd becomes 0
  // fmaxf drops a NaN: one in the row comes back with m
  const float var = (v == __builtin_inff() ? v : fmaxf(v - d * d, 0.f)) + eps;
  return {m, d, var == 0.f ? 0.f : 1.f / sqrtf(var)};
}

template <typename T, int NCH, int WPR>
__global__ __launch_bounds__(BLOCK) void k_layernorm(const T* x, const T* res, const T* __restrict__ w,
                                                     const T* __restrict__ b, int64_t rows, int D,
                                                     float eps, T* sum_out, T* y_out) {
  using Ch = Chunk<T>;
  constexpr int N = Ch::N, LANES = WAVE * WPR;
  __shared__ float red[8];
  const int wave = threadIdx.x / WAVE;
  const int lr = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
  const int64_t row = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  if (WPR == 1 && row >= rows) return;
  const int C = D / N;
  const float inv = 1.f / (float)D;
  const size_t base = (size_t)row * D;
  float h[NCH][N];
  uint4 a[NCH], r[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int ch = lr + c * LANES;
    a[c] = r[c] = uint4{0, 0, 0, 0};
    if (ch < C) a[c] = ld16_nt(x + base + (size_t)ch * N);
    if (res && ch < C) r[c] = ld16_nt(res + base + (size_t)ch * N);
  }
  const float first = element(x + base) + (res ? element(res + base) : 0.f);
  float m[1] = {0.f};
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    Ch::unpack(a[c], h[c]);
    if (res) {
      float v[N];
      Ch::unpack(r[c], v);
#pragma unroll
      for (int i = 0; i < N; ++i) h[c][i] += v[i];
      a[c] = Ch::pack(h[c]);
      Ch::unpack(a[c], h[c]);
    }
    if (lr + c * LANES < C) {
#pragma unroll
      for (int i = 0; i < N; ++i) m[0] = fmaf(h[c][i] - first, inv, m[0]);
    }
  }
  row_sums<WPR>(m, red, wave);
  const float mean = first + m[0];
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    if (lr + c * LANES < C) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        h[c][i] -= mean;
        s[0] = fmaf(h[c][i], inv, s[0]);
        s[1] = fmaf(h[c][i], h[c][i], s[1]);
      }
    }
  }
  row_sums<WPR>(s, red, wave);
  const RowStats st = row_stats(mean, s[0], s[1], D, eps);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int ch = lr + c * LANES;
    if (ch >= C) continue;
    if (sum_out) *reinterpret_cast<uint4*>(sum_out + base + (size_t)ch * N) = a[c];
    float g[N], o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = 1.f, o[i] = 0.f;
    if (w) Ch::unpack(ld16(w + (size_t)ch * N), g);
    if (b) Ch::unpack(ld16(b + (size_t)ch * N), o);
#pragma unroll
    for (int i = 0; i < N; ++i) h[c][i] = fmaf((h[c][i] - st.d) * st.rstd, g[i], o[i]);
    *reinterpret_cast<uint4*>(y_out + base + (size_t)ch * N) = Ch::pack(h[c]);
  }
}

// A row group (wave or workgroup) walks rows a fixed stride apart and keeps its parts of
// grad_w and grad_b in registers; the waves of a workgroup add theirs in wave order, and
// k_add_two adds the workgroups' parts in a fixed order: the same bits on every run.
// part: [gridDim.x, D] of grad_w, then as much of grad_b; null: no gradients.
template <typename T, int NCH, int WPR>
__global__ __launch_bounds__(BLOCK) void k_layernorm_bwd(const T* dy, const T* h_in,
                                                         const T* __restrict__ w, const T* dsum,
                                                         int64_t rows, int D, float eps, T* dx,
                                                         float* __restrict__ part) {
  using Ch = Chunk<T>;
  constexpr int N = Ch::N, LANES = WAVE * WPR;
  extern __shared__ float lds[];  // two partial rows (WPR == 1)
  __shared__ float red[16];
  const int wave = threadIdx.x / WAVE;
  const int lr = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
  const int C = D / N;
  const float inv = 1.f / (float)D;
  const int64_t row0 = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  const int64_t step = WPR == 1 ? (int64_t)gridDim.x * 4 : (int64_t)gridDim.x;
  float gw[NCH][N], gb[NCH][N];
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int i = 0; i < N; ++i) gw[c][i] = gb[c][i] = 0.f;
  // The weight stays in registers (read again for every row it is waited for twice: 32768 x
  // 2048 bf16 124 us, so 94).
  uint4 rw[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) rw[c] = w && lr + c * LANES < C ? ld16(w + (size_t)(lr + c * LANES) * N) : uint4{0, 0, 0, 0};
  for (int64_t row = row0; row < rows; row += step) {
    const size_t base = (size_t)row * D;
    uint4 rh[NCH], rd[NCH], rs[NCH];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      rh[c] = rd[c] = rs[c] = uint4{0, 0, 0, 0};
      if (ch < C) {
        rh[c] = ld16_nt(h_in + base + (size_t)ch * N);
        rd[c] = ld16_nt(dy + base + (size_t)ch * N);
        if (dsum) rs[c] = ld16_nt(dsum + base + (size_t)ch * N);
      }
    }
    const float first = element(h_in + base);
    float sum[1] = {0.f};
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (lr + c * LANES >= C) continue;
      float hv[N];
      Ch::unpack(rh[c], hv);
#pragma unroll
      for (int i = 0; i < N; ++i) sum[0] = fmaf(hv[i] - first, inv, sum[0]);
    }
    row_sums<WPR>(sum, red, wave);
    const float m = first + sum[0];
    // sums of h - m, its square, g, g (h - m)
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      if (ch >= C) continue;
      float hv[N], g[N], wv[N];
      Ch::unpack(rh[c], hv);
      Ch::unpack(rd[c], g);
#pragma unroll
      for (int i = 0; i < N; ++i) wv[i] = 1.f;
      if (w) Ch::unpack(rw[c], wv);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float v = hv[i] - m, gi = g[i] * wv[i];
        s[0] = fmaf(v, inv, s[0]);
        s[1] = fmaf(v, v, s[1]);
        s[2] = fmaf(gi, inv, s[2]);
        s[3] = fmaf(gi, v, s[3]);
      }
    }
    row_sums<WPR>(s, red, wave);
    const RowStats st = row_stats(m, s[0], s[1], D, eps);
    // mean(g xh) = rstd (sum g (h - m) / D - d mean(g))
    const float mg = s[2], mgx = st.rstd * (s[3] * inv - st.d * s[2]);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      if (ch >= C) continue;
      float hv[N], dv[N], sv[N], wv[N];
      Ch::unpack(rh[c], hv);
      Ch::unpack(rd[c], dv);
      Ch::unpack(rs[c], sv);
#pragma unroll
      for (int i = 0; i < N; ++i) wv[i] = 1.f;
      if (w) Ch::unpack(rw[c], wv);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float xh = (hv[i] - m - st.d) * st.rstd;
        gw[c][i] = fmaf(dv[i], xh, gw[c][i]);
        gb[c][i] += dv[i];
        sv[i] = fmaf(st.rstd, fmaf(-xh, mgx, fmaf(dv[i], wv[i], -mg)), sv[i]);
      }
      *reinterpret_cast<uint4*>(dx + base + (size_t)ch * N) = Ch::pack(sv);
    }
  }
  if (!part) return;
  float* ow = part + (size_t)blockIdx.x * D;
  float* ob = part + ((size_t)gridDim.x + blockIdx.x) * D;
  for (int s = 0; s < (WPR == 1 ? 4 : 1); ++s) {
    if (WPR > 1 || wave == s) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int ch = lr + c * LANES;
        if (ch >= C) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int at = ch * N + i;
          float vw = gw[c][i], vb = gb[c][i];
          if (WPR == 1 && s) vw += lds[at], vb += lds[D + at];
          if (WPR == 1 && s < 3) lds[at] = vw, lds[D + at] = vb;
          else ow[at] = vw, ob[at] = vb;
        }
      }
    }
    if (WPR == 1) __syncthreads();
  }
}

// grad_w and grad_b += the sums over their parts: 32 columns per workgroup, 32 groups of
// parts (every 32nd) added in group order.  blockIdx.y: which of the two.
__global__ __launch_bounds__(1024) void k_add_two(const float* __restrict__ part, int parts, int D,
                                                  float* __restrict__ grad_w, float* __restrict__ grad_b) {
  __shared__ float red[32][33];
  float* out = blockIdx.y ? grad_b : grad_w;
  if (!out) return;
  part += (size_t)blockIdx.y * parts * D;
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < D) {
#pragma unroll 8
    for (int p = g; p < parts; p += 32) s += part[(size_t)p * D + col];
  }
  red[g][c] = s;
  __syncthreads();
  if (g == 0 && col < D) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += red[i][c];
    out[col] += s;
  }
}

// Chunks per lane and waves per row for rows of C chunks: one wave up to 256 chunks (4 KiB), a
// workgroup of four above (32768 x 4096 bf16 forward 190-192 us, with one wave 198; backward 188,
// its two sums for each column would not fit one wave's registers).
#define PK_LAYERNORM_DISPATCH(C, F)                                       \
  do {                                                                    \
    if ((C) <= 64) { F(1, 1); }                                           \
    else if ((C) <= 128) { F(2, 1); }                                     \
    else if ((C) <= 256) { F(4, 1); }                                     \
    else if ((C) <= 512) { F(2, 4); }                                     \
    else if ((C) <= 1024) { F(4, 4); }                                    \
    else { F(8, 4); }                                                     \
  } while (0)

template <typename T>
void layernorm_launch(const void* x, const void* res, const void* w, const void* b, int64_t rows, int D,
                      float eps, void* sum_out, void* y_out, hipStream_t st) {
  const int C = D / Chunk<T>::N;
  auto slice = [&](auto* p, int64_t row) { return p ? p + (size_t)row * D : p; };
#define PK_F(NCH, WPR)                                                                             \
  constexpr int64_t per_wg = WPR == 1 ? 4 : 1, most = per_wg * LAUNCH_WORKGROUPS;                  \
  for (int64_t r = 0; r < rows; r += most) {                                                       \
    const int64_t n = rows - r < most ? rows - r : most;                                           \
    hipLaunchKernelGGL((k_layernorm<T, NCH, WPR>), dim3((unsigned)((n + per_wg - 1) / per_wg)),    \
                       dim3(BLOCK), 0, st, slice((const T*)x, r), slice((const T*)res, r),         \
                       (const T*)w, (const T*)b, n, D, eps, slice((T*)sum_out, r),                 \
                       slice((T*)y_out, r));                                                       \
  }
  PK_LAYERNORM_DISPATCH(C, PK_F);
#undef PK_F
}

template <typename T>
void layernorm_bwd_launch(const void* dy, const void* h, const void* w, const void* dsum, int64_t rows,
                          int D, float eps, void* dx, float* part, hipStream_t st) {
  const int C = D / Chunk<T>::N;
#define PK_F(NCH, WPR)                                                                            \
  hipLaunchKernelGGL((k_layernorm_bwd<T, NCH, WPR>), dim3((unsigned)norm_parts(rows)),            \
                     dim3(BLOCK), (WPR) == 1 ? 2 * D * sizeof(float) : 0, st, (const T*)dy,       \
                     (const T*)h, (const T*)w, (const T*)dsum, rows, D, eps, (T*)dx, part)
  PK_LAYERNORM_DISPATCH(C, PK_F);
#undef PK_F
}

}  // namespace

hipError_t launch_layernorm(bool bf16, const void* x, const void* res, const void* w, const void* b,
                            int64_t rows, int D, float eps, void* sum_out, void* y_out, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  LaunchTimer lt("layernorm", st);
  if (bf16) layernorm_launch<uint16_t>(x, res, w, b, rows, D, eps, sum_out, y_out, st);
  else layernorm_launch<float>(x, res, w, b, rows, D, eps, sum_out, y_out, st);
  return hipGetLastError();
}

size_t layernorm_backward_ws_bytes(int64_t rows, int D) {
  return (size_t)norm_parts(rows) * D * 2 * sizeof(float);
}

hipError_t launch_layernorm_backward(bool bf16, const void* dy, const void* h, const void* w,
                                     const void* dsum, int64_t rows, int D, float eps, void* dx,
                                     float* grad_weight, float* grad_bias, float* part, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  LaunchTimer lt("layernorm_backward", st);
  if (!grad_weight && !grad_bias) part = nullptr;
  if (bf16) layernorm_bwd_launch<uint16_t>(dy, h, w, dsum, rows, D, eps, dx, part, st);
  else layernorm_bwd_launch<float>(dy, h, w, dsum, rows, D, eps, dx, part, st);
  if (part)
    hipLaunchKernelGGL(k_add_two, dim3((unsigned)((D + 31) / 32), 2), dim3(1024), 0, st, part,
                       norm_parts(rows), D, grad_weight, grad_bias);
  return hipGetLastError();
}

}  // namespace pk
