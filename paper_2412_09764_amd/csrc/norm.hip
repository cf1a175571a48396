// Root-mean-square norm of rows with the residual's addition, its backward,
// and rows in 8 bits with one scale each.
//
//   h = x + res (stored in the row type; what is stored is normalised),
//   rstd = 1 / sqrt(mean(h^2) + eps) (0 where that sum is 0), y = h rstd w.
//
// Every kernel reads a row once into registers, 16 bytes per lane and load:
// a wave per row up to 8 KiB, four waves above.  Memory bound: two reads and
// two writes per element with the residual, three reads and one write in the
// backward, and the memory moves those bytes and no others (counters).  32768 rows of
// 2048 bf16: forward with residual 80 us called again and again (6.7 TB/s), 93 and at
// least 79 in turn with its backward, which takes 95 and at least 92 (5.7); to 8 bits
// 79 (5.9).  Four waves a row are no faster there and slower in the backward (118
// us).  Below some 4000 rows a call is bound by its launch (2000 rows: 7.5 us of kernel).
#include <type_traits>

#include "pk_internal.h"
#include "pk_norm.h"

namespace pk {

namespace {

__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float size_of(float v) { return fabsf(v); }
__device__ __forceinline__ double size_of(double v) { return fabs(v); }
template <int WPR, typename U>
__device__ __forceinline__ U row_max(U v, U* red, int wave) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = larger(v, __shfl_xor(v, m, WAVE));
  if constexpr (WPR == 1) return v;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  v = larger(larger(red[0], red[1]), larger(red[2], red[3]));
  __syncthreads();
  return v;
}

__device__ __forceinline__ float rms_rstd(float ss, int D, float eps) {
  const float m = ss / (float)D + eps;
  return m == 0.f ? 0.f : 1.f / sqrtf(m);
}

// NORM: the norm, else y = x (rows to 8 bits only).  QUANT: y in e4m3 with
// scale_out[row] = max(max|y| / 448, 2^-126); the lower limit keeps 1 / scale
// finite, a row of zeros is codes of zero.  rstd cancels in y / scale, so the codes
// are those of u / (max|u| / 448) with u = h w (times the power of two of rstd, which
// keeps it in range).  u is exact: in fp32, where h and w are bf16 or there is no w,
// with the divisor in two parts and the quotient corrected by its remainder; in fp64
// for the norm of fp32 rows.  Either way the quotient is rounded once before it is
// rounded to a code, and a value half way between two codes stays there.
template <typename T, bool NORM, bool QUANT, int NCH, int WPR>
__global__ __launch_bounds__(BLOCK) void k_rmsnorm(const T* x, const T* res,
                                                   const T* __restrict__ w, int64_t rows, int D,
                                                   float eps, T* sum_out, void* y_out,
                                                   float* __restrict__ scale_out) {
  using Ch = Chunk<T>;
  constexpr int N = Ch::N, LANES = WAVE * WPR;
  using U = typename std::conditional<NORM && sizeof(T) == 4, double, float>::type;
  __shared__ float red[4];
  const int wave = threadIdx.x / WAVE;
  const int lr = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
  const int64_t row = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  if (WPR == 1 && row >= rows) return;
  const int C = D / N;
  const size_t base = (size_t)row * D;
  float h[NCH][N];
  uint4 a[NCH], b[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int ch = lr + c * LANES;
    a[c] = b[c] = uint4{0, 0, 0, 0};
    if (ch < C) a[c] = ld16_nt(x + base + (size_t)ch * N);
    if (NORM && res && ch < C) b[c] = ld16_nt(res + base + (size_t)ch * N);
  }
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    Ch::unpack(a[c], h[c]);
    if (NORM && res) {
      float r[N];
      Ch::unpack(b[c], r);
#pragma unroll
      for (int i = 0; i < N; ++i) h[c][i] += r[i];
      a[c] = Ch::pack(h[c]);
      Ch::unpack(a[c], h[c]);
    }
    if constexpr (NORM) {
#pragma unroll
      for (int i = 0; i < N; ++i) ss = fmaf(h[c][i], h[c][i], ss);
    }
  }
  float mant = 1.f;  // QUANT: y = u * mant
  U u[QUANT ? NCH : 1][N];
  if constexpr (NORM) {
    float rstd = rms_rstd(row_sum<WPR>(ss, red, wave), D, eps);
    if constexpr (QUANT) {
      const uint32_t bits = __float_as_uint(rstd);
      mant = __uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u);
      if (rstd == rstd) rstd = __uint_as_float(bits & 0x7F800000u);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      if (ch < C && sum_out) *reinterpret_cast<uint4*>(sum_out + base + (size_t)ch * N) = a[c];
      float g[N];
#pragma unroll
      for (int i = 0; i < N; ++i) g[i] = 1.f;
      if (w && ch < C) Ch::unpack(ld16(w + (size_t)ch * N), g);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (QUANT) u[c][i] = (U)(h[c][i] * rstd) * g[i];
        else h[c][i] = h[c][i] * rstd * g[i];
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < N; ++i) u[c][i] = h[c][i];
  }
  if constexpr (!QUANT) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      if (ch < C) *reinterpret_cast<uint4*>((T*)y_out + base + (size_t)ch * N) = Ch::pack(h[c]);
    }
  } else {
    __shared__ U top[4];
    U am = 0;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < N; ++i) am = larger(am, size_of(u[c][i]));
    am = row_max<WPR>(am, top, wave);
    const float s = (float)(am * mant / (U)E4M3_MAX);
    const bool low = !(s >= 0x1p-126f);  // the codes are then y / 2^-126
    if (lr == 0) scale_out[row] = low ? 0x1p-126f : s;
    const U num = low ? (U)0x1p-126f : am, den = low ? mant : E4M3_MAX;
    const U div = num / den, inv = 1 / div;
    const U rest = sizeof(U) == 8 ? 0 : fmaf(-div, den, num) * __builtin_amdgcn_rcpf(den);
    auto code = [&](U v) -> float {
      if constexpr (sizeof(U) == 8) return (float)(v * inv);
      const float q = v * inv;
      return fmaf(fmaf(-q, rest, fmaf(-q, div, v)), inv, q);
    };
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      if (ch >= C) continue;
      uint32_t* out = reinterpret_cast<uint32_t*>((uint8_t*)y_out + base + (size_t)ch * N);
#pragma unroll
      for (int i = 0; i < N; i += 4)
        out[i / 4] = to_e4m3x4(code(u[c][i]), code(u[c][i + 1]), code(u[c][i + 2]), code(u[c][i + 3]));
    }
  }
}

// Backward: with g = dy w and xh = h rstd,
//   dx = rstd (g - xh mean(g xh)) + dsum,   grad_weight += sum over rows of dy xh.
// A row group (wave or workgroup) walks rows a fixed stride apart and keeps
// its part of grad_weight in registers; the waves of a workgroup add theirs
// in wave order, and k_add_rows adds the workgroups' parts in a fixed
// order: the same bits on every run.
template <typename T, int NCH, int WPR>
__global__ __launch_bounds__(BLOCK) void k_rmsnorm_bwd(const T* dy, const T* h_in,
                                                       const T* __restrict__ w, const T* dsum,
                                                       int64_t rows, int D, float eps, T* dx,
                                                       float* __restrict__ part) {
  using Ch = Chunk<T>;
  constexpr int N = Ch::N, LANES = WAVE * WPR;
  extern __shared__ float lds[];  // one partial row (WPR == 1)
  __shared__ float red[4];
  const int wave = threadIdx.x / WAVE;
  const int lr = WPR == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
  const int C = D / N;
  const int64_t first = WPR == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  const int64_t step = WPR == 1 ? (int64_t)gridDim.x * 4 : (int64_t)gridDim.x;
  float acc[NCH][N];
#pragma unroll
  for (int c = 0; c < NCH; ++c)
#pragma unroll
    for (int i = 0; i < N; ++i) acc[c][i] = 0.f;
  for (int64_t row = first; row < rows; row += step) {
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
    float ss = 0.f, dot = 0.f;
    float g[NCH][N];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      float hv[N], wv[N];
      Ch::unpack(rh[c], hv);
      Ch::unpack(rd[c], g[c]);
#pragma unroll
      for (int i = 0; i < N; ++i) wv[i] = 1.f;
      if (w && ch < C) Ch::unpack(ld16(w + (size_t)ch * N), wv);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        g[c][i] *= wv[i];
        ss = fmaf(hv[i], hv[i], ss);
        dot = fmaf(g[c][i], hv[i], dot);
      }
    }
    ss = row_sum<WPR>(ss, red, wave);
    dot = row_sum<WPR>(dot, red, wave);
    const float rstd = rms_rstd(ss, D, eps);
    const float mean = dot * rstd / (float)D;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      float hv[N], dv[N], sv[N];
      Ch::unpack(rh[c], hv);
      Ch::unpack(rd[c], dv);
      Ch::unpack(rs[c], sv);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float xh = hv[i] * rstd;
        acc[c][i] = fmaf(dv[i], xh, acc[c][i]);
        sv[i] += rstd * (g[c][i] - xh * mean);
      }
      if (ch < C) *reinterpret_cast<uint4*>(dx + base + (size_t)ch * N) = Ch::pack(sv);
    }
  }
  if (!part) return;
  float* out = part + (size_t)blockIdx.x * D;
  if constexpr (WPR == 1) {
    for (int s = 0; s < 4; ++s) {
      if (wave == s) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          const int ch = lr + c * LANES;
          if (ch < C)
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float v = s ? lds[ch * N + i] + acc[c][i] : acc[c][i];
              if (s < 3) lds[ch * N + i] = v;
              else out[ch * N + i] = v;
            }
        }
      }
      __syncthreads();
    }
  } else {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int ch = lr + c * LANES;
      if (ch < C)
#pragma unroll
        for (int i = 0; i < N; ++i) out[ch * N + i] = acc[c][i];
    }
  }
}

// grad[c] += sum over the parts of part[p, c]: 32 columns per workgroup, 32
// groups of parts (every 32nd) added in group order.
__global__ __launch_bounds__(1024) void k_add_rows(const float* __restrict__ part, int parts,
                                                   int D, float* __restrict__ grad) {
  __shared__ float red[32][33];
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
    grad[col] += s;
  }
}

template <typename T, bool NORM, bool QUANT>
void norm_launch(const void* x, const void* res, const void* w, int64_t rows, int D, float eps,
                 void* sum_out, void* y_out, float* scale_out, hipStream_t st) {
  const int C = D / Chunk<T>::N;
  auto slice = [&](auto* p, int64_t row) { return p ? p + (size_t)row * D : p; };
#define PK_F(NCH, WPR)                                                                             \
  constexpr int64_t per_wg = WPR == 1 ? 4 : 1, most = per_wg * LAUNCH_WORKGROUPS;                  \
  for (int64_t r = 0; r < rows; r += most) {                                                       \
    const int64_t n = rows - r < most ? rows - r : most;                                           \
    hipLaunchKernelGGL((k_rmsnorm<T, NORM, QUANT, NCH, WPR>),                                      \
                       dim3((unsigned)((n + per_wg - 1) / per_wg)), dim3(BLOCK), 0, st,            \
                       slice((const T*)x, r), slice((const T*)res, r), (const T*)w, n, D, eps,     \
                       slice((T*)sum_out, r),                                                      \
                       (void*)slice((char*)y_out, r * (QUANT ? 1 : (int64_t)sizeof(T))),           \
                       QUANT ? scale_out + r : nullptr);                                           \
  }
  PK_NORM_DISPATCH(C, PK_F);
#undef PK_F
}

template <typename T>
void norm_bwd_launch(const void* dy, const void* h, const void* w, const void* dsum, int64_t rows,
                     int D, float eps, void* dx, float* part, hipStream_t st) {
  const int C = D / Chunk<T>::N;
#define PK_F(NCH, WPR)                                                                            \
  hipLaunchKernelGGL((k_rmsnorm_bwd<T, NCH, WPR>), dim3((unsigned)norm_parts(rows)), dim3(BLOCK), \
                     (WPR) == 1 ? D * sizeof(float) : 0, st, (const T*)dy, (const T*)h,           \
                     (const T*)w, (const T*)dsum, rows, D, eps, (T*)dx, part)
  PK_NORM_DISPATCH(C, PK_F);
#undef PK_F
}

}  // namespace

void launch_add_rows(const float* part, int parts, int cols, float* out, hipStream_t st) {
  hipLaunchKernelGGL(k_add_rows, dim3((unsigned)((cols + 31) / 32)), dim3(1024), 0, st, part, parts,
                     cols, out);
}

hipError_t launch_rmsnorm(bool bf16, const void* x, const void* res, const void* w, int64_t rows,
                          int D, float eps, void* sum_out, void* y_out, float* scale_out,
                          hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  LaunchTimer lt("rmsnorm", st);
  if (bf16) {
    if (scale_out) norm_launch<uint16_t, true, true>(x, res, w, rows, D, eps, sum_out, y_out, scale_out, st);
    else norm_launch<uint16_t, true, false>(x, res, w, rows, D, eps, sum_out, y_out, nullptr, st);
  } else {
    if (scale_out) norm_launch<float, true, true>(x, res, w, rows, D, eps, sum_out, y_out, scale_out, st);
    else norm_launch<float, true, false>(x, res, w, rows, D, eps, sum_out, y_out, nullptr, st);
  }
  return hipGetLastError();
}

hipError_t launch_quantize_rows(bool bf16, const void* x, int64_t rows, int D, void* q_out,
                                float* scale_out, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  LaunchTimer lt("quantize_rows", st);
  if (bf16) norm_launch<uint16_t, false, true>(x, nullptr, nullptr, rows, D, 0.f, nullptr, q_out, scale_out, st);
  else norm_launch<float, false, true>(x, nullptr, nullptr, rows, D, 0.f, nullptr, q_out, scale_out, st);
  return hipGetLastError();
}

size_t rmsnorm_backward_ws_bytes(int64_t rows, int D) {
  return (size_t)norm_parts(rows) * D * sizeof(float);
}

hipError_t launch_rmsnorm_backward(bool bf16, const void* dy, const void* h, const void* w,
                                   const void* dsum, int64_t rows, int D, float eps, void* dx,
                                   float* grad_weight, float* part, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  LaunchTimer lt("rmsnorm_backward", st);
  if (bf16) norm_bwd_launch<uint16_t>(dy, h, w, dsum, rows, D, eps, dx, grad_weight ? part : nullptr, st);
  else norm_bwd_launch<float>(dy, h, w, dsum, rows, D, eps, dx, grad_weight ? part : nullptr, st);
  if (grad_weight) launch_add_rows(part, norm_parts(rows), D, grad_weight, st);
  return hipGetLastError();
}

}  // namespace pk
