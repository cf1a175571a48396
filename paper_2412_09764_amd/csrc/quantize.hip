// Rows, columns and tiles in 8 bits with a scale for each 128 (or 128 x 128) elements:
// the operands of the 8-bit products in blocks.
//
//   scale = max(max|x| / 448, 2^-126), code = the number nearest to 448 x / max|x| (below
//   the limit: to 2^126 x), ties to even.
//
// Every element is read once: 16 lanes hold the 128 elements of a row's block, 8 each; a
// workgroup that writes columns (transposed codes) holds 128 x 128 elements, 8 x 8 a thread,
// and turns the codes round in LDS.
//
// 32768 x 2048 bf16 rows 38 us (5.2 TB/s of reads and writes); 16384 x 2048 bf16 both ways 37
// (3.6 TB/s; the vector unit is busy 36% of it: a workgroup loads, meets, rounds, turns, meets and
// stores its square with no load of another under way); 8192 x 2048 fp32 in tiles both ways
// 22.6-23.6 (4.3-4.4).
#include "pk_internal.h"
#include "pk_row.h"

namespace pk {

namespace {

constexpr int SIDE = 128;

// Codes of the elements of one block, from the size of its largest.
template <typename T>
struct Coder;

// bf16: quotients of numbers of 8 bits come no nearer to a border between two codes than 2^-14
// of themselves, or lie on it.  x times an inverse that is within 2^-22 is therefore right
// once it is rounded to 17 bits, which puts those on a border back onto it.
template <>
struct Coder<uint16_t> {
  float inv, scale;
  __device__ __forceinline__ explicit Coder(float top) {
    constexpr float R = 1.f / E4M3_MAX;
    const float s = top * R;  // top / 448, to nearest after the correction
    scale = fmaxf(fmaf(fmaf(-s, E4M3_MAX, top), R, s), 0x1p-126f);
    if (!(top < __builtin_inff())) scale = top;
    inv = __builtin_amdgcn_rcpf(scale);
  }
  __device__ __forceinline__ float operator()(float x) const {
    return __uint_as_float((__float_as_uint(x * inv) + 0x40u) & ~0x7Fu);
  }
};

// fp32: the elements are divided as v / d, v = x f and d = max|x| f / 448 with f a power of two
// that brings max|x| to [2, 4): no product below loses digits there.  d = div + rest to 46 bits.
template <>
struct Coder<float> {
  float f, div, rest, inv, scale;
  __device__ __forceinline__ explicit Coder(float top) {
    scale = top / E4M3_MAX;
    const bool low = !(scale >= 0x1p-126f);
    if (low) scale = 0x1p-126f;
    const uint32_t e = __float_as_uint(top) & 0x7F800000u;
    f = low ? 0x1p126f : __uint_as_float(0x7F800000u - e);
    // max|x| infinite: f is 0, all codes but the infinite numbers' become 0
    const bool one = low || !(top < __builtin_inff());
    const float num = one ? 1.f : top * f, den = one ? 1.f : E4M3_MAX;
    div = num / den;
    inv = 1.f / div;
    rest = fmaf(-div, den, num) * __builtin_amdgcn_rcpf(den);
  }
  __device__ __forceinline__ float operator()(float x) const {
    const float v = x * f;
    float q = v * inv;
    q = fmaf(fmaf(-q, rest, fmaf(-q, div, v)), inv, q);
    // The quotient is rounded to 24 bits here and to a code later.  Where the 24 bits lie on a
    // border between two codes (their last 12 are 0 then) and the remainder, of 2^-34 of v at
    // least or 0 there, is not 0, one unit puts it on its own side.
    const float r = fmaf(-q, rest, fmaf(-q, div, v));
    const uint32_t b = __float_as_uint(q);
    if ((b & 0xFFFu) == 0 && fabsf(r) > fabsf(v) * 0x1p-40f)
      q = __uint_as_float((r > 0.f) == (q > 0.f) ? b + 1 : b - 1);
    return q;
  }
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    Chunk<uint16_t>::unpack(ld16_nt(p), v);
  } else {
    Chunk<float>::unpack(ld16_nt(p), v);
    Chunk<float>::unpack(ld16_nt(p + 4), v + 4);
  }
}
__device__ __forceinline__ float largest(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(v[e]));
  return m;
}
// The largest over groups of 16 lanes, in all of them.
__device__ __forceinline__ float max16(float m) {
#define PK_ROR(N) m = fmaxf(m, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(m), 0x120 + N, 15, 15, true)))
  PK_ROR(8);
  PK_ROR(4);
  PK_ROR(2);
  PK_ROR(1);
#undef PK_ROR
  return m;
}
// The largest over the wave's four lanes of equal number mod 16.
__device__ __forceinline__ float max_across(float m) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
template <typename T>
__device__ __forceinline__ uint2 codes8(const Coder<T>& c, const float (&v)[8]) {
  return uint2{to_e4m3x4(c(v[0]), c(v[1]), c(v[2]), c(v[3])), to_e4m3x4(c(v[4]), c(v[5]), c(v[6]), c(v[7]))};
}

// Rows alone: 16 rows by four blocks a workgroup.
constexpr int ROWS_AT_ONCE = 16, BLOCKS_AT_ONCE = 4;
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_rows128(const T* __restrict__ x, int64_t R, int C, int64_t groups,
                                                          unsigned char* __restrict__ q, float* __restrict__ scale) {
  const int lane = threadIdx.x & 15, blocks = (C + SIDE - 1) / SIDE;
  const int along = (blocks + BLOCKS_AT_ONCE - 1) / BLOCKS_AT_ONCE;
  for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
    const int64_t row = g / along * ROWS_AT_ONCE + (threadIdx.x >> 4);
    const int b0 = (int)(g % along) * BLOCKS_AT_ONCE;
    if (row >= R) continue;
    float v[BLOCKS_AT_ONCE][8];
#pragma unroll
    for (int i = 0; i < BLOCKS_AT_ONCE; ++i) {
      const int c = (b0 + i) * SIDE + lane * 8;
      if (c < C) load8(x + (size_t)row * C + c, v[i]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < BLOCKS_AT_ONCE; ++i) {
      const int c = (b0 + i) * SIDE + lane * 8;
      const Coder<T> code(max16(largest(v[i])));
      if (c < C) *reinterpret_cast<uint2*>(q + (size_t)row * C + c) = codes8(code, v[i]);
      if (lane == 0 && b0 + i < blocks) scale[(size_t)(b0 + i) * R + row] = code.scale;
    }
  }
}

// 128 x 128 elements a workgroup; thread t holds columns 8 (t % 16) and rows 8 (t / 16) on.
// TILE: one scale for all of them.  q and qt: either may be null.
template <typename T, bool TILE>
__global__ __launch_bounds__(256) void k_quantize_square(const T* __restrict__ x, int64_t R, int C, int64_t squares,
                                                         unsigned char* __restrict__ q, float* __restrict__ scale,
                                                         unsigned char* __restrict__ qt, float* __restrict__ scale_t) {
  constexpr int PITCH = 33;  // words of a column's codes: the 64 lanes of a write fall into all banks
  __shared__ uint32_t turned[SIDE * PITCH];
  __shared__ float tops[4][SIDE];
  const int cl = threadIdx.x & 15, rl = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int across = (C + SIDE - 1) / SIDE;
  const int64_t down = (R + SIDE - 1) / SIDE, R16 = (R + 15) / 16 * 16;
  for (int64_t s = blockIdx.x; s < squares; s += gridDim.x) {
    const int bc = (int)(s % across);
    const int64_t br = s / across;
    const int c0 = bc * SIDE + cl * 8;
    const int64_t r0 = br * SIDE + rl * 8;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (r0 + i < R && c0 < C) load8(x + (size_t)(r0 + i) * C + c0, v[i]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    }
    float top = 0.f;
    if constexpr (TILE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, largest(v[i]));
      top = max_across(max16(top));
      if ((threadIdx.x & 63) == 0) tops[wave][0] = top;
      __syncthreads();
      top = fmaxf(fmaxf(tops[0][0], tops[1][0]), fmaxf(tops[2][0], tops[3][0]));
      const Coder<T> code(top);
      if (threadIdx.x == 0) {
        if (q) scale[(size_t)bc * down + br] = code.scale;
        if (qt) scale_t[(size_t)br * across + bc] = code.scale;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint2 u = codes8(code, v[i]);
        if (q && r0 + i < R && c0 < C) *reinterpret_cast<uint2*>(q + (size_t)(r0 + i) * C + c0) = u;
#pragma unroll
        for (int e = 0; e < 8; ++e)  // the codes as bytes, for the columns
          v[i][e] = __uint_as_float(((e < 4 ? u.x : u.y) >> (8 * (e & 3))) & 0xFFu);
      }
      if (qt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t w[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i >> 2] |= __float_as_uint(v[i][e]) << (8 * (i & 3));
          turned[(cl * 8 + e) * PITCH + rl * 2] = w[0];
          turned[(cl * 8 + e) * PITCH + rl * 2 + 1] = w[1];
        }
      }
    } else {
      if (qt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i][e]));
          m = max_across(m);
          if ((threadIdx.x & 48) == 0) tops[wave][cl * 8 + e] = m;
        }
        __syncthreads();
      }
      if (q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const Coder<T> code(max16(largest(v[i])));
          if (r0 + i >= R) continue;
          if (c0 < C) *reinterpret_cast<uint2*>(q + (size_t)(r0 + i) * C + c0) = codes8(code, v[i]);
          if (cl == 0) scale[(size_t)bc * R + r0 + i] = code.scale;
        }
      }
      if (qt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = cl * 8 + e;
          const Coder<T> code(fmaxf(fmaxf(tops[0][c], tops[1][c]), fmaxf(tops[2][c], tops[3][c])));
          float col[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) col[i] = v[i][e];
          const uint2 u = codes8(code, col);
          turned[c * PITCH + rl * 2] = u.x;
          turned[c * PITCH + rl * 2 + 1] = u.y;
          if (rl == 0 && c0 + e < C) scale_t[(size_t)br * C + c0 + e] = code.scale;
        }
      }
    }
    if (qt) {
      __syncthreads();
      const int c = threadIdx.x >> 1, half = threadIdx.x & 1;
      const uint32_t* from = turned + c * PITCH + half * 16;
      const int64_t row = br * SIDE + half * 64;
      if (bc * SIDE + c < C) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (row + 16 * i < R16)
            *reinterpret_cast<uint4*>(qt + (size_t)(bc * SIDE + c) * R16 + row + 16 * i) =
                uint4{from[4 * i], from[4 * i + 1], from[4 * i + 2], from[4 * i + 3]};
      }
    }
    __syncthreads();  // turned and tops are free again
  }
}

template <typename T>
void quantize_launch(const QuantizeCall& c, hipStream_t st) {
  constexpr int64_t MOST = 1 << 20;  // workgroups; more work is walked
  const T* x = (const T*)c.x;
  unsigned char *q = (unsigned char*)c.q, *qt = (unsigned char*)c.qt;
  if (!c.tile && !qt) {
    const int blocks = (c.C + SIDE - 1) / SIDE;
    const int64_t groups = (c.R + ROWS_AT_ONCE - 1) / ROWS_AT_ONCE * ((blocks + BLOCKS_AT_ONCE - 1) / BLOCKS_AT_ONCE);
    hipLaunchKernelGGL(k_quantize_rows128<T>, dim3((unsigned)(groups < MOST ? groups : MOST)), dim3(256), 0, st, x, c.R,
                       c.C, groups, q, c.scale);
    return;
  }
  const int64_t squares = (c.R + SIDE - 1) / SIDE * ((c.C + SIDE - 1) / SIDE);
  const dim3 grid((unsigned)(squares < MOST ? squares : MOST));
  if (c.tile)
    hipLaunchKernelGGL((k_quantize_square<T, true>), grid, dim3(256), 0, st, x, c.R, c.C, squares, q, c.scale, qt, c.scale_t);
  else
    hipLaunchKernelGGL((k_quantize_square<T, false>), grid, dim3(256), 0, st, x, c.R, c.C, squares, q, c.scale, qt, c.scale_t);
}

}  // namespace

hipError_t launch_quantize_blocks(const QuantizeCall& c, hipStream_t st) {
  if (c.R <= 0) return hipSuccess;
  LaunchTimer lt("quantize_blocks", st);
  if (c.bf16) quantize_launch<uint16_t>(c, st);
  else quantize_launch<float>(c, st);
  return hipGetLastError();
}

}  // namespace pk
