// Rows in 16-byte chunks, and conversions between fp32 and the stored types,
// for the kernels around the memory (norm, projections, optimizer).
#pragma once

#include "pk_device.h"

namespace pk {

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// Two floats to bf16, to nearest even; a NaN stays one.
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{lo, hi}), bf16x2_t));
}
__device__ __forceinline__ float via_bf16(float v) { return bf16_lo(to_bf16x2(v, v)); }

// Four floats to four e4m3 codes, to nearest even; |v| <= 448 in every use.
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
__device__ __forceinline__ void from_e4m3x4(uint32_t u, float* f) {
  f[0] = __builtin_amdgcn_cvt_f32_fp8((int)u, 0);
  f[1] = __builtin_amdgcn_cvt_f32_fp8((int)u, 1);
  f[2] = __builtin_amdgcn_cvt_f32_fp8((int)u, 2);
  f[3] = __builtin_amdgcn_cvt_f32_fp8((int)u, 3);
}
constexpr float E4M3_MAX = 448.f;

// A 16-byte chunk of a row.
template <typename T>
struct Chunk;
template <>
struct Chunk<uint16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void unpack(uint4 v, float* f) {
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
  }
  __device__ static __forceinline__ uint4 pack(const float* f) {
    return uint4{to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3]), to_bf16x2(f[4], f[5]), to_bf16x2(f[6], f[7])};
  }
  __device__ static __forceinline__ float stored(float v) { return via_bf16(v); }
};
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void unpack(uint4 v, float* f) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  __device__ static __forceinline__ uint4 pack(const float* f) {
    return uint4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
  __device__ static __forceinline__ float stored(float v) { return v; }
};

}  // namespace pk
