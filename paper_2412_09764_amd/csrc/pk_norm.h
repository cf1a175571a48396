// What the norms of rows share: sums over the lanes that hold a row, and how rows are
// laid on waves and workgroups.
#pragma once

#include "pk_row.h"

namespace pk {

constexpr int BLOCK = 256;

template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* red, int wave) {
  v = group_sum<WAVE>(v);
  if constexpr (WPR == 1) return v;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  v = (red[0] + red[1]) + (red[2] + red[3]);
  __syncthreads();  // red is free again
  return v;
}
// The wave's sum in every lane, without LDS: rotations within 16 lanes, then exchanges of
// them (each adds the same two numbers in both lanes, so all lanes get the same bits).
__device__ __forceinline__ float wave_sum(float v) {
#define PK_ROR(N) v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + N, 15, 15, true))
  PK_ROR(8);
  PK_ROR(4);
  PK_ROR(2);
  PK_ROR(1);
#undef PK_ROR
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
// M sums over the lanes of a row at once; red holds 4 M numbers.
template <int WPR, int M>
__device__ __forceinline__ void row_sums(float (&v)[M], float* red, int wave) {
#pragma unroll
  for (int i = 0; i < M; ++i) v[i] = wave_sum(v[i]);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < M; ++i) red[wave * M + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = (red[i] + red[M + i]) + (red[2 * M + i] + red[3 * M + i]);
    __syncthreads();
  }
}

// Chunks per lane and waves per row for rows of C chunks: one wave up to 512
// chunks (8 KiB), a workgroup of four above.
#define PK_NORM_DISPATCH(C, F)                                            \
  do {                                                                    \
    if ((C) <= 64) { F(1, 1); }                                           \
    else if ((C) <= 128) { F(2, 1); }                                     \
    else if ((C) <= 256) { F(4, 1); }                                     \
    else if ((C) <= 512) { F(8, 1); }                                     \
    else if ((C) <= 1024) { F(4, 4); }                                    \
    else { F(8, 4); }                                                     \
  } while (0)

// One launch holds fewer than 2^32 threads: more rows go in several.
constexpr int64_t LAUNCH_WORKGROUPS = 1 << 23;

// Workgroups of the backward, fixed by the number of rows: the parts that
// grad_weight is added up from do not depend on the machine.
inline int norm_parts(int64_t rows) {
  const int64_t b = (rows + 3) / 4;
  return (int)(b < 512 ? b : 512);
}

}  // namespace pk
