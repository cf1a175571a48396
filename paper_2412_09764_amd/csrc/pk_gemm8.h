// Matrix products of e4m3 codes at the 8-bit matrix instruction's rate, for results that are
// stored in bf16: the large tiles of the products in blocks and of the gated part.
#pragma once

#include "pk_gemm.h"

namespace pk {

namespace {

constexpr int STEP_K = 128;  // k of a step: one block of scales, one 16x16x128 instruction

// See mma_e4m3 on what the instruction keeps.  The lanes' 32 k may be any, the same for both.
__device__ __forceinline__ f32x4_t mma_e4m3_16(const uint4 (&b)[2], const uint4 (&a)[2], f32x4_t c) {
  typedef __attribute__((ext_vector_type(8))) int i32x8_t;
  const i32x8_t y{(int)b[0].x, (int)b[0].y, (int)b[0].z, (int)b[0].w, (int)b[1].x, (int)b[1].y, (int)b[1].z, (int)b[1].w};
  const i32x8_t x{(int)a[0].x, (int)a[0].y, (int)a[0].z, (int)a[0].w, (int)a[1].x, (int)a[1].y, (int)a[1].z, (int)a[1].w};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(y, x, c, 0, 0, 0, 0, 0, 0);
}

// Rows of 128 bytes (a step's k) in LDS; 16-byte chunk c of row r lies at slot
// c ^ ((r >> 1) & 7): the 16 lanes that LDS serves at once then read 16 different 16-byte
// columns of its 64 banks.  GLU: as Operand's.
template <int R, int NWAVE, bool GLU>
struct Codes {
  static constexpr int BYTES = R * STEP_K, LOADS = BYTES / 1024 / NWAVE;
  // A load brings 8 rows.  Loads of one wave are a fixed number of rows apart, so one offset
  // serves them all; rows past the end lie past the end of the resource.
  static_assert(NWAVE == 4 || NWAVE == 8, "the same chunks in every load of a wave");
  const char* base;
  int64_t up;
  uint32_t off, row;
  int bytes;
  int left;  // k from the next step on

  __device__ static __forceinline__ int source_chunk(int wave, int lane) {
    return (lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7);
  }
  __device__ __forceinline__ void init(const void* p, int64_t row0, int64_t rows, int64_t K, int wave, int lane) {
    left = (int)K;
    base = (const char*)p + row0 * K;
    up = rows * K;
    row = (uint32_t)K;
    bytes = (int)((rows - row0 < R ? rows - row0 : R) * K);
    off = (uint32_t)((GLU ? (wave & 3) : wave) * 8 + (lane >> 3)) * row + source_chunk(wave, lane) * 16;
    if (GLU && (wave & 4)) base += up;
  }
  // All loads of this wave of a step.  bytes counts from the step's k on, so that the last row
  // ends with the resource; where k has ended nothing is read and the slots become 0.
  __device__ __forceinline__ void load(unsigned char* lds, int wave, int lane) {
    const uint32_t room = bytes > 0 ? (uint32_t)bytes : 0u;
    const uint32_t o = left >= STEP_K || source_chunk(wave, lane) * 16 < left ? off : OUTSIDE;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const bool other = GLU && NWAVE == 4 && (i & 1);  // the up projection's rows
      const uint32_t r = GLU ? (NWAVE == 4 ? i / 2 : i) * 32 : i * NWAVE * 8;
      lds_dma16_buf(raw_buffer(other ? base + up : base, room), o + r * row, 0u, lds + (i * NWAVE + wave) * 1024);
    }
    base += STEP_K;
    bytes -= STEP_K;
    left -= STEP_K;
  }
  // This lane's 32 codes of row r: chunks q and q + 4, q = lane / 16.
  __device__ static __forceinline__ void read(const unsigned char* lds, int r, int lane, uint4 (&f)[2]) {
    const int c = (lane >> 4) ^ ((r >> 1) & 7);
    f[0] = ld16(lds + r * STEP_K + c * 16);
    f[1] = ld16(lds + r * STEP_K + (c ^ 4) * 16);
  }
};

// Tiles of BM x BN by WM x WN waves with 64 columns each, two steps in LDS.  A step: the waves
// meet when its codes have landed and the step before has been read, the loads of the next one
// are issued, and each wave walks down its blocks of 16 rows, the fragments of a block read
// while the one before is multiplied.  The last block's operands stay in registers over the
// meeting, so that the matrix cores have work while the first reads return.  MODE: G_GLU (sums
// in place), G_BLOCKS8 and G_BLOCKS8_TILED (a step's sums are added with their scales two
// products later).
template <int BM, int BN, int WM, int WN, int MODE>
__global__ __launch_bounds__(WM* WN * 64) void k_gemm8(const GemmArgs g) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NJ = BN / WN / 16;
  constexpr bool GLU = MODE == G_GLU, TILED = MODE == G_BLOCKS8_TILED;
  static_assert(NJ == 4, "64 columns a wave");
  using CA = Codes<BM, NW, false>;
  using CB = Codes<BN, NW, GLU>;
  constexpr int SCALE_LOADS = GLU ? 0 : (BM + BN) / 64 / NW, SCALES_AT = CA::BYTES + CB::BYTES;
  constexpr int L = CA::LOADS + CB::LOADS + SCALE_LOADS, BYTES = SCALES_AT + (GLU ? 0 : (BM + BN) * 4);
  __shared__ __align__(1024) unsigned char st0[BYTES], st1[BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // tiles in the order of k_gemm's
  const int nwg = gridDim.x, x = blockIdx.x & 7, q = nwg >> 3, rem = nwg & 7;
  int pid = x * q + (x < rem ? x : rem) + (blockIdx.x >> 3);
  const int group = pid / (4 * g.tiles_n), m_first = group * 4;
  const int m_count = g.tiles_m - m_first < 4 ? g.tiles_m - m_first : 4;
  pid -= group * 4 * g.tiles_n;
  const int64_t i0 = (int64_t)(m_first + pid % m_count) * BM;
  const int j0 = pid / m_count * (GLU ? BN / 2 : BN);

  CA ca;
  CB cb;
  ca.init(g.a, i0, g.M, g.K, wave, lane);
  cb.init(g.b, j0, g.N, g.K, wave, lane);
  const int wi = (wave / WN) * (BM / WM), wj = (wave % WN) * 64;
  const float* scale_at[SCALE_LOADS ? SCALE_LOADS : 1];
  int scale_step[SCALE_LOADS ? SCALE_LOADS : 1];
#pragma unroll
  for (int i = 0; i < SCALE_LOADS; ++i) {  // rows past the end take the last one's: their codes are 0
    const int r = (i * NW + wave) * 64 + lane;
    if (r < BM) {
      scale_at[i] = g.a_block + (i0 + r < g.M ? i0 + r : g.M - 1);
      scale_step[i] = (int)g.M;
    } else {
      const int j = j0 + r - BM < g.N ? j0 + r - BM : g.N - 1;
      scale_at[i] = g.b_block + (TILED ? j / SCALE_K : j);
      scale_step[i] = TILED ? (g.N + SCALE_K - 1) / SCALE_K : g.N;
    }
  }
  auto fill = [&](unsigned char* st) PK_INLINE {
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {
      lds_dma4(scale_at[i], st + SCALES_AT + (i * NW + wave) * 256);
      if (ca.left > STEP_K) scale_at[i] += scale_step[i];  // after the last block: that one again
    }
    ca.load(st, wave, lane);
    cb.load(st + CA::BYTES, wave, lane);
  };

  f32x4_t acc[MI][NJ], p[3];
  uint4 fa[2][2], fb[NJ][2];
  float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[NJ][TILED ? 1 : 4];
  const uint4 none{0, 0, 0, 0};
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // before the first step: a last block of zeros
#pragma unroll
  for (int nj = 0; nj < NJ; ++nj) {
    fb[nj][0] = fb[nj][1] = none;
#pragma unroll
    for (int e = 0; e < (TILED ? 1 : 4); ++e) sb[nj][e] = 0.f;
  }
  fa[(MI - 1) & 1][0] = fa[(MI - 1) & 1][1] = none;

  auto read_a = [&](const unsigned char* st, int mi) PK_INLINE {
    const int r = wi + mi * 16 + (lane & 15);
    CA::read(st, r, lane, fa[mi & 1]);
    if constexpr (!GLU) sa[mi & 3] = reinterpret_cast<const float*>(st + SCALES_AT)[r];
  };
  auto read_sb = [&](const unsigned char* st) PK_INLINE {
    if constexpr (!GLU) {
      const float* sc = reinterpret_cast<const float*>(st + SCALES_AT) + BM + wj;
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj) {
        if constexpr (TILED) {
          if (nj == 0) sb[0][0] = sc[0];  // 64 columns of one tile
        } else {
          const float4 f = *reinterpret_cast<const float4*>(sc + nj * 16 + 4 * (lane >> 4));
          sb[nj][0] = f.x; sb[nj][1] = f.y; sb[nj][2] = f.z; sb[nj][3] = f.w;
        }
      }
    }
  };
  auto multiply = [&](int mi, int nj) PK_INLINE {
    if constexpr (GLU) acc[mi][nj] = mma_e4m3_16(fb[nj], fa[mi & 1], acc[mi][nj]);
    else p[(mi * NJ + nj) % 3] = mma_e4m3_16(fb[nj], fa[mi & 1], f32x4_t{0.f, 0.f, 0.f, 0.f});
    __builtin_amdgcn_sched_barrier(0);
  };
  float s_tile = 0.f;
  auto add = [&](int mi, int nj) PK_INLINE {
    if constexpr (!GLU) {
      const f32x4_t& v = p[(mi * NJ + nj) % 3];
      if constexpr (TILED) {
        if (nj == 0) s_tile = sa[mi & 3] * sb[0][0];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mi][nj][e] = fmaf(v[e], s_tile, acc[mi][nj][e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mi][nj][e] = fmaf(v[e] * sb[nj][e], sa[mi & 3], acc[mi][nj][e]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto step = [&](const unsigned char* st, unsigned char* next) PK_INLINE {
    wait_and_meet<0>();
    read_a(st, 0);
    __builtin_amdgcn_sched_barrier(0);
    constexpr int LAST = MI - 1;
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) {
      multiply(LAST, nj);
      CB::read(st + CA::BYTES, wj + nj * 16 + (lane & 15), lane, fb[nj]);
      __builtin_amdgcn_sched_barrier(0);
      if (nj >= 2) add(LAST, nj - 2);
    }
    fill(next);
    add(LAST, NJ - 2);
    add(LAST, NJ - 1);
    read_sb(st);
#pragma unroll
    for (int mi = 0; mi < LAST; ++mi) {
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj) {
        multiply(mi, nj);
        if (nj == 0) {
          read_a(st, mi + 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        const int t = mi * NJ + nj - 2;
        if (t >= 0) add(t / NJ, t % NJ);
      }
    }
    add(LAST - 1, NJ - 2);
    add(LAST - 1, NJ - 1);
  };
  const int steps = (int)((g.K + STEP_K - 1) / STEP_K);
  fill(st0);
  int s = 0;
  for (; s + 2 <= steps; s += 2) {
    step(st0, st1);
    step(st1, st0);
  }
  if (s < steps) step(st0, st1);
  wait_loads<0>();  // no load may reach LDS after the workgroup has left it
#pragma unroll
  for (int nj = 0; nj < NJ; ++nj) multiply(MI - 1, nj), add(MI - 1, nj);

  // The sums leave through LDS, 64 rows of a wave's 64 columns at a time, as k_gemm's.
  __syncthreads();
  constexpr int PIECE = 64 * 256, PER = BYTES / PIECE;
  static_assert(PER * 2 >= NW, "a piece for each wave");
  unsigned char* buf = (wave < PER ? st0 : st1) + wave % PER * PIECE;
  constexpr int ROW_LANES = GLU ? 4 : 8, STEP = 64 / ROW_LANES, ROWS = 64 / STEP;
  const int rr = lane / ROW_LANES, cc = lane % ROW_LANES;
  const int j = j0 + (GLU ? wj / 2 : wj) + 8 * cc;
  typename std::conditional<GLU, GluEpilogue, Epilogue>::type epi;
  epi.init(g, j);
#pragma unroll
  for (int mp = 0; mp < MI; mp += 4) {
    const int64_t ip = i0 + wi + mp * 16 + rr;
    Raw8 res[ROWS];
    if constexpr (!GLU) {
      if (g.res && j < g.N) {
#pragma unroll
        for (int t = 0; t < ROWS; ++t)
          if (ip + STEP * t < g.M) res[t].load(g.res, (size_t)(ip + STEP * t) * g.N + j, true);
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj) {
        const f32x4_t& c = acc[mp + m][nj];
        const int row = m * 16 + (lane & 15), ch = nj * 4 + (lane >> 4);
        *reinterpret_cast<float4*>(buf + row * 256 + ((ch ^ (row & 15)) << 4)) = float4{c[0], c[1], c[2], c[3]};
      }
    if (j < g.N) {
#pragma unroll
      for (int t = 0; t < ROWS; ++t) {
        const int row = rr + STEP * t;
        const int64_t i = ip + STEP * t;
        if (i >= g.M) continue;
        auto gather = [&](int c, float (&v)[8]) PK_INLINE {
          Chunk<float>::unpack(ld16(buf + row * 256 + ((c ^ (row & 15)) << 4)), v);
          Chunk<float>::unpack(ld16(buf + row * 256 + (((c + 1) ^ (row & 15)) << 4)), v + 4);
        };
        float v[8];
        gather(2 * cc, v);
        if constexpr (GLU) {
          float u[8];
          gather(8 + 2 * cc, u);
          epi.store(g, i, j, g.a_scale ? g.a_scale[i] : 1.f, v, u);
        } else {
          epi.store(g, (size_t)i * g.N + j, 1.f, res[t], v);
        }
      }
    }
  }
}

template <int BM, int BN, int WM, int WN, int MODE>
void gemm8_launch(GemmArgs g, hipStream_t st) {
  g.tiles_m = ceil_div(g.M, BM);
  g.tiles_n = ceil_div(g.N, MODE == G_GLU ? BN / 2 : BN);
  hipLaunchKernelGGL((k_gemm8<BM, BN, WM, WN, MODE>), dim3((unsigned)(g.tiles_m * g.tiles_n)), dim3(WM * WN * 64), 0,
                     st, g);
}

}  // namespace

}  // namespace pk
