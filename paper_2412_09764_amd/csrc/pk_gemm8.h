// The large tiles of the products in blocks and of the gated part, for results that are stored
// in bf16: e4m3 codes at the 8-bit matrix instruction's rate, and bf16.
//
// What bounds them: a step of a 256-wide tile takes 1.45 us in bf16 (0.84 of it matrix cores at
// 2.4 GHz; the clock is lower) and 1.5-1.6 in codes; a tile's start and end 5 us more.
#pragma once

#include "pk_gemm.h"

namespace pk {

namespace {

constexpr int STEP_BYTES = 128;  // of k in a step; codes: one block of scales, one 16x16x128 instruction

// A step's products of two blocks of 16 rows; the lanes' k may be any, the same for both.  See
// mma_e4m3 on what the instruction of codes keeps.
template <int DT>
__device__ __forceinline__ f32x4_t mma_step(const uint4 (&b)[2], const uint4 (&a)[2], f32x4_t c) {
  if constexpr (DT == D_BF16) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b[h]), __builtin_bit_cast(bf16x8_t, a[h]),
                                                  c, 0, 0, 0);
    return c;
  } else {
    typedef __attribute__((ext_vector_type(8))) int i32x8_t;
    const i32x8_t y{(int)b[0].x, (int)b[0].y, (int)b[0].z, (int)b[0].w, (int)b[1].x, (int)b[1].y, (int)b[1].z, (int)b[1].w};
    const i32x8_t x{(int)a[0].x, (int)a[0].y, (int)a[0].z, (int)a[0].w, (int)a[1].x, (int)a[1].y, (int)a[1].z, (int)a[1].w};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(y, x, c, 0, 0, 0, 0, 0, 0);
  }
}

// Rows of 128 bytes (a step's k) in LDS; 16-byte chunk c of row r lies at slot
// c ^ ((r >> 1) & 7): the 16 lanes that LDS serves at once then read 16 different 16-byte
// columns of its 64 banks.  GLU: as Operand's.
template <int R, int NWAVE, bool GLU>
struct Codes {
  static constexpr int BYTES = R * STEP_BYTES, LOADS = BYTES / 1024 / NWAVE;
  // A load brings 8 rows.  Loads of one wave are a fixed number of rows apart, so one offset
  // serves them all; rows past the end lie past the end of the resource.
  static_assert(NWAVE == 4 || NWAVE == 8, "the same chunks in every load of a wave");
  const char* base;
  int64_t up;
  uint32_t off, row;
  int bytes;
  int left;  // bytes of k from the next step on

  __device__ static __forceinline__ int source_chunk(int wave, int lane) {
    return (lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7);
  }
  __device__ __forceinline__ void init(const void* p, int64_t row0, int64_t rows, int64_t row_bytes, bool in, int wave, int lane) {
    left = in ? (int)row_bytes : 0;
    base = (const char*)p + row0 * row_bytes;
    up = rows * row_bytes;
    row = (uint32_t)row_bytes;
    bytes = in ? (int)((rows - row0 < R ? rows - row0 : R) * row_bytes) : 0;
    off = (uint32_t)((GLU ? (wave & 3) : wave) * 8 + (lane >> 3)) * row + source_chunk(wave, lane) * 16;
    if (GLU && (wave & 4)) base += up;
  }
  // All loads of this wave of a step.  bytes counts from the step's k on, so that the last row
  // ends with the resource; where k has ended nothing is read and the slots become 0.
  __device__ __forceinline__ void load(unsigned char* lds, int wave, int lane) {
    const uint32_t room = bytes > 0 ? (uint32_t)bytes : 0u;
    const uint32_t o = left >= STEP_BYTES || source_chunk(wave, lane) * 16 < left ? off : OUTSIDE;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const bool other = GLU && NWAVE == 4 && (i & 1);  // the up projection's rows
      const uint32_t r = GLU ? (NWAVE == 4 ? i / 2 : i) * 32 : i * NWAVE * 8;
      lds_dma16_buf(raw_buffer(other ? base + up : base, room), o + r * row, 0u, lds + (i * NWAVE + wave) * 1024);
    }
    base += STEP_BYTES;
    bytes -= STEP_BYTES;
    left -= STEP_BYTES;
  }
  // Where this lane's codes of row r (its number in a block of 16 rows: lane % 16) lie: chunks
  // q and q + 4, q = lane / 16, the second one 64 bytes up or down.
  __device__ static __forceinline__ uint32_t place(int r, int lane) {
    return r * STEP_BYTES + (((lane >> 4) ^ ((r >> 1) & 7)) << 4);
  }
};

// Tiles of BM x BN by WM x WN waves with 64 columns each, two steps in LDS.  A step: the waves
// meet when its codes have landed and the step before has been read, the loads of the next one
// are issued, and each wave walks down its blocks of 16 rows, the fragments of a block read
// while the one before is multiplied.  The last block's operands stay in registers over the
// meeting, so that the matrix cores have work while the first reads return.  A workgroup
// takes tile after tile: in the last step of one the loads of the next one's first step are
// issued, and its results leave (through LDS that step has used) while they arrive.  MODE: G_GLU
// (sums in place), G_BLOCKS8 and G_BLOCKS8_TILED (a step's sums are added with their scales
// two products later).
template <int DT, int BM, int BN, int WM, int WN, int MODE>
__global__ __launch_bounds__(WM* WN * 64) void k_gemm8(const GemmArgs g) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NJ = BN / WN / 16;
  constexpr bool GLU = MODE == G_GLU, TILED = MODE == G_BLOCKS8_TILED;
  static_assert(GLU || DT == D_E4M3, "scales are of codes");
  static_assert(NJ == 4, "64 columns a wave");
  using CA = Codes<BM, NW, false>;
  using CB = Codes<BN, NW, GLU>;
  constexpr int SCALE_LOADS = GLU ? 0 : (BM + BN) / 64 / NW, SCALES_AT = CA::BYTES + CB::BYTES;
  constexpr int BYTES = SCALES_AT + (GLU ? 0 : (BM + BN) * 4);
  __shared__ __align__(1024) unsigned char st0[BYTES], st1[BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wi = (wave / WN) * (BM / WM), wj = (wave % WN) * 64;

  // Tiles in the order of k_gemm's: XCD x has a contiguous run of them, of which its
  // workgroups take one after another.
  const int tiles = g.tiles_m * g.tiles_n, x = blockIdx.x & 7, rem = tiles & 7;
  const int mine = (int)((gridDim.x - x + 7) >> 3);  // workgroups of this XCD
  const int run_end = (x + 1) * (tiles >> 3) + (x + 1 < rem ? x + 1 : rem);
  int tile = x * (tiles >> 3) + (x < rem ? x : rem) + (int)(blockIdx.x >> 3);

  CA ca;
  CB cb;
  const float* scale_at[SCALE_LOADS ? SCALE_LOADS : 1];
  int scale_step[SCALE_LOADS ? SCALE_LOADS : 1];
  int64_t i0 = 0;
  int j0 = 0;
  // What follows depends on the lane alone and would be kept over the steps, which need every
  // register: it is computed again for each tile.
  auto again = [&]() PK_INLINE {
    int l = lane;
    asm volatile("" : "+v"(l));
    return l;
  };
  // The operands of tile t; past the run's end: none.
  auto set_tile = [&](int t, int64_t& ti, int& tj) PK_INLINE {
    const int lane = again();
    const bool in = t < run_end;
    if (!in) t = 0;
    const int group = t / (4 * g.tiles_n), m_first = group * 4;
    const int m_count = g.tiles_m - m_first < 4 ? g.tiles_m - m_first : 4;
    t -= group * 4 * g.tiles_n;
    ti = (int64_t)(m_first + t % m_count) * BM;
    tj = t / m_count * (GLU ? BN / 2 : BN);
    ca.init(g.a, ti, g.M, g.K * elem_size(DT), in, wave, lane);
    cb.init(g.b, tj, g.N, g.K * elem_size(DT), in, wave, lane);
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {  // rows past the end take the last one's: their codes are 0
      const int r = (i * NW + wave) * 64 + lane;
      if (r < BM) {
        scale_at[i] = g.a_block + (ti + r < g.M ? ti + r : g.M - 1);
        scale_step[i] = (int)g.M;
      } else {
        const int j = tj + r - BM < g.N ? tj + r - BM : g.N - 1;
        scale_at[i] = g.b_block + (TILED ? j / SCALE_K : j);
        scale_step[i] = TILED ? (g.N + SCALE_K - 1) / SCALE_K : g.N;
      }
    }
  };
  auto fill = [&](unsigned char* st) PK_INLINE {
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {
      lds_dma4(scale_at[i], st + SCALES_AT + (i * NW + wave) * 256);
      if (ca.left > STEP_BYTES) scale_at[i] += scale_step[i];  // after the last block: that one again
    }
    ca.load(st, wave, lane);
    cb.load(st + CA::BYTES, wave, lane);
  };

  f32x4_t acc[MI][NJ], p[3];
  uint4 fa[2][2], fb[NJ][2];
  float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[NJ][TILED ? 1 : 4];
  const uint4 none{0, 0, 0, 0};
  // Before a tile's first step: no sums, and a last block of zeros.
  auto clear = [&]() PK_INLINE {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) {
      fb[nj][0] = fb[nj][1] = none;
#pragma unroll
      for (int e = 0; e < (TILED ? 1 : 4); ++e) sb[nj][e] = 0.f;
    }
    fa[(MI - 1) & 1][0] = fa[(MI - 1) & 1][1] = none;
    sa[(MI - 1) & 3] = 0.f;
  };

  // 16 rows are 2048 bytes and swizzled alike: one place serves all blocks of rows
  const uint32_t at_a = CA::place(wi + (lane & 15), lane), at_b = CB::place(wj + (lane & 15), lane);
  const uint32_t at_sa = SCALES_AT + (wi + (lane & 15)) * 4, at_sb = SCALES_AT + (BM + wj + (TILED ? 0 : 4 * (lane >> 4))) * 4;
  auto read_a = [&](const unsigned char* st, int mi) PK_INLINE {
    fa[mi & 1][0] = ld16(st + at_a + mi * 16 * STEP_BYTES);
    fa[mi & 1][1] = ld16(st + (at_a ^ 64) + mi * 16 * STEP_BYTES);
    if constexpr (!GLU) sa[mi & 3] = *reinterpret_cast<const float*>(st + at_sa + mi * 64);
  };
  auto read_b = [&](const unsigned char* st, int nj) PK_INLINE {
    fb[nj][0] = ld16(st + CA::BYTES + at_b + nj * 16 * STEP_BYTES);
    fb[nj][1] = ld16(st + CA::BYTES + (at_b ^ 64) + nj * 16 * STEP_BYTES);
  };
  auto read_sb = [&](const unsigned char* st) PK_INLINE {
    if constexpr (!GLU) {
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj) {
        if constexpr (TILED) {
          if (nj == 0) sb[0][0] = *reinterpret_cast<const float*>(st + at_sb);  // 64 columns of one tile
        } else {
          const float4 f = *reinterpret_cast<const float4*>(st + at_sb + nj * 64);
          sb[nj][0] = f.x; sb[nj][1] = f.y; sb[nj][2] = f.z; sb[nj][3] = f.w;
        }
      }
    }
  };
  auto multiply = [&](int mi, int nj) PK_INLINE {
    if constexpr (GLU) acc[mi][nj] = mma_step<DT>(fb[nj], fa[mi & 1], acc[mi][nj]);
    else p[(mi * NJ + nj) % 3] = mma_step<DT>(fb[nj], fa[mi & 1], f32x4_t{0.f, 0.f, 0.f, 0.f});
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
    read_a(st, 0);
    __builtin_amdgcn_sched_barrier(0);
    constexpr int LAST = MI - 1;
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) {
      multiply(LAST, nj);
      read_b(st, nj);
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
  // The results are formed where the sums lie (a lane has 4 consecutive columns of a row, the
  // gate's and the up projection's alike), rounded, and leave through LDS, 32 rows of a wave at a time,
  // so that every store covers whole cache lines.  Rows of 128 bytes (64 for GLU's y); 16-byte
  // chunk c of row r lies at slot c ^ (r / 2) (c ^ (r / 4)) modulo the chunks of a row.
  constexpr int Z_PIECE = 32 * 128, Y_ROW = GLU ? 64 : 128, Y_PIECE = 32 * Y_ROW;
  static_assert(BYTES >= NW * (Z_PIECE + Y_PIECE), "pieces for each wave");
  constexpr int ROW_LANES = Y_ROW / 16, STEP = 64 / ROW_LANES;
  constexpr int STORES = MI * 16 / STEP;  // of y, by a wave and tile
  // Loads and stores go through resources that end with the tile's rows (or are empty), so that no
  // branch hides from the compiler how many of them are under way.
  auto leave_as = [&](auto act, auto with_z, auto with_res) PK_INLINE {
    constexpr int ACT = decltype(act)::value;
    constexpr bool Z = decltype(with_z)::value, RES = decltype(with_res)::value;
    constexpr bool SCALED = GLU && DT == D_E4M3;
    const int lane = again(), il = lane & 15, q4 = 4 * (lane >> 4);
    unsigned char *zb = st1 + wave * (Z_PIECE + Y_PIECE), *yb = zb + Z_PIECE;
    const int64_t tile_rows = g.M - i0 < BM ? g.M - i0 : BM;
    const uint32_t row_y = 2u * g.N, row_z = (GLU ? 2 : 1) * row_y;
    auto rows_of = [&](const void* p, uint32_t row_bytes) PK_INLINE {
      return raw_buffer((const char*)p + (size_t)i0 * row_bytes, (uint32_t)tile_rows * row_bytes);
    };
    const auto out = rows_of(g.out, row_y), zs = rows_of(g.z, Z ? row_z : 0), rs = rows_of(g.res, RES ? row_y : 0);
    const auto sx_rows = raw_buffer(g.a_scale + (SCALED ? i0 : 0), SCALED ? (uint32_t)tile_rows * 4 : 0);
    // column block nj of this lane: GLU: 0 and 1 are the gate's, 2 and 3 the up projection's
    auto column = [&](int nj) PK_INLINE { return j0 + (GLU ? wj / 2 + (nj & 1) * 16 : wj + nj * 16) + q4; };
    float bias[NJ][4], scale[SCALED ? NJ : 1][4];
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) {
      const size_t at = (size_t)column(nj) + (GLU && nj >= 2 ? g.N : 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) bias[nj][e] = 0.f;
      if (column(nj) < g.N) {
        if (g.bias) {
          const uint2 r = *reinterpret_cast<const uint2*>((const uint16_t*)g.bias + at);
          bias[nj][0] = bf16_lo(r.x); bias[nj][1] = bf16_hi(r.x); bias[nj][2] = bf16_lo(r.y); bias[nj][3] = bf16_hi(r.y);
        }
        if constexpr (SCALED) load4(g.b_scale, at, scale[nj]);
      }
    }
    // where 8 bytes of block nj (or a half of GLU's y) of row r go
    auto slot = [&](unsigned char* p, int row_bytes, int r, int block) PK_INLINE {
      const int c = block * 2 + (lane >> 5), x = row_bytes == 128 ? (r >> 1) & 7 : (r >> 2) & 3;
      return reinterpret_cast<uint2*>(p + r * row_bytes + ((c ^ x) << 4) + ((lane >> 4) & 1) * 8);
    };
    // whole rows of 128 bytes: 8 rows an access, this lane's 16 bytes of them
    const int row8 = lane >> 3, chunk = lane & 7;
    const int jz = j0 + (GLU ? wj / 2 + 8 * (chunk & 3) : wj + 8 * chunk);
    const uint32_t oz = jz < g.N ? (wi + row8) * row_z + 2u * (jz + (GLU && chunk >= 4 ? g.N : 0)) : OUTSIDE;
    const uint32_t orow = !GLU ? oz : 0;
    // rows of y: this lane's 16 bytes
    const int rr = lane / ROW_LANES, cc = lane % ROW_LANES, jy = j0 + (GLU ? wj / 2 : wj) + 8 * cc;
    const uint32_t oy = jy < g.N ? (wi + rr) * row_y + 2u * jy : OUTSIDE;
    // What the rows of a piece bring along, loaded a piece ahead: the residual in whole cache
    // lines, turned round in y's place.
    uint4 res[4];
    float sx[2] = {1.f, 1.f};
    auto ahead = [&](int mp) PK_INLINE {
#pragma unroll
      for (int m = 0; m < 2; ++m)
        if constexpr (SCALED)
          sx[m] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sx_rows, (wi + (mp + m) * 16 + il) * 4, 0, 0));
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if constexpr (RES)
          res[t] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, orow + (mp * 16 + 8 * t) * row_y, 0, 0));
    };
    ahead(0);
#pragma unroll
    for (int mp = 0; mp < MI; mp += 2) {
      const float sx0 = sx[0], sx1 = sx[1];
      if constexpr (RES) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int r = 8 * t + row8;
          *reinterpret_cast<uint4*>(yb + r * Y_ROW + ((chunk ^ ((r >> 1) & 7)) << 4)) = res[t];
        }
      }
      if (mp + 2 < MI) ahead(mp + 2);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const int r = m * 16 + il;
        float v[NJ][4];
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[nj][e] = SCALED ? fmaf(acc[mp + m][nj][e], (m ? sx1 : sx0) * scale[SCALED ? nj : 0][e], bias[nj][e]) : acc[mp + m][nj][e] + bias[nj][e];
          if constexpr (Z) *slot(zb, 128, r, nj) = uint2{to_bf16x2(v[nj][0], v[nj][1]), to_bf16x2(v[nj][2], v[nj][3])};
        }
#pragma unroll
        for (int nj = 0; nj < (GLU ? 2 : NJ); ++nj) {
          float u[4] = {0.f, 0.f, 0.f, 0.f};
          if constexpr (RES) {
            const uint2 w = *slot(yb, Y_ROW, r, nj);
            u[0] = bf16_lo(w.x), u[1] = bf16_hi(w.x), u[2] = bf16_lo(w.y), u[3] = bf16_hi(w.y);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a = act_of<true, ACT>(v[nj][e]);
            u[e] = GLU ? a * v[(nj + 2) % NJ][e] : RES ? a + u[e] : a;
          }
          *slot(yb, Y_ROW, r, nj) = uint2{to_bf16x2(u[0], u[1]), to_bf16x2(u[2], u[3])};
        }
      }
#pragma unroll
      for (int t = 0; t < 32 / STEP; ++t) {
        const int r = rr + STEP * t, x = GLU ? (r >> 2) & 3 : (r >> 1) & 7;
        store16(out, ld16(yb + r * Y_ROW + ((cc ^ x) << 4)), oy + (mp * 16 + STEP * t) * row_y);
      }
      if constexpr (Z) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int r = row8 + 8 * t;
          store16(zs, ld16(zb + r * 128 + ((chunk ^ ((r >> 1) & 7)) << 4)), oz + (mp * 16 + 8 * t) * row_z);
        }
      }
    }
  };
  auto leave_z = [&](auto z, auto res) PK_INLINE {
    if (g.act == PKMEM_ACT_NONE) leave_as(std::integral_constant<int, PKMEM_ACT_NONE>(), z, res);
    else if (g.act == PKMEM_ACT_SILU) leave_as(std::integral_constant<int, PKMEM_ACT_SILU>(), z, res);
    else if (g.act == PKMEM_ACT_GELU) leave_as(std::integral_constant<int, PKMEM_ACT_GELU>(), z, res);
    else leave_as(std::integral_constant<int, PKMEM_ACT_RELU>(), z, res);
  };
  auto leave = [&]() PK_INLINE {
    if (g.z) {
      if (!GLU && g.res) leave_z(std::true_type(), std::bool_constant<!GLU>());
      else leave_z(std::true_type(), std::false_type());
    } else {
      if (!GLU && g.res) leave_z(std::false_type(), std::bool_constant<!GLU>());
      else leave_z(std::false_type(), std::false_type());
    }
  };

  // Steps in pairs, so that every tile starts in st0 (an odd last one gets an empty one).
  const int pairs = (int)((g.K * elem_size(DT) + 2 * STEP_BYTES - 1) / (2 * STEP_BYTES));
  set_tile(tile, i0, j0);
  fill(st0);
  bool first = true;
  while (true) {
    clear();
    // the first step's loads are older than the stores of the tile before, STORES at least, which
    // need not be waited for
    if (first) wait_and_meet<0>();
    else wait_and_meet<STORES>();
    first = false;
    step(st0, st1);
    for (int s = 1; s < pairs; ++s) {
      wait_and_meet<0>();
      step(st1, st0);
      wait_and_meet<0>();
      step(st0, st1);
    }
    int64_t next_i;
    int next_j;
    set_tile(tile + mine, next_i, next_j);
    wait_and_meet<0>();
    step(st1, st0);
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) multiply(MI - 1, nj), add(MI - 1, nj);
    // the additions stay here: the compiler would move them to where the sums are used, and spill
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj) asm volatile("" : "+v"(acc[mi][nj]));
    wait_and_meet<63>();  // st1 has been read
    leave();
    tile += mine;
    if (tile >= run_end) break;
    i0 = next_i;
    j0 = next_j;
  }
  wait_loads<0>();  // no load may reach LDS after the workgroup has left it
}

template <int DT, int BM, int BN, int WM, int WN, int MODE>
void gemm8_launch(GemmArgs g, hipStream_t st) {
  g.tiles_m = ceil_div(g.M, BM);
  g.tiles_n = ceil_div(g.N, MODE == G_GLU ? BN / 2 : BN);
  const int tiles = g.tiles_m * g.tiles_n, most = step_tile_places(BM == 256 ? TILE_256 : TILE_128);
  hipLaunchKernelGGL((k_gemm8<DT, BM, BN, WM, WN, MODE>), dim3((unsigned)(tiles < most ? tiles : most)), dim3(WM * WN * 64), 0,
                     st, g);
}

}  // namespace

}  // namespace pk
