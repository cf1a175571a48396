// Matrix products C[i, j] = sum_k A(i, k) B(j, k) on the matrix cores with their
// epilogues: the kernels of the projections, of the gated feed-forward part and of the 8-bit products in
// blocks.
#pragma once

#include <type_traits>

#include "pk_internal.h"
#include "pk_linear_plan.h"
#include "pk_mfma.h"
#include "pk_row.h"

namespace pk {

namespace {

constexpr int STAGE_K = 64;  // bytes of k per stage
constexpr uint32_t OUTSIDE = 0x80000000u;  // past the end of every buffer resource

typedef __attribute__((ext_vector_type(4))) short s16x4_t;

enum { D_F32 = 0, D_BF16 = 1, D_E4M3 = 2 };
constexpr int elem_size(int d) { return d == D_F32 ? 4 : d == D_BF16 ? 2 : 1; }

// Waits until at most VM of this wave's vector loads are outstanding and none of
// its LDS reads.
template <int VM>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | (7 << 4));
}
// The same, then the workgroup's barrier; nothing moves across.
template <int VM>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  wait_loads<VM>();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// What a kernel's product and epilogue are:
//   PLAIN  y = act(C * scales + bias) + res;
//   GLU    B has 2 N rows, a gate's N and then as many of an up projection:
//          y[i, j] = act(z[i, j]) z[i, N + j], z = C * scales + bias.
//   BLOCKS C = sum over blocks of 128 k of a_block[block, i] b_block[block, j] times the
//          sum over the block, then as PLAIN; TILED: one b_block for 128 j.  Exact products:
//          here a block's 128 k are summed for themselves and then added with their
//          scales, in k_gemm_few each 64 k.
//   BLOCKS8 the same with the 8-bit matrix instruction (see mma_e4m3): here each 64 k are
//          added with their scales, in k_gemm8 (pk_gemm8.h) each 128.
enum { G_PLAIN, G_GLU, G_BLOCKS, G_BLOCKS_TILED, G_BLOCKS8, G_BLOCKS8_TILED };
constexpr int SCALE_K = 128;  // elements along k (and j where TILED) that share a scale

struct GemmArgs {
  const void* a;  // rows i
  const void* b;  // rows j
  int64_t M;
  int N;  // GLU: of the gate (and of y)
  int64_t K;
  int64_t k_split;  // k of one split (a multiple of a stage's)
  int tiles_m, tiles_n;
  // epilogue
  const float* a_scale;
  const float* b_scale;
  const float* a_block;  // BLOCKS
  const float* b_block;
  const void* bias;
  const void* res;
  void* z;
  void* out;
  float* part;  // [splits, M, N] when the product is split
  // sums of A over k (the bias gradient, where A is dz): added to bias_sum, or, when
  // split, the parts [splits * tiles_n, M] written to it; null: none
  float* bias_sum;
  int act;
  int out_bf16;
};

__device__ __forceinline__ void mma_bf16(uint4 b, uint4 a, f32x16_t& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, b),
                                              __builtin_bit_cast(bf16x8_t, a), c, 0, 0, 0);
}
// Eight fp32 numbers as sums of three bf16 numbers each, 8 bits of mantissa at a
// time (what is left is below 2^-26 of the number).
__device__ __forceinline__ void split8(uint4 lo, uint4 hi, uint4 (&part)[3]) {
  float v[8];
  Chunk<float>::unpack(lo, v);
  Chunk<float>::unpack(hi, v + 4);
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    part[q] = Chunk<uint16_t>::pack(v);
    if (q < 2) {
      float u[8];
      Chunk<uint16_t>::unpack(part[q], u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] -= u[e];
    }
  }
}
// Of the nine products of two numbers in three parts, the six above 2^-24 of the
// whole, smallest first: the parts of b and of a.
constexpr int SPLIT_B[6] = {2, 0, 1, 1, 0, 0}, SPLIT_A[6] = {0, 2, 1, 0, 1, 0};
__device__ __forceinline__ uint32_t word(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
// 8 e4m3 codes as bf16 (exact).  The 8-bit matrix instructions align the products
// of each 8 k to the largest of them and keep 13 bits below it; a sum in fp32 takes
// the bf16 instruction.  (Measured: beside a product of 2^16 one of 2^2 is lost.)
__device__ __forceinline__ uint4 widen8(uint32_t lo, uint32_t hi) {
  return uint4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true))};
}

// 64 k of codes at once: twice the rate of the widened form, for results that are rounded to
// bf16.  The instruction aligns the products of each 8 k to the largest of them and keeps 13
// bits below it, so each is within 2^-13 of that largest one, a sum therefore within 2^-10 of the
// sum of its sizes; the groups are added in 24 bits.  On random codes it is 2^-18 of the sum of
// sizes: of 2000 x 4096 results of 2048 k (a norm's output, a weight) 1.4% are then the bf16
// number beside the nearest one, of an fp32 product of the numbers that the codes stand for 0.06%,
// and both are 1.7e-3 off the unrounded sums (rms, relative).
__device__ __forceinline__ f32x16_t mma_e4m3(uint4 b0, uint4 b1, uint4 a0, uint4 a1) {
  typedef __attribute__((ext_vector_type(8))) int i32x8_t;
  const i32x8_t b{(int)b0.x, (int)b0.y, (int)b0.z, (int)b0.w, (int)b1.x, (int)b1.y, (int)b1.z, (int)b1.w};
  const i32x8_t a{(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, f32x16_t{}, 0, 0, 0, 0, 0, 0);
}

// An operand's tile: R rows by one stage of k.
//   KS = false: LDS [R][64 bytes of k]; 16-byte chunk c of row r lies at slot
//     c ^ ((r >> 2) & 3): the 16 lanes that LDS serves at once (lanes 0-3, 12-15,
//     20-27 and so on) then read 16 different 16-byte columns of its 64 banks.
//   KS = true: LDS [k][R elements]; the 64-byte (bf16) or 128-byte (fp32) units
//     of a k row are permuted by k so that the k rows of one read instruction
//     lie in different banks.
//   GLU: blocks of 32 rows are the gate's and the up projection's in turn.
template <int DT, bool KS, int R, int NWAVE, bool GLU = false>
struct Operand {
  static constexpr int E = elem_size(DT);
  static constexpr int BYTES = R * STAGE_K;
  static constexpr int ROW = KS ? R * E : STAGE_K;    // bytes of an LDS row
  static constexpr int LOADS = BYTES / 1024 / NWAVE;  // direct loads per wave and stage
  static constexpr int STAGE_ROWS = STAGE_K / E;      // k of a stage
  static_assert(BYTES % (1024 * NWAVE) == 0, "whole loads");
  static constexpr int UNITS = ROW / 64;

  uint32_t off[LOADS];  // this lane's source offsets in a stage; OUTSIDE: no such row
  uint32_t rd[R / 32 < 8 ? R / 32 : 8];
  const char* base;     // of the next stage
  int64_t step;         // bytes from stage to stage
  int64_t up;           // GLU: bytes from the gate's rows to the up projection's
  int whole;            // stages left that lie within k

  // rows: first row of the tile, of `rows`; k range [k0, k1) of ld = K (or rows) elements
  __device__ __forceinline__ void init(const void* p, int64_t row0, int64_t rows, int64_t K,
                                       int64_t k0, int64_t k1, int wave, int lane) {
    whole = k1 > k0 ? (int)((k1 - k0) / STAGE_ROWS) : 0;
    const int64_t ld = (KS ? rows : K) * E;
    base = (const char*)p + (KS ? k0 * ld + row0 * E : row0 * ld + k0 * E);
    step = KS ? (int64_t)STAGE_ROWS * ld : STAGE_K;
    up = rows * ld;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int slot = (i * NWAVE + wave) * 64 + lane;
      if constexpr (!KS) {
        const int r = GLU ? ((slot >> 8) << 5) | ((slot >> 2) & 31) : slot >> 2;
        off[i] = row0 + r < rows ? (uint32_t)(r * ld + source_chunk(slot) * 16) : OUTSIDE;
      } else {
        const int k = slot / (ROW / 16), c = source_chunk(slot);
        off[i] = row0 + c * (16 / E) < rows ? (uint32_t)(k * ld + c * 16) : OUTSIDE;
      }
    }
  }
  // The 16-byte chunk of its row that a slot of the stage holds.
  __device__ static __forceinline__ int source_chunk(int slot) {
    if constexpr (!KS) return (slot & 3) ^ ((slot >> 4) & 3);
    const int k = slot / (ROW / 16), c = slot % (ROW / 16);
    if constexpr (DT == D_F32) return UNITS >= 4 ? c ^ (((k >> 2) & 1) << 3) : c;
    return c ^ ((((k & 3) | ((k >> 1) & 4)) & (UNITS - 1)) << 2);
  }
  // Load i of this wave of the next stage into lds; `left`: k of the range from
  // that stage on (0 or less: nothing is read, the slots become 0).
  __device__ __forceinline__ void load(int i, unsigned char* lds, int wave, int lane, int left) const {
    uint32_t o = off[i];
    if (whole <= 0) {  // the end of k lies in this stage, or before it
      const int slot = (i * NWAVE + wave) * 64 + lane;
      const int k = KS ? slot / (ROW / 16) : source_chunk(slot) * (16 / E);
      o = k < left ? o : OUTSIDE;
    }
    const char* from = base;
    if constexpr (GLU) {  // the 16 rows of a load lie in one block of 32
      if ((i * NWAVE + wave) & 2) from += up;
    }
    lds_dma16_buf(raw_buffer(from, 0x7FFFFFFFu), o, 0u, lds + (i * NWAVE + wave) * 1024);
  }
  __device__ __forceinline__ void advance() {
    base += step;
    --whole;
  }
  // KS: adds the stage's k to sums of 16 bytes of rows each, for this thread of
  // THREADS that share the stage: rows chunk t % CHUNKS, k from t / CHUNKS on.
  static constexpr int CHUNKS = ROW / 16, THREADS = NWAVE * 64, K_GROUPS = THREADS / CHUNKS;
  __device__ __forceinline__ void add_rows(const unsigned char* lds, int t, float (&sum)[16 / E]) const {
    const int c = t % CHUNKS;
#pragma unroll
    for (int k = t / CHUNKS, u = 0; u < STAGE_ROWS / K_GROUPS; ++u, k += K_GROUPS) {
      // source_chunk is its own inverse within a row
      const uint4 v = ld16(lds + k * ROW + source_chunk(k * CHUNKS + c) % CHUNKS * 16);
      float f[16 / E];
      if constexpr (DT == D_F32) Chunk<float>::unpack(v, f);
      else Chunk<uint16_t>::unpack(v, f);
#pragma unroll
      for (int e = 0; e < 16 / E; ++e) sum[e] += f[e];
    }
  }
  // Read addresses of this lane for blocks of 32 rows from row r0 on.
  template <int NB>
  __device__ __forceinline__ void init_read(int r0, int lane) {
    if constexpr (!KS) {
      const int r = r0 + (lane & 31);
      rd[0] = r * STAGE_K + (((lane >> 5) ^ ((r >> 2) & 3)) << 4);
    } else if constexpr (DT == D_F32) {
      const int kh = lane >> 5;
#pragma unroll
      for (int b = 0; b < NB; ++b)
        rd[b] = 4 * kh * ROW + (((r0 / 32 + b) ^ (UNITS >= 4 ? kh : 0)) * 128) + (lane & 31) * 4;
    } else {
      const int g = lane >> 4, i = lane & 15;
      const int f = ((i >> 2) | ((g >> 1) << 2)) & (UNITS - 1);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        rd[b] = (8 * (g >> 1) + (i >> 2)) * ROW + (((r0 / 32 + b) ^ f) * 64) + 32 * (g & 1) + 8 * (i & 3);
    }
  }
  // Fragment of block b, half h of the stage (32 bytes of k).
  __device__ __forceinline__ uint4 frag(const unsigned char* lds, int b, int h) const {
    if constexpr (!KS) {
      return *reinterpret_cast<const uint4*>(lds + ((rd[0] ^ (h << 5)) + b * 32 * STAGE_K));
    } else if constexpr (DT == D_F32) {
      const unsigned char* p = lds + rd[b] + h * 8 * ROW;
      return uint4{*reinterpret_cast<const uint32_t*>(p), *reinterpret_cast<const uint32_t*>(p + ROW),
                   *reinterpret_cast<const uint32_t*>(p + 2 * ROW),
                   *reinterpret_cast<const uint32_t*>(p + 3 * ROW)};
    } else {
      const unsigned char* p = lds + rd[b] + h * 16 * ROW;
      typedef __attribute__((address_space(3))) s16x4_t* lp;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(unsigned char*)p);
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(unsigned char*)(p + 4 * ROW));
      const uint2 l = __builtin_bit_cast(uint2, lo), u = __builtin_bit_cast(uint2, hi);
      return uint4{l.x, l.y, u.x, u.y};
    }
  }
};

// ---- activations -------------------------------------------------------------
// FAST: for values that are rounded to bf16 afterwards.
template <bool FAST>
__device__ __forceinline__ float sigmoid_of(float z) {
  if constexpr (FAST) return __builtin_amdgcn_rcpf(1.f + __expf(-z));
  return 1.f / (1.f + expf(-z));
}
// The normal distribution's tail Q(|z|) = erfc(|z| / sqrt 2) / 2, and e = exp(-z^2 / 2).
// For negative z it is the factor of z in GELU by itself: 1 + erf would cancel.
// Q = e times a polynomial in t = 1 / (1 + p |z|) without a constant term, fitted to
// exp(a^2) erfc(a) for 0 <= a <= 10 with the least largest relative error: 5 terms
// 3.2e-5 (FAST), 9 terms 2e-8 (7 units of 2^-24 as evaluated; the library's erfcf took
// 4096 x 2048 through the activation's backward in 23.4 us, this 18.8).
template <bool FAST>
__device__ __forceinline__ float tail_of(float z, float& e) {
  if constexpr (!FAST) {
    e = expf(-0.5f * z * z);
    const float t = 1.f / fmaf(0.212132037f, fabsf(z), 1.f);
    return e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0647613257f, 0.242780983f), -0.256137729f), 0.273858458f), -0.0473242477f), 0.107462533f), 0.0741697177f), 0.0853575915f), 0.0845940039f);
  } else {
    e = __expf(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.374766594f, fabsf(z), 1.f));
    return e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.090499118f, 0.20043318f), 0.0834558904f), 0.157641605f), 0.148969173f);
  }
}
template <bool FAST, int ACT>
__device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == PKMEM_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if constexpr (ACT == PKMEM_ACT_SILU) return FAST ? z * sigmoid_of<true>(z) : z / (1.f + expf(-z));
  if constexpr (ACT == PKMEM_ACT_GELU) {
    float e;
    const float q = tail_of<FAST>(z, e);
    return z * (z < 0.f ? q : 1.f - q);
  }
  return z;
}
template <bool FAST, int ACT>
__device__ __forceinline__ float act_grad_of(float z) {
  if constexpr (ACT == PKMEM_ACT_RELU) return z > 0.f ? 1.f : (z != z ? z : 0.f);
  if constexpr (ACT == PKMEM_ACT_SILU) {
    const float s = sigmoid_of<FAST>(z);
    return s * (1.f + z * (1.f - s));
  }
  if constexpr (ACT == PKMEM_ACT_GELU) {
    float e;
    const float q = tail_of<FAST>(z, e);
    return (z < 0.f ? q : 1.f - q) + z * e * 0.39894228040143268f;
  }
  return 1.f;
}
template <bool FAST, int N>
__device__ __forceinline__ void apply_act(float (&v)[N], int act) {
#define PK_ACT(A)                                             \
  case A: {                                                   \
    _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] = act_of<FAST, A>(v[e]); \
    break;                                                    \
  }
  switch (act) {
    PK_ACT(PKMEM_ACT_RELU)
    PK_ACT(PKMEM_ACT_SILU)
    PK_ACT(PKMEM_ACT_GELU)
    default: break;
  }
#undef PK_ACT
}

__device__ __forceinline__ void load4(const float* p, size_t at, float (&v)[4]) {
  const float4 f = *reinterpret_cast<const float4*>(p + at);
  v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
}
__device__ __forceinline__ void store4(float* p, size_t at, const float (&v)[4]) {
  *reinterpret_cast<float4*>(p + at) = float4{v[0], v[1], v[2], v[3]};
}
// Eight consecutive elements of a bf16 or fp32 array, as stored.
struct Raw8 {
  uint4 lo, hi;  // bf16: lo
  __device__ __forceinline__ void load(const void* p, size_t at, bool bf16) {
    if (bf16) {
      lo = ld16((const uint16_t*)p + at);
    } else {
      lo = ld16((const float*)p + at);
      hi = ld16((const float*)p + at + 4);
    }
  }
  __device__ __forceinline__ void unpack(bool bf16, float (&v)[8]) const {
    if (bf16) {
      Chunk<uint16_t>::unpack(lo, v);
    } else {
      Chunk<float>::unpack(lo, v);
      Chunk<float>::unpack(hi, v + 4);
    }
  }
};
__device__ __forceinline__ void store8(void* p, size_t at, bool bf16, const float (&v)[8]) {
  if (bf16) {
    *reinterpret_cast<uint4*>((uint16_t*)p + at) = Chunk<uint16_t>::pack(v);
  } else {
    *reinterpret_cast<uint4*>((float*)p + at) = Chunk<float>::pack(v);
    *reinterpret_cast<uint4*>((float*)p + at + 4) = Chunk<float>::pack(v + 4);
  }
}

// The epilogue of 8 columns (from j on, the same for every row a lane handles):
// scales, bias, activation and residual in fp32, one rounding.
struct Epilogue {
  float scale[8], bias[8];
  __device__ __forceinline__ void init(const GemmArgs& g, int j) {
    if (j >= g.N) return;
    if (g.b_scale) {
      Raw8 r;
      r.load(g.b_scale, j, false);
      r.unpack(false, scale);
    }
    if (g.bias) {
      Raw8 r;
      r.load(g.bias, j, g.out_bf16);
      r.unpack(g.out_bf16, bias);
    }
  }
  __device__ __forceinline__ void store(const GemmArgs& g, size_t at, float sa, const Raw8& res,
                                        float (&v)[8]) const {
    const bool h = g.out_bf16;
    if (g.b_scale) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= sa * scale[e];
    }
    if (g.bias) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += bias[e];
    }
    if (g.z) store8(g.z, at, h, v);
    if (h) apply_act<true>(v, g.act);
    else apply_act<false>(v, g.act);
    if (g.res) {
      float r[8];
      res.unpack(h, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    store8(g.out, at, h, v);
  }
};

// The same for 8 columns of a gated product.
struct GluEpilogue {
  float scale[2][8], bias[2][8];
  __device__ __forceinline__ void init(const GemmArgs& g, int j) {
    if (j >= g.N) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      Raw8 r;
      if (g.b_scale) {
        r.load(g.b_scale, (size_t)u * g.N + j, false);
        r.unpack(false, scale[u]);
      }
      if (g.bias) {
        r.load(g.bias, (size_t)u * g.N + j, g.out_bf16);
        r.unpack(g.out_bf16, bias[u]);
      }
    }
  }
  __device__ __forceinline__ void store(const GemmArgs& g, int64_t i, int j, float sa, float (&gate)[8],
                                        float (&up)[8]) const {
    const bool h = g.out_bf16;
    if (g.b_scale) {
#pragma unroll
      for (int e = 0; e < 8; ++e) gate[e] *= sa * scale[0][e], up[e] *= sa * scale[1][e];
    }
    if (g.bias) {
#pragma unroll
      for (int e = 0; e < 8; ++e) gate[e] += bias[0][e], up[e] += bias[1][e];
    }
    if (g.z) {
      const size_t at = (size_t)i * 2 * g.N + j;
      store8(g.z, at, h, gate);
      store8(g.z, at + g.N, h, up);
    }
    if (h) apply_act<true>(gate, g.act);
    else apply_act<false>(gate, g.act);
#pragma unroll
    for (int e = 0; e < 8; ++e) gate[e] *= up[e];
    store8(g.out, (size_t)i * g.N + j, h, gate);
  }
};

// KG groups of waves share the tile's k.  GRAD: C is added to fp32 `out`, or written to `part` when split; else the
// epilogue above.
template <int DT, bool AKS, bool BKS, bool GRAD, int BM, int BN, int WM, int WN, int KG, int MODE = G_PLAIN>
__global__ __launch_bounds__(WM* WN* KG * 64) void k_gemm(const GemmArgs g) {
  constexpr int NW = WM * WN, MI = BM / WM / 32, NJ = BN / WN / 32;
  constexpr bool GLU = MODE == G_GLU, BLOCKS = MODE >= G_BLOCKS, BLOCKS8 = MODE >= G_BLOCKS8;
  constexpr bool TILED = MODE == G_BLOCKS_TILED || MODE == G_BLOCKS8_TILED;
  static_assert(!BLOCKS || (DT == D_E4M3 && !AKS && !BKS && !GRAD), "codes with k consecutive");
  static_assert(!GLU || (NJ == 2 && !BKS && !GRAD), "a wave holds a gate's block of columns and the up projection's");
  using OA = Operand<DT, AKS, BM, NW>;
  using OB = Operand<DT, BKS, BN, NW, GLU>;
  // BLOCKS: a stage holds the scales of its rows too, A's first
  constexpr int SCALE_LOADS = BLOCKS ? (BM + BN) / 64 / NW : 0, SCALES_AT = OA::BYTES + OB::BYTES;
  constexpr int L = OA::LOADS + OB::LOADS + SCALE_LOADS;
  constexpr int GROUP_BYTES = SCALES_AT + (BLOCKS ? (BM + BN) * 4 : 0), BYTES = KG * GROUP_BYTES;
  // a variable for each stage: the compiler then knows which loads a read of
  // LDS depends on, and waits for no other
  __shared__ __align__(1024) unsigned char st0[BYTES], st1[BYTES], st2[BYTES], st3[BYTES];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = w % NW, kg = w / NW;

  // XCD x (workgroup number mod 8) takes a contiguous run of tiles; within it
  // four rows of tiles at a time, so that what one XCD's L2 holds is shared.
  const int tiles = g.tiles_m * g.tiles_n, nwg = gridDim.x;
  const int x = blockIdx.x & 7, q = nwg >> 3, rem = nwg & 7;
  int pid = x * q + (x < rem ? x : rem) + (blockIdx.x >> 3);
  const int split = pid / tiles;
  pid -= split * tiles;
  const int group = pid / (4 * g.tiles_n);
  const int m_first = group * 4;
  const int m_count = g.tiles_m - m_first < 4 ? g.tiles_m - m_first : 4;
  pid -= group * 4 * g.tiles_n;
  const int64_t i0 = (int64_t)(m_first + pid % m_count) * BM;
  const int tile_n = pid / m_count, j0 = tile_n * (GLU ? BN / 2 : BN);
  int64_t k0 = split * g.k_split;
  int64_t k1 = k0 + g.k_split < g.K ? k0 + g.k_split : g.K;
  // this group's share of k; all groups take the same number of steps
  int steps = (int)((k1 - k0 + KG * OA::STAGE_ROWS - 1) / (KG * OA::STAGE_ROWS));
  // BLOCKS: two stages are a block of scales, whose sums are held over both of them; an odd
  // last stage gets an empty one.
  constexpr bool HOLD = BLOCKS && !BLOCKS8;
  static_assert(!HOLD || (MI * NJ <= 4 && 2 * OA::STAGE_ROWS == SCALE_K), "registers for two sets of sums");
  if constexpr (HOLD) steps += steps & 1;
  if constexpr (KG > 1) {
    k0 += (int64_t)kg * steps * OA::STAGE_ROWS;
    const int64_t end = k0 + (int64_t)steps * OA::STAGE_ROWS;
    k1 = end < k1 ? end : k1;
  }

  OA oa;
  OB ob;
  oa.init(g.a, i0, g.M, g.K, k0, k1, wave, lane);
  ob.init(g.b, j0, g.N, g.K, k0, k1, wave, lane);
  const int wi = (wave / WN) * (BM / WM), wj = (wave % WN) * (BN / WN);
  oa.template init_read<MI>(wi, lane);
  ob.template init_read<NJ>(wj, lane);

  const float* scale_at[SCALE_LOADS ? SCALE_LOADS : 1];
  int scale_step[SCALE_LOADS ? SCALE_LOADS : 1];  // from block to block
  int64_t scale_k = k0;
  if constexpr (BLOCKS) {  // rows past the end take the last one's: their codes are 0
#pragma unroll
    for (int i = 0; i < SCALE_LOADS; ++i) {
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
  }

  f32x16_t acc[MI][NJ];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x16_t{};

  const int group_at = KG > 1 ? kg * GROUP_BYTES : 0;
  int left = k1 > k0 ? (int)(k1 - k0 < 0x7FFFFFFF ? k1 - k0 : 0x7FFFFFFF) : 0;
  // Load i of a stage (A's first), and the step to the next one.
  auto load = [&](unsigned char* st, int i) PK_INLINE {
    if (i < OA::LOADS) {
      oa.load(i, st + group_at, wave, lane, left);
    } else if (i < OA::LOADS + OB::LOADS) {
      ob.load(i - OA::LOADS, st + group_at + OA::BYTES, wave, lane, left);
    } else if constexpr (BLOCKS) {
      const int u = i - OA::LOADS - OB::LOADS;
      const int block = (int)((scale_k < g.K ? scale_k : g.K - 1) / SCALE_K);
      lds_dma4(scale_at[u] + (size_t)block * scale_step[u], st + group_at + SCALES_AT + (u * NW + wave) * 256);
    }
  };
  auto advance = [&]() PK_INLINE {
    oa.advance();
    ob.advance();
    left -= OA::STAGE_ROWS;
    scale_k += OA::STAGE_ROWS;
  };
  auto fill = [&](unsigned char* st) PK_INLINE {
#pragma unroll
    for (int i = 0; i < L; ++i) load(st, i);
    advance();
  };
  // Fragments of the halves 0 and 1 of a stage; in fp32 and blocks where every wave
  // multiplies all the time, of two stages in turn.
  constexpr bool TURNS = NW * KG == 8;
  constexpr int SETS = (DT == D_F32 || BLOCKS) && !TURNS ? 2 : 1;
  uint4 fa[SETS][2][MI], fb[SETS][2][NJ];
  constexpr int SJ = TILED ? 1 : 16;  // scales of a block of columns: the lane's 16 rows of the result
  float scale_a[BLOCKS ? SETS : 1][MI], scale_b[BLOCKS ? SETS : 1][NJ][SJ];
  auto read = [&](const unsigned char* st, int h, int set = 0) PK_INLINE {
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) fb[set][h][nj] = ob.frag(st + group_at + OA::BYTES, nj, h);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) fa[set][h][mi] = oa.frag(st + group_at, mi, h);
    if constexpr (BLOCKS) {
      if (h == 0) {
        const float* sc = reinterpret_cast<const float*>(st + group_at + SCALES_AT);
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) scale_a[set][mi] = sc[wi + mi * 32 + (lane & 31)];
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
          for (int e = 0; e < SJ; e += 4) {
            const float* p = sc + BM + wj + nj * 32;
            if constexpr (TILED) {
              scale_b[set][nj][0] = *p;
            } else {
              const float4 f = *reinterpret_cast<const float4*>(p + 2 * e + 4 * (lane >> 5));
              scale_b[set][nj][e] = f.x; scale_b[set][nj][e + 1] = f.y;
              scale_b[set][nj][e + 2] = f.z; scale_b[set][nj][e + 3] = f.w;
            }
          }
      }
    }
  };
  // bf16, e4m3: the products of half h, in MI or 2 MI groups; between them, where
  // asked for, the loads of a stage into st.
  auto products = [&](int h, bool refill, unsigned char* st) PK_INLINE {
    constexpr int GROUPS = DT == D_E4M3 ? 2 * MI : MI;
    uint4 b[NJ];
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
      const int mi = q % MI;
      if constexpr (DT == D_E4M3) {
        if (mi == 0) {
#pragma unroll
          for (int nj = 0; nj < NJ; ++nj)
            b[nj] = q ? widen8(fb[0][h][nj].z, fb[0][h][nj].w) : widen8(fb[0][h][nj].x, fb[0][h][nj].y);
        }
        const uint4 a = q >= MI ? widen8(fa[0][h][mi].z, fa[0][h][mi].w) : widen8(fa[0][h][mi].x, fa[0][h][mi].y);
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj) mma_bf16(b[nj], a, acc[mi][nj]);
      } else {
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj) mma_bf16(fb[0][h][nj], fa[0][h][mi], acc[mi][nj]);
      }
      if (refill) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = q * L / GROUPS; i < (q + 1) * L / GROUPS; ++i) load(st, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  // fp32: the products of a whole stage, six bf16 ones for each.  (The fp32 matrix
  // instructions take 2.7 times their cycles.)
  auto products_f32 = [&](int set) PK_INLINE {
    uint4 b[NJ][3];
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) split8(fb[set][0][nj], fb[set][1][nj], b[nj]);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      uint4 a[3];
      split8(fa[set][0][mi], fa[set][1][mi], a);
#pragma unroll
      for (int t = 0; t < 6; ++t)
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj) mma_bf16(b[nj][SPLIT_B[t]], a[SPLIT_A[t]], acc[mi][nj]);
    }
  };
  // blocks: a stage's (HOLD: a block's) sums, then their addition with the scales, a tile behind
  // them so that it runs while the matrix cores form the next sums.
  f32x16_t held[HOLD ? MI * NJ : 1];
  auto products_blocks = [&](int set, bool second) PK_INLINE {
    uint4 b[NJ][4];
    if constexpr (!BLOCKS8) {
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 f = fb[set][q >> 1][nj];
          b[nj][q] = q & 1 ? widen8(f.z, f.w) : widen8(f.x, f.y);
        }
    }
    auto add = [&](const f32x16_t& p, int t) PK_INLINE {
      const int mi = t / NJ, nj = t % NJ;
      if constexpr (TILED) {
        const float s = scale_a[set][mi] * scale_b[set][nj][0];
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[mi][nj][e] = fmaf(p[e], s, acc[mi][nj][e]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[mi][nj][e] = fmaf(p[e] * scale_b[set][nj][e], scale_a[set][mi], acc[mi][nj][e]);
      }
    };
    if constexpr (BLOCKS8) {
      f32x16_t p[2];
#pragma unroll
      for (int t = 0; t < MI * NJ; ++t) {
        const int mi = t / NJ, nj = t % NJ;
        p[t & 1] = mma_e4m3(fb[set][0][nj], fb[set][1][nj], fa[set][0][mi], fa[set][1][mi]);
        __builtin_amdgcn_sched_barrier(0);  // or one set of registers would do, and wait
        if (t > 0) add(p[(t - 1) & 1], t - 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      add(p[(MI * NJ - 1) & 1], MI * NJ - 1);
    } else {
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        uint4 a[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 f = fa[set][q >> 1][mi];
          a[q] = q & 1 ? widen8(f.z, f.w) : widen8(f.x, f.y);
        }
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj)
          if (!second) held[mi * NJ + nj] = f32x16_t{};
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int nj = 0; nj < NJ; ++nj) mma_bf16(b[nj][q], a[q], held[mi * NJ + nj]);
        if (second && mi > 0) {
#pragma unroll
          for (int nj = 0; nj < NJ; ++nj) add(held[(mi - 1) * NJ + nj], (mi - 1) * NJ + nj);
        }
      }
      if (second) {
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj) add(held[(MI - 1) * NJ + nj], (MI - 1) * NJ + nj);
      }
    }
  };
  // The sums over A's k: when split, the tiles along j take the stages in turn, else
  // the first of them takes all.
  constexpr int BIAS = AKS ? 16 / OA::E : 1;
  float bias[BIAS];
#pragma unroll
  for (int e = 0; e < BIAS; ++e) bias[e] = 0.f;
  int bias_turn = !AKS || !g.bias_sum || (!g.part && tile_n > 0) ? -1 : g.part ? tile_n : 0;
  const int bias_every = g.part ? g.tiles_n : 1;
  auto add_bias = [&](const unsigned char* st) PK_INLINE {
    if constexpr (AKS) {
      if (bias_turn == 0) {
        oa.add_rows(st + group_at, wave * 64 + lane, bias);
        bias_turn = bias_every;
      }
      if (bias_turn > 0) --bias_turn;
    }
  };
  if constexpr (TURNS) {
    // Two waves share a SIMD, one of the first four and one of the last: while one
    // of them multiplies a stage the other reads its next one and issues the loads,
    // and they change places at a barrier, so the matrix cores always have a
    // wave with all its operands in registers (against all waves reading and
    // multiplying at once: 8192^3 878 -> 860 us, 2000 x 2048 x 2048 in e4m3 20 -> 18).
    // Stage s: the first four multiply, the last four read it; then the first
    // four read stage s + 1 and refill s.
    auto multiply = [&](bool second) PK_INLINE {
      __builtin_amdgcn_s_setprio(1);
      if constexpr (DT == D_F32) {
        products_f32(0);
      } else if constexpr (BLOCKS) {
        products_blocks(0, second);
      } else {
        products(0, false, st0);
        products(1, false, st0);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    auto read_all = [&](const unsigned char* st) PK_INLINE {
      read(st, 0);
      read(st, 1);
      add_bias(st);
    };
    auto first = [&](unsigned char* st, const unsigned char* next, bool second = false) PK_INLINE {
      multiply(second);
      wait_and_meet<2 * L>();  // the next stage has landed
      read_all(next);
      fill(st);
      wait_and_meet<63>();  // 63: for LDS alone
    };
    auto last = [&](unsigned char* st, unsigned char* before, bool second = false) PK_INLINE {
      read_all(st);
      fill(before);
      wait_and_meet<2 * L>();
      multiply(second);
      wait_and_meet<63>();
    };
    fill(st0);
    fill(st1);
    fill(st2);
    int s = 0;
    if (w < 4) {
      fill(st3);
      wait_and_meet<3 * L>();
      read_all(st0);
      for (; s + 4 <= steps; s += 4) {
        first(st0, st1);
        first(st1, st2, true);
        first(st2, st3);
        first(st3, st0, true);
      }
      if (s < steps) first(st0, st1);
      if (s + 1 < steps) first(st1, st2, true);
      if (s + 2 < steps) first(st2, st3);
    } else {
      wait_and_meet<2 * L>();
      for (; s + 4 <= steps; s += 4) {
        last(st0, st3);
        last(st1, st0, true);
        last(st2, st1);
        last(st3, st2, true);
      }
      if (s < steps) last(st0, st3);
      if (s + 1 < steps) last(st1, st0, true);
      if (s + 2 < steps) last(st2, st1);
    }
  } else if constexpr (DT == D_F32 || BLOCKS) {
    // One stage: it is in the registers of set; next has landed for all after the
    // barrier, and is read while the products run.
    auto stage = [&](int set, unsigned char* st, const unsigned char* next) PK_INLINE {  // set: the stage's parity
      wait_and_meet<2 * L>();
      read(next, 0, set ^ 1);
      read(next, 1, set ^ 1);
      __builtin_amdgcn_sched_barrier(0);
      add_bias(next);
      fill(st);
      if constexpr (BLOCKS) products_blocks(set, set == 1);
      else products_f32(set);
    };
    fill(st0);
    fill(st1);
    fill(st2);
    fill(st3);
    wait_and_meet<3 * L>();
    read(st0, 0, 0);
    read(st0, 1, 0);
    add_bias(st0);
    int s = 0;
    for (; s + 4 <= steps; s += 4) {
      stage(0, st0, st1);
      stage(1, st1, st2);
      stage(0, st2, st3);
      stage(1, st3, st0);
    }
    if (s < steps) stage(0, st0, st1);
    if (s + 1 < steps) stage(1, st1, st2);
    if (s + 2 < steps) stage(0, st2, st3);
  } else {
    // One stage: st is visible to all, half 0 of it in registers.  After the
    // barrier every wave has read st, and next has landed for all.  The reads of
    // a half are issued before the products of the half before it and return
    // while these run.
    auto stage = [&](unsigned char* st, const unsigned char* next) PK_INLINE {
      read(st, 1);
      __builtin_amdgcn_sched_barrier(0);
      products(0, false, st);
      add_bias(st);
      wait_and_meet<2 * L>();
      read(next, 0);
      __builtin_amdgcn_sched_barrier(0);
      products(1, true, st);
      advance();
    };
    fill(st0);
    fill(st1);
    fill(st2);
    fill(st3);
    wait_and_meet<3 * L>();
    read(st0, 0);
    int s = 0;
    for (; s + 4 <= steps; s += 4) {
      stage(st0, st1);
      stage(st1, st2);
      stage(st2, st3);
      stage(st3, st0);
    }
    if (s < steps) stage(st0, st1);
    if (s + 1 < steps) stage(st1, st2);
    if (s + 2 < steps) stage(st2, st3);
  }
  wait_loads<0>();  // no load may reach LDS after the workgroup has left it

  // The sums leave through LDS, 64 rows of a wave's 64 columns at a time (16 KiB a
  // wave; 32 of 32 in the smallest tiles), so that eight lanes hold a row's 64
  // columns: every load and store of the epilogue covers whole cache lines.
  // 16-byte chunk c of row r lies at slot c ^ (r mod the chunks of a row).  The
  // waves of the groups of k that share a piece add its parts in group order,
  // each for its share of the rows.
  __syncthreads();
  constexpr int MP = MI < 2 ? MI : 2;             // blocks of rows of a piece
  constexpr int ROW_BYTES = NJ * 128, CH = ROW_BYTES / 16;
  constexpr int PIECE = MP * 32 * ROW_BYTES, WAVES_PER_STAGE = BYTES / PIECE;
  constexpr int ROW_LANES = GLU ? 4 : NJ * 4, STEP = 64 / ROW_LANES;  // lanes of a row, rows of an access
  constexpr int ACCESSES = MP * 32 / STEP, ROWS = ACCESSES < KG ? 1 : ACCESSES / KG;
  static_assert(MI % MP == 0 && WAVES_PER_STAGE >= 1 && WAVES_PER_STAGE * 4 >= NW * KG, "pieces fit the stages");
  auto piece = [&](int q) PK_INLINE {
    const int v = q * NW + wave, si = v / WAVES_PER_STAGE;
    return (si == 0 ? st0 : si == 1 ? st1 : si == 2 ? st2 : st3) + (v % WAVES_PER_STAGE) * PIECE;
  };
  if constexpr (AKS) {
    if (g.bias_sum && (g.part || tile_n == 0)) {  // the threads' sums in the order of their k
      float* all = reinterpret_cast<float*>(st0);
      constexpr int GROUPS = KG * OA::K_GROUPS;
      static_assert(GROUPS * BM * 4 <= BYTES, "the sums of a workgroup fit a stage");
      const int t = wave * 64 + lane, at = (kg * OA::K_GROUPS + t / OA::CHUNKS) * BM + t % OA::CHUNKS * BIAS;
#pragma unroll
      for (int e = 0; e < BIAS; ++e) all[at + e] = bias[e];
      __syncthreads();
      const int r = threadIdx.x;
      if (r < BM && i0 + r < g.M) {
        float v = 0.f;
        for (int q = 0; q < GROUPS; ++q) v += all[q * BM + r];
        if (g.part) g.bias_sum[(size_t)(split * g.tiles_n + tile_n) * g.M + i0 + r] = v;
        else g.bias_sum[i0 + r] += v;
      }
      __syncthreads();
    }
  }
  unsigned char* buf = piece(kg);
  const int il = lane & 31, kh = lane >> 5, rr = lane / ROW_LANES, cc = lane % ROW_LANES;
  const int j = j0 + (GLU ? wj / 2 : wj) + 8 * cc;
  typename std::conditional<GLU, GluEpilogue, Epilogue>::type epi;
  if constexpr (!GRAD) epi.init(g, j);
#pragma unroll
  for (int mp = 0; mp < MI; mp += MP) {
    const int row0 = kg * ROWS * STEP + rr;
    const int64_t ip = i0 + wi + mp * 32 + row0;
    const bool mine = j < g.N && (ACCESSES >= KG || kg < ACCESSES);
    Raw8 res[ROWS];
    if constexpr (!GRAD && !GLU) {
      if (g.res) {
#pragma unroll
        for (int t = 0; t < ROWS; ++t)
          if (mine && ip + STEP * t < g.M) res[t].load(g.res, (size_t)(ip + STEP * t) * g.N + j, g.out_bf16);
      }
    }
#pragma unroll
    for (int m = 0; m < MP; ++m)
#pragma unroll
      for (int nj = 0; nj < NJ; ++nj)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x16_t& c = acc[mp + m][nj];
          const int row = m * 32 + il, ch = nj * 8 + 2 * r + kh;
          *reinterpret_cast<float4*>(buf + row * ROW_BYTES + ((ch ^ (row & (CH - 1))) << 4)) =
              float4{c[4 * r], c[4 * r + 1], c[4 * r + 2], c[4 * r + 3]};
        }
    if constexpr (KG > 1) __syncthreads();
    if (mine) {
#pragma unroll
      for (int t = 0; t < ROWS; ++t) {
        const int row = row0 + STEP * t;
        const int64_t i = ip + STEP * t;
        if (i >= g.M) continue;
        // the row's 8 columns from 16-byte chunk c on, the groups' parts added in order
        auto gather = [&](int c, float (&v)[8]) PK_INLINE {
#pragma unroll
          for (int q = 0; q < KG; ++q) {
            const unsigned char* from = KG > 1 ? piece(q) : buf;
            Raw8 a;
            a.lo = ld16(from + row * ROW_BYTES + ((c ^ (row & (CH - 1))) << 4));
            a.hi = ld16(from + row * ROW_BYTES + (((c + 1) ^ (row & (CH - 1))) << 4));
            float u[8];
            a.unpack(false, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = q ? v[e] + u[e] : u[e];
          }
        };
        float v[8];
        gather(2 * cc, v);
        if constexpr (GLU) {
          float up[8];
          gather(8 + 2 * cc, up);
          epi.store(g, i, j, g.a_scale ? g.a_scale[i] : 1.f, v, up);
          continue;
        }
        const size_t at = (size_t)i * g.N + j;
        if constexpr (GRAD) {
          if (g.part) {
            store8(g.part + (size_t)split * g.M * g.N, at, false, v);
          } else {
            float o[8];
            Raw8 old;
            old.load(g.out, at, false);
            old.unpack(false, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += o[e];
            store8(g.out, at, false, v);
          }
        } else {
          if constexpr (BLOCKS) {
            if (g.part) {
              store8(g.part + (size_t)split * g.M * g.N, at, false, v);
              continue;
            }
          }
          if constexpr (!GLU) epi.store(g, at, g.a_scale ? g.a_scale[i] : 1.f, res[t], v);
        }
      }
    }
    if constexpr (KG > 1 && MI > MP) __syncthreads();  // the pieces are read before they are written again
  }
}

// Few rows of x (up to 8): a workgroup takes 16 rows of W and all of x; its
// waves share k in chunks of 64 bytes, straight from memory into the 16x16
// fragments (rows past the end are read as the last one and dropped), and add
// their sums through LDS in wave order.  Bound by reading W once: 5.8 us for one
// row at 2048 x 2048 bf16 in a graph (5.2 of kernel) and 30 us (4.4 TB/s) at
// 16384 x 4096.  Timed from the host, the 32 x 32 tiles took 6.4 and 32 us where this
// form took 4.8 and 28.6; with 16 rows 6.4 and 33.8, this form 6.8 and 41.
constexpr int FEW_WAVES = 8, FEW_T = 8;

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
template <int DT>
__device__ __forceinline__ void mma16(uint4 w, uint4 x, f32x4_t& c) {
  if constexpr (DT == D_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(w, i)), __uint_as_float(word(x, i)), c, 0, 0, 0);
  } else if constexpr (DT == D_BF16) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w),
                                                __builtin_bit_cast(bf16x8_t, x), c, 0, 0, 0);
  } else {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, widen8(w.x, w.y)),
                                                __builtin_bit_cast(bf16x8_t, widen8(x.x, x.y)), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, widen8(w.z, w.w)),
                                                __builtin_bit_cast(bf16x8_t, widen8(x.z, x.w)), c, 0, 0, 0);
  }
}

template <int DT, int MODE = G_PLAIN>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_gemm_few(const GemmArgs g) {
  // Chunks in flight.  (GLU, 1 x 8192 x 2048 bf16: 16.3 us, with 4 17.3.)
  constexpr int AHEAD = MODE == G_GLU ? 8 : 4;
  constexpr int U = MODE == G_GLU ? 2 : 1;  // rows of W with the same column of y
  constexpr bool BLOCKS = MODE == G_BLOCKS || MODE == G_BLOCKS_TILED, TILED = MODE == G_BLOCKS_TILED;
  static_assert(MODE < G_BLOCKS8, "products are widened here");
  __shared__ __align__(16) float sums[U][FEW_WAVES][16][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n0 = blockIdx.x * 16, kq = (lane >> 4) * 16;
  const int64_t row_bytes = g.K * elem_size(DT);
  const int n = n0 + (lane & 15), r0 = lane & 15;
  const char* wp = (const char*)g.b + (int64_t)(n < g.N ? n : g.N - 1) * row_bytes + kq;
  const char* xp = (const char*)g.a + (r0 < g.M ? r0 : g.M - 1) * row_bytes + kq;
  const int64_t up = g.N * row_bytes;
  f32x4_t acc[U];
#pragma unroll
  for (int u = 0; u < U; ++u) acc[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const uint4 zero{0, 0, 0, 0};
  for (int64_t kb = wave * 64; kb < row_bytes; kb += FEW_WAVES * 64 * AHEAD) {
    uint4 w[U][AHEAD], x[AHEAD];
    float4 sw[AHEAD];
    float sx[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int64_t at = kb + a * (FEW_WAVES * 64);
      const bool in = at + kq < row_bytes;
      if constexpr (BLOCKS) {  // a chunk lies in one block; past the end: the last one's
        const int64_t block = (at < row_bytes ? at : row_bytes - 1) / SCALE_K;
        sx[a] = g.a_block[block * g.M + (r0 < g.M ? r0 : g.M - 1)];
        if constexpr (TILED) {
          const float s = g.b_block[block * ((g.N + SCALE_K - 1) / SCALE_K) + n0 / SCALE_K];
          sw[a] = float4{s, s, s, s};
        } else {
          const int j = n0 + 4 * (lane >> 4);
          sw[a] = *reinterpret_cast<const float4*>(g.b_block + block * g.N + (j < g.N ? j : g.N - 4));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) w[u][a] = in ? ld16_nt(wp + u * up + at) : zero;
      x[a] = in ? ld16(xp + at) : zero;
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if constexpr (BLOCKS) {
          f32x4_t p = {0.f, 0.f, 0.f, 0.f};
          mma16<DT>(w[u][a], x[a], p);
          acc[u][0] = fmaf(p[0] * sw[a].x, sx[a], acc[u][0]);
          acc[u][1] = fmaf(p[1] * sw[a].y, sx[a], acc[u][1]);
          acc[u][2] = fmaf(p[2] * sw[a].z, sx[a], acc[u][2]);
          acc[u][3] = fmaf(p[3] * sw[a].w, sx[a], acc[u][3]);
        } else {
          mma16<DT>(w[u][a], x[a], acc[u]);
        }
      }
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    *reinterpret_cast<float4*>(&sums[u][wave][lane & 15][4 * (lane >> 4)]) =
        float4{acc[u][0], acc[u][1], acc[u][2], acc[u][3]};
  __syncthreads();
  const int i = threadIdx.x >> 1, c = (threadIdx.x & 1) * 8, j = n0 + c;
  if (i >= g.M || j >= g.N) return;  // M <= 8
  float v[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[u][e] = sums[u][0][i][c + e];
    for (int q = 1; q < FEW_WAVES; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] += sums[u][q][i][c + e];
  }
  const float sa = g.a_scale ? g.a_scale[i] : 1.f;
  if constexpr (MODE == G_GLU) {
    GluEpilogue epi;
    epi.init(g, j);
    epi.store(g, i, j, sa, v[0], v[1]);
  } else {
    Epilogue epi;
    epi.init(g, j);
    Raw8 res;
    const size_t at = (size_t)i * g.N + j;
    if (g.res) res.load(g.res, at, g.out_bf16);
    epi.store(g, at, sa, res, v[0]);
  }
}

}  // namespace

}  // namespace pk
