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

struct GemmArgs {
  const void* a;  // rows i
  const void* b;  // rows j
  int64_t M;
  int N;
  int64_t K;
  int64_t k_split;  // k of one split (a multiple of a stage's)
  int tiles_m, tiles_n;
  // epilogue
  const float* a_scale;
  const float* b_scale;
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

// An operand's tile: R rows by one stage of k.
//   KS = false: LDS [R][64 bytes of k]; 16-byte chunk c of row r lies at slot
//     c ^ ((r >> 2) & 3): the 16 lanes that LDS serves at once (lanes 0-3, 12-15,
//     20-27 and so on) then read 16 different 16-byte columns of its 64 banks.
//   KS = true: LDS [k][R elements]; the 64-byte (bf16) or 128-byte (fp32) units
//     of a k row are permuted by k so that the k rows of one read instruction
//     lie in different banks.
template <int DT, bool KS, int R, int NWAVE>
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
  int whole;            // stages left that lie within k

  // rows: first row of the tile, of `rows`; k range [k0, k1) of ld = K (or rows) elements
  __device__ __forceinline__ void init(const void* p, int64_t row0, int64_t rows, int64_t K,
                                       int64_t k0, int64_t k1, int wave, int lane) {
    whole = k1 > k0 ? (int)((k1 - k0) / STAGE_ROWS) : 0;
    const int64_t ld = (KS ? rows : K) * E;
    base = (const char*)p + (KS ? k0 * ld + row0 * E : row0 * ld + k0 * E);
    step = KS ? (int64_t)STAGE_ROWS * ld : STAGE_K;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int slot = (i * NWAVE + wave) * 64 + lane;
      if constexpr (!KS) {
        const int r = slot >> 2;
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
    lds_dma16_buf(raw_buffer(base, 0x7FFFFFFFu), o, 0u, lds + (i * NWAVE + wave) * 1024);
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

// KG groups of waves share the tile's k.  GRAD: C is added to fp32 `out`, or written to `part` when split; else the
// epilogue above.
template <int DT, bool AKS, bool BKS, bool GRAD, int BM, int BN, int WM, int WN, int KG>
__global__ __launch_bounds__(WM* WN* KG * 64) void k_gemm(const GemmArgs g) {
  constexpr int NW = WM * WN, MI = BM / WM / 32, NJ = BN / WN / 32;
  using OA = Operand<DT, AKS, BM, NW>;
  using OB = Operand<DT, BKS, BN, NW>;
  constexpr int L = OA::LOADS + OB::LOADS;
  constexpr int GROUP_BYTES = OA::BYTES + OB::BYTES, BYTES = KG * GROUP_BYTES;
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
  const int tile_n = pid / m_count, j0 = tile_n * BN;
  int64_t k0 = split * g.k_split;
  int64_t k1 = k0 + g.k_split < g.K ? k0 + g.k_split : g.K;
  // this group's share of k; all groups take the same number of steps
  const int steps = (int)((k1 - k0 + KG * OA::STAGE_ROWS - 1) / (KG * OA::STAGE_ROWS));
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

  f32x16_t acc[MI][NJ];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x16_t{};

  const int group_at = KG > 1 ? kg * GROUP_BYTES : 0;
  int left = k1 > k0 ? (int)(k1 - k0 < 0x7FFFFFFF ? k1 - k0 : 0x7FFFFFFF) : 0;
  // Load i of a stage (A's first), and the step to the next one.
  auto load = [&](unsigned char* st, int i) PK_INLINE {
    if (i < OA::LOADS) oa.load(i, st + group_at, wave, lane, left);
    else ob.load(i - OA::LOADS, st + group_at + OA::BYTES, wave, lane, left);
  };
  auto advance = [&]() PK_INLINE {
    oa.advance();
    ob.advance();
    left -= OA::STAGE_ROWS;
  };
  auto fill = [&](unsigned char* st) PK_INLINE {
#pragma unroll
    for (int i = 0; i < L; ++i) load(st, i);
    advance();
  };
  // Fragments of the halves 0 and 1 of a stage; in fp32 where every wave multiplies
  // all the time, of two stages in turn.
  constexpr bool TURNS = NW * KG == 8;
  constexpr int SETS = DT == D_F32 && !TURNS ? 2 : 1;
  uint4 fa[SETS][2][MI], fb[SETS][2][NJ];
  auto read = [&](const unsigned char* st, int h, int set = 0) PK_INLINE {
#pragma unroll
    for (int nj = 0; nj < NJ; ++nj) fb[set][h][nj] = ob.frag(st + group_at + OA::BYTES, nj, h);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) fa[set][h][mi] = oa.frag(st + group_at, mi, h);
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
    auto multiply = [&]() PK_INLINE {
      __builtin_amdgcn_s_setprio(1);
      if constexpr (DT == D_F32) {
        products_f32(0);
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
    auto first = [&](unsigned char* st, const unsigned char* next) PK_INLINE {
      multiply();
      wait_and_meet<2 * L>();  // the next stage has landed
      read_all(next);
      fill(st);
      wait_and_meet<63>();  // 63: for LDS alone
    };
    auto last = [&](unsigned char* st, unsigned char* before) PK_INLINE {
      read_all(st);
      fill(before);
      wait_and_meet<2 * L>();
      multiply();
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
        first(st1, st2);
        first(st2, st3);
        first(st3, st0);
      }
      if (s < steps) first(st0, st1);
      if (s + 1 < steps) first(st1, st2);
      if (s + 2 < steps) first(st2, st3);
    } else {
      wait_and_meet<2 * L>();
      for (; s + 4 <= steps; s += 4) {
        last(st0, st3);
        last(st1, st0);
        last(st2, st1);
        last(st3, st2);
      }
      if (s < steps) last(st0, st3);
      if (s + 1 < steps) last(st1, st0);
      if (s + 2 < steps) last(st2, st1);
    }
  } else if constexpr (DT == D_F32) {
    // One stage: it is in the registers of set; next has landed for all after the
    // barrier, and is read while the products run.
    auto stage = [&](int set, unsigned char* st, const unsigned char* next) PK_INLINE {
      wait_and_meet<2 * L>();
      read(next, 0, set ^ 1);
      read(next, 1, set ^ 1);
      __builtin_amdgcn_sched_barrier(0);
      add_bias(next);
      fill(st);
      products_f32(set);
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
  constexpr int ROW_LANES = NJ * 4, STEP = 64 / ROW_LANES;  // lanes of a row, rows of an access
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
  const int j = j0 + wj + 8 * cc;
  Epilogue epi;
  if constexpr (!GRAD) epi.init(g, j);
#pragma unroll
  for (int mp = 0; mp < MI; mp += MP) {
    const int row0 = kg * ROWS * STEP + rr;
    const int64_t ip = i0 + wi + mp * 32 + row0;
    const bool mine = j < g.N && (ACCESSES >= KG || kg < ACCESSES);
    Raw8 res[ROWS];
    if constexpr (!GRAD) {
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
        float v[8];
#pragma unroll
        for (int q = 0; q < KG; ++q) {
          const unsigned char* from = KG > 1 ? piece(q) : buf;
          Raw8 a;
          a.lo = ld16(from + row * ROW_BYTES + (((2 * cc) ^ (row & (CH - 1))) << 4));
          a.hi = ld16(from + row * ROW_BYTES + (((2 * cc + 1) ^ (row & (CH - 1))) << 4));
          float u[8];
          a.unpack(false, u);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = q ? v[e] + u[e] : u[e];
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
          epi.store(g, at, g.a_scale ? g.a_scale[i] : 1.f, res[t], v);
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

template <int DT>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_gemm_few(const GemmArgs g) {
  constexpr int AHEAD = 4;  // chunks in flight
  __shared__ __align__(16) float sums[FEW_WAVES][16][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n0 = blockIdx.x * 16, kq = (lane >> 4) * 16;
  const int64_t row_bytes = g.K * elem_size(DT);
  const int n = n0 + (lane & 15), r0 = lane & 15;
  const char* wp = (const char*)g.b + (int64_t)(n < g.N ? n : g.N - 1) * row_bytes + kq;
  const char* xp = (const char*)g.a + (r0 < g.M ? r0 : g.M - 1) * row_bytes + kq;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  const uint4 zero{0, 0, 0, 0};
  for (int64_t kb = wave * 64; kb < row_bytes; kb += FEW_WAVES * 64 * AHEAD) {
    uint4 w[AHEAD], x[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int64_t at = kb + a * (FEW_WAVES * 64);
      const bool in = at + kq < row_bytes;
      w[a] = in ? ld16_nt(wp + at) : zero;
      x[a] = in ? ld16(xp + at) : zero;
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) mma16<DT>(w[a], x[a], acc);
  }
  *reinterpret_cast<float4*>(&sums[wave][lane & 15][4 * (lane >> 4)]) = float4{acc[0], acc[1], acc[2], acc[3]};
  __syncthreads();
  const int i = threadIdx.x >> 1, c = (threadIdx.x & 1) * 8, j = n0 + c;
  if (i >= g.M || j >= g.N) return;  // M <= 8
  Epilogue epi;
  epi.init(g, j);
  Raw8 res;
  const size_t at = (size_t)i * g.N + j;
  if (g.res) res.load(g.res, at, g.out_bf16);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = sums[0][i][c + e];
  for (int q = 1; q < FEW_WAVES; ++q)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += sums[q][i][c + e];
  epi.store(g, at, g.a_scale ? g.a_scale[i] : 1.f, res, v);
}

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
