// AdamW over many tensors in one launch, or over the touched rows of a table.
//
//   g = grad * scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g g;
//   p = p (1 - lr wd) - (m / (sqrt(v) / sqrt(1 - b2^t) + eps)) * lr / (1 - b1^t).
//
// Memory bound: parameter and states read and written once, the gradient
// read once (28 bytes an element in fp32, 12 for a bf16 parameter with 8-bit
// states), and the memory moves those bytes and no others (counters).  Median and
// least of several runs: 2^28 elements in fp32 1.48 ms (5.09 TB/s); 2^29 with 8-bit
// states 1.36 and 1.31 ms (4.8 TB/s: the vector arithmetic of quotient, root, hash and
// two roundings takes nearly as long as the memory; up to 1.5 ms a call in a kernel
// trace); 400001 touched rows of 1024 1.17 and 1.11 ms (4.2; up to 1.3).  A lane holds
// 8 consecutive elements (16- and 32-byte accesses), 16 lanes the 128 elements that
// share the scales of their 8-bit states, so the largest element of a block is found
// by four lane exchanges.
//
// 8-bit states hold m and r = sqrt(v) in e4m3 with one fp32 scale per 128
// elements (largest / 448).  The root halves the range of exponents that v
// needs.  Both are rounded up or down at random, in proportion to what is
// cut off: a step moves v by (1 - b2) of itself, far below half a step of a
// 3-bit mantissa, and rounding to nearest would leave it where it is for
// good.  r > 0 never becomes 0 (the update divides by it).  bf16 parameters
// are rounded at random for the same reason.  The random bits are a hash of
// seed, step, tensor and element: the same call gives the same bits.
// Arithmetic is fp32 without contraction to fma, in the order written above,
// so that a plain elementwise program gives the same numbers.
#include <math.h>

#include "pk_internal.h"
#include "pk_row.h"

#pragma clang fp contract(off)

namespace pk {

namespace {

constexpr int BLOCK = 256;
constexpr int LANE_ELEMS = 8;
constexpr int UNIT = ADAMW_STATE_BLOCK;           // 128 elements: 16 lanes
constexpr int UNIT_LANES = UNIT / LANE_ELEMS;
constexpr int WG_UNITS = BLOCK / UNIT_LANES;      // units per workgroup and pass
constexpr int PASSES = 2;                         // passes of a workgroup
// Workgroups of one launch, which holds fewer than 2^32 threads.
constexpr uint64_t LAUNCH_WORKGROUPS = (1 << 24) - 1;
static_assert(ADAMW_MAX_NUMEL == LAUNCH_WORKGROUPS * WG_UNITS * PASSES * UNIT, "a tensor fits one launch");

struct Tensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* sm;
  float* sv;
  uint64_t n;
  uint32_t first;  // first workgroup
  uint32_t key;    // added to the step's key of the hash
};
constexpr int MAX_TENSORS = 40;  // of one launch: 2.6 KB of kernel arguments
struct Args {
  AdamwScalars c;
  const float* grad_scale;
  const float* lr_dev;
  const int64_t* step_dev;
  double lr, beta1, beta2, wd;
  uint32_t seed_lo, seed_hi;
  int count;
  Tensor t[MAX_TENSORS];
};
// Touched rows of one table.
struct RowArgs {
  AdamwScalars c;
  const float* grad_scale;
  const float* lr_dev;
  const int64_t* step_dev;
  double lr, beta1, beta2, wd;
  uint32_t seed_lo, seed_hi;
  Tensor t;
  const int64_t* rows;
  int64_t U, N;
  int D, per_row;  // per_row = ceil(D / 128)
  uint32_t first;  // first unit of this launch
};

__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}
__host__ __device__ __forceinline__ uint32_t step_key(uint32_t lo, uint32_t hi, int64_t step) {
  return mix32(mix32(mix32(lo) + hi) + (uint32_t)step);
}
__device__ __forceinline__ uint32_t random_bits(uint64_t at, uint32_t key) {
  return mix32(((uint32_t)at + key) ^ ((uint32_t)(at >> 32) * 0x3C6EF373u));
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// bf16 bits of p, up with the probability of the part cut off (12 bits of h).
// An infinity stays one (its mantissa is 0).
__device__ __forceinline__ uint32_t round_bf16(float p, uint32_t h) {
  const uint32_t up = (__float_as_uint(p) + (((h & 0xFFFu) << 4) | 8u)) >> 16;
  return p == p ? up : 0x7FC0u;
}
// x / scale on the e4m3 grid, up with the probability of the part cut off:
// `more` holds random bits below the third mantissa bit.  Below 2^-6 the grid
// is even (2^-9): an offset of 2^-6 gives those numbers the same mantissa.  The
// largest value of a block comes out at 448 and at most 4 units in the last
// place above, too few to carry past it with any `more`.
// ROOT: x >= 0, and a value above 0 stays above 0.
template <bool ROOT>
__device__ __forceinline__ float round_e4m3(float x, float inv, uint32_t more) {
  const float a = ROOT ? x * inv : fabsf(x * inv);
  const float low = a < 0x1p-6f ? 0x1p-6f : 0.f;
  float b = __uint_as_float((__float_as_uint(a + low) + more) & 0xFFF00000u) - low;
  if constexpr (ROOT) b = fmaxf(b, a > 0.f ? 0x1p-9f : 0.f);
  else b = copysignf(b, x);
  return finite(x) ? b : __uint_as_float(0x7FC00000u);
}
__device__ __forceinline__ float unit_max(float v) {
  v = fmaxf(v, __uint_as_float(xor_lane<1>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(xor_lane<2>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(xor_lane<4>(__float_as_uint(v))));
  return fmaxf(v, __uint_as_float(xor_lane<8>(__float_as_uint(v))));
}
// A block's scale: its largest finite value over 448, 0 below 2^-126 (then
// every code is 0), and the factor into the grid.  fmaxf passes over a NaN; an
// infinity sends the block through a second look at finite values alone.
__device__ __forceinline__ float unit_scale(const float (&x)[LANE_ELEMS], float& inv) {
  float am = 0.f;
#pragma unroll
  for (int i = 0; i < LANE_ELEMS; ++i) am = fmaxf(am, fabsf(x[i]));
  am = unit_max(am);
  if (__builtin_expect(!finite(am), 0)) {
    am = 0.f;
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i) am = fmaxf(am, finite(x[i]) ? fabsf(x[i]) : 0.f);
    am = unit_max(am);
  }
  float s = am * (1.f / E4M3_MAX);
  s = s < 0x1p-126f ? 0.f : s;
  inv = s > 0.f ? 1.f / s : 0.f;
  return s;
}

// 8 consecutive elements as fp32; whole: all there and 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool whole, int count, float (&f)[LANE_ELEMS]) {
  if (whole) {
#pragma unroll
    for (int c = 0; c < LANE_ELEMS / Chunk<T>::N; ++c)
      Chunk<T>::unpack(ld16_nt(p + c * Chunk<T>::N), f + c * Chunk<T>::N);
  } else {
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i) {
      f[i] = 0.f;
      if (i < count) {
        if constexpr (sizeof(T) == 2) f[i] = bf16_to_f32(p[i]);
        else f[i] = p[i];
      }
    }
  }
}
__device__ __forceinline__ void load_codes(const uint8_t* p, bool whole, int count,
                                           float (&f)[LANE_ELEMS]) {
  uint2 u{0, 0};
  if (whole) {
    u = *reinterpret_cast<const uint2*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i)
      if (i < count) (i < 4 ? u.x : u.y) |= (uint32_t)p[i] << (8 * (i & 3));
  }
  from_e4m3x4(u.x, f);
  from_e4m3x4(u.y, f + 4);
}
__device__ __forceinline__ void store_codes(uint8_t* p, bool whole, int count,
                                            const float (&f)[LANE_ELEMS]) {
  const uint2 u{to_e4m3x4(f[0], f[1], f[2], f[3]), to_e4m3x4(f[4], f[5], f[6], f[7])};
  if (whole) {
    *reinterpret_cast<uint2*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i)
      if (i < count) p[i] = (uint8_t)((i < 4 ? u.x : u.y) >> (8 * (i & 3)));
  }
}
__device__ __forceinline__ void store_f32(float* p, bool whole, int count,
                                          const float (&f)[LANE_ELEMS]) {
  if (whole) {
    st16_nt(p, Chunk<float>::pack(f));
    st16_nt(p + 4, Chunk<float>::pack(f + 4));
  } else {
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i)
      if (i < count) p[i] = f[i];
  }
}

// The step on a lane's elements off .. off + count - 1 (0 <= count <= 8) of
// tensor t, whose 128-element block has scales at `block`.  Every lane of the
// block calls it.  g: the scaled gradient; at: the first element's place for
// the hash.
template <typename P, bool S8>
__device__ __forceinline__ void step8(const Tensor& t, const AdamwScalars& c, uint32_t key,
                                      uint64_t off, uint64_t block, int count, bool whole,
                                      const float (&g)[LANE_ELEMS]) {
  float p[LANE_ELEMS], m[LANE_ELEMS], v[LANE_ELEMS], r[LANE_ELEMS];
  P* pp = (P*)t.p + off;
  load8(pp, whole, count, p);
  if constexpr (S8) {
    const float sm = t.sm[block], sv = t.sv[block];
    load_codes((const uint8_t*)t.m + off, whole, count, m);
    load_codes((const uint8_t*)t.v + off, whole, count, r);
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i) {
      m[i] = m[i] * sm;
      r[i] = r[i] * sv;
      v[i] = r[i] * r[i];
    }
  } else {
    load8((const float*)t.m + off, whole, count, m);
    load8((const float*)t.v + off, whole, count, v);
  }
#pragma unroll
  for (int i = 0; i < LANE_ELEMS; ++i) {
    m[i] = m[i] * c.beta1 + g[i] * c.rest1;
    v[i] = v[i] * c.beta2 + (g[i] * g[i]) * c.rest2;
    r[i] = sqrtf(v[i]);
    p[i] = p[i] * c.decay - (m[i] / (r[i] * c.root2 + c.eps)) * c.rate;
  }
  uint32_t h[LANE_ELEMS];
  if constexpr (S8 || sizeof(P) == 2) {
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i) h[i] = random_bits(off + i, key);
  }
  if constexpr (sizeof(P) == 2) {
    uint32_t b[LANE_ELEMS];
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i) b[i] = round_bf16(p[i], h[i]);
    if (whole) {
      st16_nt(pp, uint4{b[0] | b[1] << 16, b[2] | b[3] << 16, b[4] | b[5] << 16, b[6] | b[7] << 16});
    } else {
#pragma unroll
      for (int i = 0; i < LANE_ELEMS; ++i)
        if (i < count) pp[i] = (P)b[i];
    }
  } else {
    store_f32((float*)pp, whole, count, p);
  }
  if constexpr (S8) {
    float im, ir;
    const float sm = unit_scale(m, im), sv = unit_scale(r, ir);
    if (count > 0 && (threadIdx.x & (UNIT_LANES - 1)) == 0) {
      t.sm[block] = sm;
      t.sv[block] = sv;
    }
#pragma unroll
    for (int i = 0; i < LANE_ELEMS; ++i) {
      m[i] = round_e4m3<false>(m[i], im, ((h[i] >> 12) & 0xFF000u) | (1u << 11));
      r[i] = round_e4m3<true>(r[i], ir, ((h[i] >> 4) & 0xFFF00u) | (1u << 7));
    }
    store_codes((uint8_t*)t.m + off, whole, count, m);
    store_codes((uint8_t*)t.v + off, whole, count, r);
  } else {
    store_f32((float*)t.m + off, whole, count, m);
    store_f32((float*)t.v + off, whole, count, v);
  }
}

// Scalars that depend on values in device memory (a captured step whose rate
// and step number move on): one thread forms them for its workgroup.  False:
// the gradient's scale is 0 or not finite or the step number below 1, and
// nothing is changed.
template <typename A>
__device__ __forceinline__ bool scalars(const A& a, AdamwScalars& c, float& gs, uint32_t& key,
                                        AdamwScalars* shared_c, uint32_t* shared_key) {
  gs = a.grad_scale ? *a.grad_scale : 1.f;
  if (gs == 0.f || !finite(gs) || (a.step_dev && *a.step_dev < 1)) return false;
  c = a.c;
  key = c.key;
  if (a.lr_dev || a.step_dev) {
    if (threadIdx.x == 0) {
      AdamwScalars d = a.c;
      const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
      d.decay = (float)(1.0 - lr * a.wd);
      double c1 = a.c.corr1;
      if (a.step_dev) {
        const int64_t step = *a.step_dev;
        c1 = 1.0 - pow(a.beta1, (double)step);
        d.root2 = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)step)));
        d.key = step_key(a.seed_lo, a.seed_hi, step);
      }
      d.rate = (float)(lr / c1);
      *shared_c = d;
      *shared_key = d.key;
    }
    __syncthreads();
    c = *shared_c;
    key = *shared_key;
  }
  return true;
}

template <typename P, typename G, bool S8>
__global__ __launch_bounds__(BLOCK) void k_adamw(const Args a) {
  __shared__ AdamwScalars sc;
  __shared__ uint32_t skey;
  AdamwScalars c;
  float gs;
  uint32_t key;
  if (!scalars(a, c, gs, key, &sc, &skey)) return;
  int i = 0;
  for (int k = 1; k < a.count; ++k)
    if (blockIdx.x >= a.t[k].first) i = k;
  const Tensor t = a.t[i];
  const bool aligned = ((((uintptr_t)t.p | (uintptr_t)t.g) & 15) | (((uintptr_t)t.m | (uintptr_t)t.v) & (S8 ? 7 : 15))) == 0;
  const uint64_t units = (t.n + UNIT - 1) / UNIT;
  uint64_t unit = (uint64_t)(blockIdx.x - t.first) * (WG_UNITS * PASSES) + threadIdx.x / UNIT_LANES;
#pragma unroll
  for (int s = 0; s < PASSES; ++s, unit += WG_UNITS) {
    if (unit >= units) break;  // the 16 lanes of a block leave together
    const uint64_t off = unit * UNIT + (threadIdx.x % UNIT_LANES) * LANE_ELEMS;
    const int count = off >= t.n ? 0 : t.n - off >= LANE_ELEMS ? LANE_ELEMS : (int)(t.n - off);
    const bool whole = aligned && count == LANE_ELEMS;
    float g[LANE_ELEMS];
    load8((const G*)t.g + off, whole, count, g);
#pragma unroll
    for (int e = 0; e < LANE_ELEMS; ++e) g[e] *= gs;
    step8<P, S8>(t, c, key + t.key, off, unit, count, whole, g);
  }
}

// Units of 128 elements of the touched rows.  Row numbers ascend; equal
// neighbours are one row whose gradients are added in order, by the first.
template <typename P, bool S8>
__global__ __launch_bounds__(BLOCK) void k_adamw_rows(const RowArgs a) {
  __shared__ AdamwScalars sc;
  __shared__ uint32_t skey;
  AdamwScalars c;
  float gs;
  uint32_t key;
  if (!scalars(a, c, gs, key, &sc, &skey)) return;
  const uint32_t units = (uint32_t)a.U * (uint32_t)a.per_row;  // below 2^31
  uint32_t unit = a.first + blockIdx.x * (WG_UNITS * PASSES) + threadIdx.x / UNIT_LANES;
#pragma unroll
  for (int s = 0; s < PASSES; ++s, unit += WG_UNITS) {
    if (unit >= units) break;
    const int64_t u = unit / (uint32_t)a.per_row;
    const int b = (int)(unit % (uint32_t)a.per_row);
    const int64_t row = a.rows[u];
    if (row < 0 || row >= a.N || (u > 0 && a.rows[u - 1] == row)) continue;
    const int col = b * UNIT + (threadIdx.x % UNIT_LANES) * LANE_ELEMS;
    const int count = col < a.D ? LANE_ELEMS : 0;  // D % 8 == 0
    const bool whole = count == LANE_ELEMS;
    float g[LANE_ELEMS];
    const float* gp = (const float*)a.t.g + (size_t)u * a.D + col;
    load8(gp, whole, count, g);
    for (int64_t n = u + 1; n < a.U && a.rows[n] == row; ++n) {
      float more[LANE_ELEMS];
      load8(gp + (size_t)(n - u) * a.D, whole, count, more);
#pragma unroll
      for (int e = 0; e < LANE_ELEMS; ++e) g[e] += more[e];
    }
#pragma unroll
    for (int e = 0; e < LANE_ELEMS; ++e) g[e] *= gs;
    step8<P, S8>(a.t, c, key, (uint64_t)row * a.D + col, (uint64_t)row * a.per_row + b, count, whole, g);
  }
}

// Ascending row numbers (equal neighbours allowed) in [0, N)?
__global__ __launch_bounds__(BLOCK) void k_check_rows(const int64_t* __restrict__ rows, int64_t U,
                                                      int64_t N, uint32_t* __restrict__ bad) {
  for (int64_t i = (int64_t)blockIdx.x * BLOCK + threadIdx.x; i < U; i += (int64_t)gridDim.x * BLOCK) {
    const int64_t r = rows[i];
    if (r < 0 || r >= N || (i > 0 && rows[i - 1] > r)) *bad = 1u;
  }
}

template <typename A>
void common_args(A& a, const pkmem_adamw_opts& o) {
  a.grad_scale = o.grad_scale;
  a.lr_dev = o.lr_dev;
  a.step_dev = o.step_dev;
  a.lr = o.lr;
  a.beta1 = o.beta1;
  a.beta2 = o.beta2;
  a.wd = o.weight_decay;
  a.seed_lo = (uint32_t)o.seed;
  a.seed_hi = (uint32_t)(o.seed >> 32);
  AdamwScalars& c = a.c;
  c.beta1 = (float)o.beta1;
  c.rest1 = (float)(1.0 - o.beta1);
  c.beta2 = (float)o.beta2;
  c.rest2 = (float)(1.0 - o.beta2);
  c.eps = (float)o.eps;
  c.decay = (float)(1.0 - o.lr * o.weight_decay);
  c.corr1 = 1.0 - pow(o.beta1, (double)o.step);
  c.rate = (float)(o.lr / c.corr1);
  c.root2 = (float)(1.0 / sqrt(1.0 - pow(o.beta2, (double)o.step)));
  c.key = step_key(a.seed_lo, a.seed_hi, o.step);
}

template <typename P, typename G, bool S8>
void adamw_launch(const Args& a, unsigned blocks, hipStream_t st) {
  hipLaunchKernelGGL((k_adamw<P, G, S8>), dim3(blocks), dim3(BLOCK), 0, st, a);
}

}  // namespace

hipError_t launch_adamw(const pkmem_adamw_tensor* tensors, int count, const pkmem_adamw_opts& o,
                        hipStream_t st) {
  LaunchTimer lt("adamw", st);
  Args a;
  common_args(a, o);
  // one launch for each combination of types that occurs, per 40 tensors
  for (int kind = 0; kind < 8; ++kind) {
    const bool p16 = kind & 1, g16 = kind & 2, s8 = kind & 4;
    a.count = 0;
    uint64_t blocks = 0;
    auto flush = [&]() -> hipError_t {
      if (!a.count) return hipSuccess;
      if (s8) {
        if (p16) { if (g16) adamw_launch<uint16_t, uint16_t, true>(a, (unsigned)blocks, st); else adamw_launch<uint16_t, float, true>(a, (unsigned)blocks, st); }
        else { if (g16) adamw_launch<float, uint16_t, true>(a, (unsigned)blocks, st); else adamw_launch<float, float, true>(a, (unsigned)blocks, st); }
      } else {
        if (p16) { if (g16) adamw_launch<uint16_t, uint16_t, false>(a, (unsigned)blocks, st); else adamw_launch<uint16_t, float, false>(a, (unsigned)blocks, st); }
        else { if (g16) adamw_launch<float, uint16_t, false>(a, (unsigned)blocks, st); else adamw_launch<float, float, false>(a, (unsigned)blocks, st); }
      }
      a.count = 0;
      blocks = 0;
      return hipGetLastError();
    };
    for (int i = 0; i < count; ++i) {
      const pkmem_adamw_tensor& t = tensors[i];
      if ((t.param_dt == PKMEM_BF16) != p16 || (t.grad_dt == PKMEM_BF16) != g16 ||
          (t.state_dt == PKMEM_E4M3) != s8 || t.numel <= 0)
        continue;
      const uint64_t units = ((uint64_t)t.numel + UNIT - 1) / UNIT;
      const uint64_t need = (units + WG_UNITS * PASSES - 1) / (WG_UNITS * PASSES);
      if (a.count == MAX_TENSORS || blocks + need > LAUNCH_WORKGROUPS) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      a.t[a.count++] = Tensor{t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale,
                              t.exp_avg_sq_scale, (uint64_t)t.numel, (uint32_t)blocks,
                              (uint32_t)i * 0x9E3779B1u};
      blocks += need;
    }
    const hipError_t e = flush();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_adamw_rows(const pkmem_adamw_tensor& t, int64_t N, int D, const int64_t* rows,
                             int64_t U, const pkmem_adamw_opts& o, hipStream_t st) {
  LaunchTimer lt("adamw_rows", st);
  RowArgs a;
  common_args(a, o);
  a.t = Tensor{t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, 0, 0, 0};
  a.rows = rows;
  a.U = U;
  a.N = N;
  a.D = D;
  a.per_row = (D + UNIT - 1) / UNIT;
  const bool p16 = t.param_dt == PKMEM_BF16, s8 = t.state_dt == PKMEM_E4M3;
  const uint64_t units = (uint64_t)U * a.per_row, most = LAUNCH_WORKGROUPS * WG_UNITS * PASSES;
  for (uint64_t first = 0; first < units; first += most) {
    const uint64_t n = units - first < most ? units - first : most;
    const dim3 grid((unsigned)((n + WG_UNITS * PASSES - 1) / (WG_UNITS * PASSES))), block(BLOCK);
    a.first = (uint32_t)first;
    if (p16 && s8) hipLaunchKernelGGL((k_adamw_rows<uint16_t, true>), grid, block, 0, st, a);
    else if (p16) hipLaunchKernelGGL((k_adamw_rows<uint16_t, false>), grid, block, 0, st, a);
    else if (s8) hipLaunchKernelGGL((k_adamw_rows<float, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_adamw_rows<float, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

hipError_t launch_check_rows(const int64_t* rows, int64_t U, int64_t N, uint32_t* bad, hipStream_t st) {
  hipError_t e = launch_fill_u32(bad, 0u, 1, st);
  if (e != hipSuccess || U <= 0) return e;
  int64_t blocks = (U + BLOCK - 1) / BLOCK;
  if (blocks > 4096) blocks = 4096;
  hipLaunchKernelGGL(k_check_rows, dim3((unsigned)blocks), dim3(BLOCK), 0, st, rows, U, N, bad);
  return hipGetLastError();
}

}  // namespace pk
