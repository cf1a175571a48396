// C ABI of the product-key memory hot path: argument checks on the host,
// workspace carving, dispatch to the kernels.  Declared in include/pkmem.h.
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>
#include <mutex>
#include <string>
#include <utility>
#include <vector>

#include "pkmem.h"
#include "pk_internal.h"

namespace {

thread_local std::string g_last_error;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return code;
}

int hip_status(hipError_t e, const char* where) {
  if (e == hipSuccess) return PKMEM_OK;
  return fail(PKMEM_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t esize(pkmem_dtype t) { return t == PKMEM_BF16 ? 2 : 4; }
inline bool dtype_ok(int t) { return t == PKMEM_F32 || t == PKMEM_BF16; }

struct SearchWs {
  uint64_t* cand;
  uint32_t* cnts;
  float* thr;
  int32_t* half_idx;
  float* half_score;
  uint32_t* ovf;
  float2* qstats;  // per (token, head) query (mean, rstd) when normalising
  float* sink_part;  // per (token, head) the two halves' parts of the sink's score
  size_t bytes;
};

// The search workspace carved from base (only its size when base is null).
SearchWs search_ws(void* base, int64_t T, int H, int k) {
  const size_t rows = (size_t)T * H * 2;
  char* p = reinterpret_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) -> char* {
    char* at = p ? p + off : nullptr;
    off += align256(bytes);
    return at;
  };
  // candidate runs come in groups of 32 tokens (one per scoring wave)
  const size_t grows = (size_t)((T + 31) / 32) * 32 * H * 2;
  SearchWs w;
  w.cand = reinterpret_cast<uint64_t*>(take(grows * pk::CAND_CAP * sizeof(uint64_t)));
  w.cnts = reinterpret_cast<uint32_t*>(take(rows * 2 * sizeof(uint32_t)));
  w.thr = reinterpret_cast<float*>(take(rows * sizeof(float)));
  w.half_idx = reinterpret_cast<int32_t*>(take(rows * k * sizeof(int32_t)));
  w.half_score = reinterpret_cast<float*>(take(rows * k * sizeof(float)));
  w.ovf = reinterpret_cast<uint32_t*>(take((rows + 1) * sizeof(uint32_t)));
  w.qstats = reinterpret_cast<float2*>(take((size_t)T * H * sizeof(float2)));
  w.sink_part = reinterpret_cast<float*>(take((size_t)T * H * 2 * sizeof(float)));
  w.bytes = off;
  return w;
}

// k is the selection size (1 <= k <= min(S, KMAX)), or with slots the number
// of product-key slots per row (1 <= k <= KMAX; extras may exceed S).
int check_search_shapes(const char* fn, const void* q, pkmem_dtype q_dt, const void* subkeys,
                        pkmem_dtype k_dt, int64_t T, int H, int n, int S, int k,
                        bool slots = false) {
  if (!dtype_ok(q_dt) || !dtype_ok(k_dt)) return fail(PKMEM_ERR_INVALID, "%s: unknown dtype", fn);
  if (q_dt != k_dt) return fail(PKMEM_ERR_UNSUPPORTED, "%s: queries and sub-keys must share a dtype", fn);
  if (T < 0) return fail(PKMEM_ERR_INVALID, "%s: T must be >= 0", fn);
  if (H < 1) return fail(PKMEM_ERR_INVALID, "%s: H must be >= 1", fn);
  if (n < 2 || n % 2 != 0) return fail(PKMEM_ERR_INVALID, "%s: n must be even and >= 2 (got %d)", fn, n);
  const int d = n / 2;
  if (q_dt == PKMEM_BF16 && (d % 8 != 0 || d > PKMEM_DHALF_MAX))
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: bf16 needs n/2 a multiple of 8 and <= %d (got %d)", fn, PKMEM_DHALF_MAX, d);
  if (q_dt == PKMEM_F32 && (d % 4 != 0 || d > 64))
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: fp32 needs n/2 a multiple of 4 and <= 64 (got %d)", fn, d);
  if (S < 1) return fail(PKMEM_ERR_INVALID, "%s: S must be >= 1", fn);
  if (S > PKMEM_SMAX) return fail(PKMEM_ERR_UNSUPPORTED, "%s: S > %d", fn, PKMEM_SMAX);
  if (k < 1 || (!slots && k > S)) return fail(PKMEM_ERR_INVALID, "%s: need 1 <= k <= S (k=%d, S=%d)", fn, k, S);
  if (k > PKMEM_KMAX) return fail(PKMEM_ERR_UNSUPPORTED, "%s: k > %d", fn, PKMEM_KMAX);
  if ((T * H * 2) > (int64_t)0xFFFFFFFF) return fail(PKMEM_ERR_UNSUPPORTED, "%s: T*H*2 must be < 2^32", fn);
  if (T > 0 && (!q || !subkeys)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(q, 16) || !aligned(subkeys, 16)) return fail(PKMEM_ERR_INVALID, "%s: q and subkeys must be 16-byte aligned", fn);
  return PKMEM_OK;
}

int check_bag_shapes(const char* fn, pkmem_dtype v_dt, int64_t N, int D, int64_t T, int bag) {
  if (!dtype_ok(v_dt)) return fail(PKMEM_ERR_INVALID, "%s: unknown value dtype %d", fn, (int)v_dt);
  if (N < 1) return fail(PKMEM_ERR_INVALID, "%s: N must be >= 1 (got %lld)", fn, (long long)N);
  if (N > (int64_t(1) << 32)) return fail(PKMEM_ERR_UNSUPPORTED, "%s: N > 2^32 rows", fn);
  if (T < 0) return fail(PKMEM_ERR_INVALID, "%s: T must be >= 0", fn);
  if (bag < 1) return fail(PKMEM_ERR_INVALID, "%s: bag (H*k) must be >= 1", fn);
  if (D < 8 || D % 8 != 0) return fail(PKMEM_ERR_UNSUPPORTED, "%s: D must be a positive multiple of 8 (got %d)", fn, D);
  const int chunks = (int)(D * esize(v_dt) / 16);
  if (chunks > 512) return fail(PKMEM_ERR_UNSUPPORTED, "%s: rows wider than 8 KiB are not supported (D=%d)", fn, D);
  if ((T * (int64_t)bag) > (int64_t)0xFFFFFFFF) return fail(PKMEM_ERR_UNSUPPORTED, "%s: T*bag must be < 2^32", fn);
  return PKMEM_OK;
}

// grad_w when the caller passes none; for the sorted strategy the sort, then
// the partial rows of long rows' chunks.
size_t bwd_ws_bytes(int64_t T, int H, int k, int D, int mode) {
  const int64_t L = T * H * k;
  size_t b = align256((size_t)L * sizeof(float));
  if (mode == PKMEM_BWD_SORTED) b += pk::sorted_workspace_bytes(L) + pk::long_partial_bytes(L, D);
  return b;
}

// What PKMEM_BWD_AUTO means for L = T*H*k lookups of rows of D elements:
// atomic adds when L*D <= 2^26 fp32 updates and D <= 1024, the sorted
// strategy otherwise.  Measured on MI355X (uniform indices over 2^20 rows,
// D = 64..2048, L = 32K..2M): the atomic kernel costs about 3.5 ps per
// updated element plus one launch, the sort a fixed ~0.05 ms (its launches;
// up to 2^19 lookups one per pass) plus its row streaming, so atomics win only
// small batches: D = 64, 524288 lookups 0.11 against 0.16 ms, but D = 128,
// 1048576 lookups 0.44 against 0.38.  At D = 2048 the sort wins from 256 tokens
// on.  The line is fixed in the interface (pkmem.h states it: workspaces are sized
// and the sum's order, bitwise deterministic or not, is chosen by it); at its upper edge
// for D of 512 and more the sort is the faster one by 9 to 11% (D = 512, 131072
// lookups 0.229 against 0.208 ms; D = 1024, 32768 0.137 against 0.122).
// PKMEM_BWD_MODE=atomic|sorted in the environment overrides the choice (read at
// every call).
int resolve_mode(int mode, int D, int64_t L) {
  if (mode != PKMEM_BWD_AUTO) return mode;
  const char* env = getenv("PKMEM_BWD_MODE");
  if (env && strcmp(env, "atomic") == 0) return PKMEM_BWD_ATOMIC;
  if (env && strcmp(env, "sorted") == 0) return PKMEM_BWD_SORTED;
  return (D <= 1024 && L * (int64_t)D <= (int64_t(1) << 26)) ? PKMEM_BWD_ATOMIC : PKMEM_BWD_SORTED;
}

// PKMEM_DEBUG=1 in the environment (read at every call) checks on the device
// that every index lies in [0, limit) before the kernels that use them run:
// the call waits for the check and fails with PKMEM_ERR_INVALID otherwise.
// The flag it needs is the only device memory the library allocates (4 bytes
// per device, once, and only in debug mode).
bool debug_checks() {
  const char* env = getenv("PKMEM_DEBUG");
  return env && env[0] && strcmp(env, "0") != 0;
}

// The debug check's flag on the current device (allocated at first use).
int debug_flag(const char* fn, uint32_t** flag) {
  static uint32_t* flags[64] = {};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_status(e, fn);
  if (dev < 0 || dev >= 64) return fail(PKMEM_ERR_UNSUPPORTED, "%s: device %d", fn, dev);
  if (!flags[dev]) {
    e = hipMalloc(reinterpret_cast<void**>(&flags[dev]), sizeof(uint32_t));
    if (e != hipSuccess) return hip_status(e, fn);
  }
  *flag = flags[dev];
  return PKMEM_OK;
}

// Waits for the check launched (status e) and reads its flag.
int debug_outcome(const char* fn, hipError_t e, uint32_t* flag, int64_t limit, hipStream_t st) {
  uint32_t bad = 0;
  if (e == hipSuccess) e = hipMemcpyAsync(&bad, flag, sizeof(bad), hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hip_status(e, fn);
  if (bad) return fail(PKMEM_ERR_INVALID, "%s: an index lies outside [0, %lld) (PKMEM_DEBUG)", fn, (long long)limit);
  return PKMEM_OK;
}

int check_indices(const char* fn, const int64_t* idx, int64_t count, int64_t limit, hipStream_t st) {
  if (!debug_checks() || count <= 0) return PKMEM_OK;
  uint32_t* flag = nullptr;
  int rc = debug_flag(fn, &flag);
  if (rc) return rc;
  hipError_t e = pk::launch_check_indices(idx, count, limit, flag, st);
  return debug_outcome(fn, e, flag, limit, st);
}

// check_indices over the first cols slots of each of rows rows, stride apart.
int check_indices_strided(const char* fn, const int64_t* idx, int64_t rows, int cols, int stride,
                          int64_t limit, hipStream_t st) {
  if (cols == stride) return check_indices(fn, idx, rows * cols, limit, st);
  if (!debug_checks() || rows <= 0) return PKMEM_OK;
  uint32_t* flag = nullptr;
  int rc = debug_flag(fn, &flag);
  if (rc) return rc;
  hipError_t e = pk::launch_check_indices_strided(idx, rows, cols, stride, limit, flag, st);
  return debug_outcome(fn, e, flag, limit, st);
}

int bag_backward_common(const char* fn, const void* dy, const void* values, pkmem_dtype v_dt,
                        int64_t N, int D, const int64_t* idx, const float* w, int64_t T, int H,
                        int k, float* grad_values, int64_t* rows_out, float* grad_rows_out,
                        int64_t cap, int64_t* num_rows_out, float* grad_w, float* grad_scores,
                        int mode, void* ws, size_t ws_bytes, hipStream_t st) {
  if (H < 1 || k < 1) return fail(PKMEM_ERR_INVALID, "%s: H and k must be >= 1", fn);
  int rc = check_bag_shapes(fn, v_dt, N, D, T, H * k);
  if (rc) return rc;
  if (mode != PKMEM_BWD_AUTO && mode != PKMEM_BWD_ATOMIC && mode != PKMEM_BWD_SORTED)
    return fail(PKMEM_ERR_INVALID, "%s: unknown mode %d", fn, mode);
  const bool sparse = rows_out != nullptr || num_rows_out != nullptr;
  const int m = sparse ? PKMEM_BWD_SORTED : resolve_mode(mode, D, T * H * (int64_t)k);
  if (T > 0 && (!dy || !values || !idx || !w))
    return fail(PKMEM_ERR_INVALID, "%s: null input pointer", fn);
  if (!aligned(dy, 16) || !aligned(values, 16))
    return fail(PKMEM_ERR_INVALID, "%s: dy and values must be 16-byte aligned", fn);
  if (grad_values && !aligned(grad_values, 16))
    return fail(PKMEM_ERR_INVALID, "%s: grad_values must be 16-byte aligned", fn);
  const int64_t L = T * H * k;
  if (sparse) {
    if (!rows_out || !grad_rows_out || !num_rows_out)
      return fail(PKMEM_ERR_INVALID, "%s: rows_out, grad_rows_out and num_rows_out are required", fn);
    if (!aligned(grad_rows_out, 16)) return fail(PKMEM_ERR_INVALID, "%s: grad_rows_out must be 16-byte aligned", fn);
    const int64_t need = L < N ? L : N;
    if (cap < need)
      return fail(PKMEM_ERR_INVALID, "%s: cap %lld < min(T*H*k, N) = %lld", fn, (long long)cap, (long long)need);
  }
  const size_t need_ws = bwd_ws_bytes(T, H, k, D, m);
  if (!ws || ws_bytes < need_ws)
    return fail(PKMEM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need_ws, ws ? ws_bytes : (size_t)0);
  if (!aligned(ws, 256)) return fail(PKMEM_ERR_INVALID, "%s: workspace must be 256-byte aligned", fn);
  if (sparse) *num_rows_out = 0;
  if (T == 0) return PKMEM_OK;
  rc = check_indices(fn, idx, L, N, st);
  if (rc) return rc;

  char* p = reinterpret_cast<char*>(ws);
  float* gw = grad_w ? grad_w : reinterpret_cast<float*>(p);
  p += align256((size_t)L * sizeof(float));
  const bool bf16 = v_dt == PKMEM_BF16;
  hipError_t e;
  if (m == PKMEM_BWD_ATOMIC) {
    e = pk::launch_bag_backward_atomic(bf16, dy, values, D, idx, w, T, H * k, grad_values, gw, st);
    if (e != hipSuccess) return hip_status(e, fn);
  } else {
    uint32_t* nrows_dev = nullptr;
    float* part = reinterpret_cast<float*>(p + pk::sorted_workspace_bytes(L));
    e = pk::launch_bag_backward_sorted(bf16, dy, values, N, D, idx, w, T, H * k,
                                       sparse ? nullptr : grad_values, sparse ? rows_out : nullptr,
                                       grad_rows_out, gw, p, part, &nrows_dev, st);
    if (e != hipSuccess) return hip_status(e, fn);
    if (sparse) {
      uint32_t U = 0;
      e = hipMemcpyAsync(&U, nrows_dev, sizeof(U), hipMemcpyDeviceToHost, st);
      if (e == hipSuccess) e = hipStreamSynchronize(st);
      if (e != hipSuccess) return hip_status(e, fn);
      *num_rows_out = U;
    }
  }
  if (grad_scores) {
    e = pk::launch_softmax_backward(w, gw, T * H, k, grad_scores, st);
    if (e != hipSuccess) return hip_status(e, fn);
  }
  return PKMEM_OK;
}

// Benchmark timer state (host side, single-threaded use).
struct TimedLaunch {
  int kernel;  // position of the kernel's name in the timer's list
  hipEvent_t start, stop;
};
struct TimerState {
  std::vector<std::string> names;
  bool on = false;
  std::vector<TimedLaunch> events;
};
TimerState g_timer;

int timer_slot(const char* name) {
  for (size_t i = 0; i < g_timer.names.size(); ++i)
    if (g_timer.names[i] == name) return (int)i;
  return -1;
}

}  // namespace

namespace pk {

LaunchTimer::LaunchTimer(const char* name, hipStream_t st) : st_(st) {
  if (!g_timer.on) return;
  const int slot = timer_slot(name);
  if (slot < 0) return;
  hipEvent_t a, b;
  if (hipEventCreate(&a) != hipSuccess) return;
  if (hipEventCreate(&b) != hipSuccess) { (void)hipEventDestroy(a); return; }
  if (hipEventRecord(a, st_) != hipSuccess) {
    (void)hipEventDestroy(a);
    (void)hipEventDestroy(b);
    return;
  }
  stop_ = b;
  g_timer.events.push_back({slot, a, b});
}

LaunchTimer::~LaunchTimer() {
  if (stop_) (void)hipEventRecord(stop_, st_);
}

}  // namespace pk

extern "C" {

int mem_timer_start(const char* kernels) {
  if (!kernels) return fail(PKMEM_ERR_INVALID, "mem_timer_start: null kernel list");
  g_timer.names.clear();
  std::string cur;
  for (const char* c = kernels;; ++c) {
    if (*c == ',' || *c == '\0') {
      if (!cur.empty()) g_timer.names.push_back(cur);
      cur.clear();
      if (*c == '\0') break;
    } else if (*c != ' ') {
      cur.push_back(*c);
    }
  }
  g_timer.on = !g_timer.names.empty();
  return PKMEM_OK;
}

int mem_timer_stop(void) {
  g_timer.on = false;
  return PKMEM_OK;
}

int mem_timer_read(float* ms_out, int* kernel_out, int cap) {
  int n = 0;
  hipError_t err = hipSuccess;
  for (auto& ev : g_timer.events) {
    float ms = 0.f;
    hipError_t e = hipEventSynchronize(ev.stop);
    if (e == hipSuccess) e = hipEventElapsedTime(&ms, ev.start, ev.stop);
    if (e != hipSuccess && err == hipSuccess) err = e;
    if (n < cap) {
      if (ms_out) ms_out[n] = ms;
      if (kernel_out) kernel_out[n] = ev.kernel;
    }
    ++n;
    (void)hipEventDestroy(ev.start);
    (void)hipEventDestroy(ev.stop);
  }
  g_timer.events.clear();
  if (err != hipSuccess) return hip_status(err, "mem_timer_read");
  return n;
}

const char* mem_last_error(void) { return g_last_error.c_str(); }

int mem_version(void) { return 1; }

size_t mem_search_workspace_size(int64_t T, int H, int S, int k) {
  (void)S;
  if (T < 0 || H < 1 || k < 1) return 0;
  return search_ws(nullptr, T, H, k).bytes;
}

// The search, with the queries normalised (qnorm) or not.
static int search_common(const char* fn, const void* q, pkmem_dtype q_dt, const void* subkeys,
                         pkmem_dtype k_dt, int64_t T, int H, int n, int S, int k, bool qnorm,
                         float eps, int nex, const int64_t* ex_idx, bool has_sink,
                         const void* sink, int64_t sink_row0, int64_t* idx_out, float* w_out, float* score_out,
                         int32_t* half_idx_out, void* qhat_out, float* stats_out, void* ws,
                         size_t ws_bytes, pkmem_stream_t stream) {
  int rc = check_search_shapes(fn, q, q_dt, subkeys, k_dt, T, H, n, S, k);
  if (rc) return rc;
  if (nex < 0) return fail(PKMEM_ERR_INVALID, "%s: r must be >= 0", fn);
  if (k + nex + (has_sink ? 1 : 0) > PKMEM_KMAX)
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: k + r%s must be <= %d (k=%d, r=%d)", fn,
                has_sink ? " + 1" : "", PKMEM_KMAX, k, nex);
  if (has_sink) {
    if (T > 0 && !sink) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
    if (!aligned(sink, 16)) return fail(PKMEM_ERR_INVALID, "%s: sink_keys must be 16-byte aligned", fn);
    if (sink_row0 < (int64_t)S * S || sink_row0 > INT64_MAX - H)
      return fail(PKMEM_ERR_INVALID, "%s: sink_row0 must be >= S*S = %lld (got %lld)", fn,
                  (long long)S * S, (long long)sink_row0);
  }
  if (T > 0 && nex > 0 && !ex_idx) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (T > 0 && (!idx_out || !w_out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (qnorm && !(eps >= 0.f && eps <= 3.0e38f))
    return fail(PKMEM_ERR_INVALID, "%s: eps must be finite and >= 0", fn);
  if (!aligned(qhat_out, 16) || !aligned(stats_out, 8))
    return fail(PKMEM_ERR_INVALID, "%s: qhat_out must be 16-byte and stats_out 8-byte aligned", fn);
  const SearchWs need = search_ws(nullptr, T, H, k);
  if (!ws || ws_bytes < need.bytes)
    return fail(PKMEM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need.bytes, ws ? ws_bytes : (size_t)0);
  if (!aligned(ws, 256)) return fail(PKMEM_ERR_INVALID, "%s: workspace must be 256-byte aligned", fn);
  if (T == 0) return PKMEM_OK;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  SearchWs w = search_ws(ws, T, H, k);
  const bool bf16 = q_dt == PKMEM_BF16;
  float2* qstats = nullptr;
  hipError_t e = hipSuccess;
  if (qnorm) {
    qstats = stats_out ? reinterpret_cast<float2*>(stats_out) : w.qstats;
    e = pk::launch_qnorm(bf16, q, T * H, n, eps, qstats, qhat_out, st);
    if (e != hipSuccess) return hip_status(e, fn);
  }
  int32_t* hidx = half_idx_out ? half_idx_out : w.half_idx;
  pk::SplitPlan plan{0, 0, 0, 0};  // parts = 0: half lists, no part records
  if (pk::split_plan(bf16, T, H, n, S, k, &plan))
    e = pk::launch_search_split(bf16, q, subkeys, T, H, n, S, k, qstats, has_sink ? sink : nullptr,
                                w.sink_part, plan, w.cand, st);
  else
    e = pk::launch_search_half(bf16, q, subkeys, T, H, n, S, k, qstats, has_sink ? sink : nullptr,
                               w.sink_part, w.cand, w.cnts, w.thr, hidx, w.half_score, w.ovf, st);
  if (e != hipSuccess) return hip_status(e, fn);
  if (nex > 0) {
    rc = check_indices(fn, ex_idx, T * H * nex, (int64_t)S * S, st);
    if (rc) return rc;
  }
  e = pk::launch_cartesian(hidx, w.half_score, w.cand, plan, half_idx_out, T, H, S, k, bf16, q,
                           subkeys, n, ex_idx, nex, has_sink ? w.sink_part : nullptr, sink_row0,
                           idx_out, w_out, score_out, st);
  if (e != hipSuccess) return hip_status(e, fn);
  return PKMEM_OK;
}

int mem_search(const void* q, pkmem_dtype q_dt, const void* subkeys, pkmem_dtype k_dt, int64_t T,
               int H, int n, int S, int k, int64_t* idx_out, float* w_out, float* score_out,
               int32_t* half_idx_out, void* ws, size_t ws_bytes, pkmem_stream_t stream) {
  return search_common("mem_search", q, q_dt, subkeys, k_dt, T, H, n, S, k, false, 0.f, 0, nullptr,
                       false, nullptr, 0, idx_out, w_out, score_out, half_idx_out, nullptr, nullptr, ws, ws_bytes,
                       stream);
}

}  // extern "C"

// Workspace of mem_search_noalloc: one array per GPU, part of the library's
// code object, held until the process ends.  Host code never uses its name as
// an address: the device address comes from hipGetSymbolAddress, looked up
// once per device with that device current.
static __device__ __align__(256) unsigned char scratch[PKMEM_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int SCRATCH_DEVICES = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[SCRATCH_DEVICES] = {};

// The current device's address of the scratch array (looked up at the first
// call on that device).
int scratch_on_current_device(const char* fn, void** out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_status(e, fn);
  if (dev < 0 || dev >= SCRATCH_DEVICES) return fail(PKMEM_ERR_UNSUPPORTED, "%s: device %d", fn, dev);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return hip_status(e, fn);
    if (!p) return fail(PKMEM_ERR_HIP, "%s: no device address for the scratch array", fn);
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return PKMEM_OK;
}

}  // namespace

extern "C" {

int mem_search_noalloc(const void* q, pkmem_dtype q_dt, const void* subkeys, pkmem_dtype k_dt,
                       int64_t T, int H, int n, int S, int k, int64_t* idx_out, float* w_out,
                       float* score_out, int32_t* half_idx_out, pkmem_stream_t stream) {
  const char* fn = "mem_search_noalloc";
  int rc = check_search_shapes(fn, q, q_dt, subkeys, k_dt, T, H, n, S, k);
  if (rc) return rc;
  const size_t need = search_ws(nullptr, T, H, k).bytes;
  if (need > PKMEM_NOALLOC_SCRATCH_BYTES)
    return fail(PKMEM_ERR_UNSUPPORTED,
                "%s: T=%lld, H=%d, k=%d needs %zu bytes of scratch, more than its %zu "
                "(use mem_search with a workspace)",
                fn, (long long)T, H, k, need, (size_t)PKMEM_NOALLOC_SCRATCH_BYTES);
  if (T > 0 && (!idx_out || !w_out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (T == 0) return PKMEM_OK;
  void* ws = nullptr;
  rc = scratch_on_current_device(fn, &ws);
  if (rc) return rc;
  return search_common(fn, q, q_dt, subkeys, k_dt, T, H, n, S, k, false, 0.f, 0, nullptr, false,
                       nullptr, 0, idx_out, w_out, score_out, half_idx_out, nullptr, nullptr, ws,
                       PKMEM_NOALLOC_SCRATCH_BYTES, stream);
}

int mem_search_qnorm(const void* q, pkmem_dtype q_dt, const void* subkeys, pkmem_dtype k_dt,
                     int64_t T, int H, int n, int S, int k, float eps, int64_t* idx_out,
                     float* w_out, float* score_out, int32_t* half_idx_out, void* qhat_out,
                     float* stats_out, void* ws, size_t ws_bytes, pkmem_stream_t stream) {
  return search_common("mem_search_qnorm", q, q_dt, subkeys, k_dt, T, H, n, S, k, true, eps, 0,
                       nullptr, false, nullptr, 0, idx_out, w_out, score_out, half_idx_out, qhat_out, stats_out, ws,
                       ws_bytes, stream);
}

int mem_search_extra(const void* q, pkmem_dtype q_dt, const void* subkeys, pkmem_dtype k_dt,
                     int64_t T, int H, int n, int S, int k, int r, const int64_t* extra_idx,
                     int64_t* idx_out, float* w_out, float* score_out, int32_t* half_idx_out,
                     void* ws, size_t ws_bytes, pkmem_stream_t stream) {
  return search_common("mem_search_extra", q, q_dt, subkeys, k_dt, T, H, n, S, k, false, 0.f, r,
                       extra_idx, false, nullptr, 0, idx_out, w_out, score_out, half_idx_out, nullptr,
                       nullptr, ws, ws_bytes, stream);
}

int mem_search_sink(const void* q, pkmem_dtype q_dt, const void* subkeys, pkmem_dtype k_dt,
                    int64_t T, int H, int n, int S, int k, int r, const int64_t* extra_idx,
                    const void* sink_keys, int64_t sink_row0, int64_t* idx_out, float* w_out,
                    float* score_out, int32_t* half_idx_out, void* ws, size_t ws_bytes,
                    pkmem_stream_t stream) {
  return search_common("mem_search_sink", q, q_dt, subkeys, k_dt, T, H, n, S, k, false, 0.f, r,
                       extra_idx, true, sink_keys, sink_row0, idx_out, w_out, score_out,
                       half_idx_out, nullptr, nullptr, ws, ws_bytes, stream);
}

size_t mem_search_backward_workspace_size(int64_t T, int H, int S, int k) {
  (void)S;
  if (T < 0 || H < 1 || k < 1) return 0;
  // the sort and its inputs, then the queries' (mean, rstd) for the normalised variant
  return pk::search_backward_ws_bytes(T, H, k) + align256((size_t)T * H * sizeof(float2));
}

size_t mem_search_backward_sink_workspace_size(int64_t T, int H, int n, int S, int k) {
  (void)S;
  if (T < 0 || H < 1 || n < 2 || k < 1) return 0;
  // the sort and its inputs, then the per-chunk partial sums of grad_sink
  return pk::search_backward_ws_bytes(T, H, k) +
         align256((size_t)pk::sink_chunks(T) * H * n * sizeof(float));
}

// k: product-key slots per row.  With a sink the rows of idx and grad_scores
// hold k + 1 slots, the last the sink's.
static int search_backward_common(const char* fn, const void* q, pkmem_dtype q_dt,
                                  const void* subkeys, pkmem_dtype k_dt, int64_t T, int H, int n,
                                  int S, int k, bool qnorm, float eps, const int64_t* idx,
                                  const float* grad_scores, bool has_sink, const void* sink,
                                  float* grad_q, float* grad_subkeys, float* grad_sink, void* ws,
                                  size_t ws_bytes, pkmem_stream_t stream) {
  int rc = check_search_shapes(fn, q, q_dt, subkeys, k_dt, T, H, n, S, k, true);
  if (rc) return rc;
  if (k > PKMEM_KMAX - (has_sink ? 1 : 0))
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: more than %d slots per row", fn, PKMEM_KMAX);
  if (has_sink) {
    if (T > 0 && (grad_q || grad_sink) && !sink) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
    if (!aligned(sink, 16) || !aligned(grad_sink, 4))
      return fail(PKMEM_ERR_INVALID, "%s: sink_keys must be 16-byte and grad_sink 4-byte aligned", fn);
  }
  if (T > 0 && (!idx || !grad_scores)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (qnorm && !(eps >= 0.f && eps <= 3.0e38f))
    return fail(PKMEM_ERR_INVALID, "%s: eps must be finite and >= 0", fn);
  if (2 * T * (int64_t)H * k >= (int64_t(1) << 32))
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: 2*T*H*k must be < 2^32", fn);
  if (2 * (int64_t)H * S >= (int64_t(1) << 31))
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: 2*H*S must be < 2^31", fn);
  if (!aligned(grad_subkeys, 16) || !aligned(grad_q, 4))
    return fail(PKMEM_ERR_INVALID, "%s: grad_subkeys must be 16-byte and grad_q 4-byte aligned", fn);
  const size_t need = has_sink ? mem_search_backward_sink_workspace_size(T, H, n, S, k)
                               : mem_search_backward_workspace_size(T, H, S, k);
  if (!ws || ws_bytes < need)
    return fail(PKMEM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
  if (!aligned(ws, 256)) return fail(PKMEM_ERR_INVALID, "%s: workspace must be 256-byte aligned", fn);
  if (T == 0 || (!grad_q && !grad_subkeys && !grad_sink)) return PKMEM_OK;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const int kst = k + (has_sink ? 1 : 0);
  rc = check_indices_strided(fn, idx, T * H, k, kst, (int64_t)S * S, st);
  if (rc) return rc;
  const bool bf16 = q_dt == PKMEM_BF16;
  float2* qstats = nullptr;
  if (qnorm) {
    qstats = reinterpret_cast<float2*>(reinterpret_cast<char*>(ws) +
                                       pk::search_backward_ws_bytes(T, H, k));
    hipError_t e = pk::launch_qnorm(bf16, q, T * H, n, eps, qstats, nullptr, st);
    if (e != hipSuccess) return hip_status(e, fn);
  }
  float* sink_part = has_sink ? reinterpret_cast<float*>(reinterpret_cast<char*>(ws) +
                                                        pk::search_backward_ws_bytes(T, H, k))
                              : nullptr;
  hipError_t e = pk::launch_search_backward(bf16, q, subkeys, T, H, n, S, k, kst, idx, grad_scores,
                                            qstats, has_sink ? sink : nullptr, grad_q,
                                            grad_subkeys, has_sink ? grad_sink : nullptr,
                                            sink_part, ws, st);
  return hip_status(e, fn);
}

int mem_search_backward(const void* q, pkmem_dtype q_dt, const void* subkeys, pkmem_dtype k_dt,
                        int64_t T, int H, int n, int S, int k, const int64_t* idx,
                        const float* grad_scores, float* grad_q, float* grad_subkeys, void* ws,
                        size_t ws_bytes, pkmem_stream_t stream) {
  return search_backward_common("mem_search_backward", q, q_dt, subkeys, k_dt, T, H, n, S, k,
                                false, 0.f, idx, grad_scores, false, nullptr, grad_q, grad_subkeys,
                                nullptr, ws, ws_bytes, stream);
}

int mem_search_backward_sink(const void* q, pkmem_dtype q_dt, const void* subkeys,
                             pkmem_dtype k_dt, int64_t T, int H, int n, int S, int k,
                             const int64_t* idx, const float* grad_scores, const void* sink_keys,
                             float* grad_q, float* grad_subkeys, float* grad_sink, void* ws,
                             size_t ws_bytes, pkmem_stream_t stream) {
  return search_backward_common("mem_search_backward_sink", q, q_dt, subkeys, k_dt, T, H, n, S, k,
                                false, 0.f, idx, grad_scores, true, sink_keys, grad_q,
                                grad_subkeys, grad_sink, ws, ws_bytes, stream);
}

int mem_search_backward_qnorm(const void* q, pkmem_dtype q_dt, const void* subkeys,
                              pkmem_dtype k_dt, int64_t T, int H, int n, int S, int k, float eps,
                              const int64_t* idx, const float* grad_scores, float* grad_q,
                              float* grad_subkeys, void* ws, size_t ws_bytes,
                              pkmem_stream_t stream) {
  return search_backward_common("mem_search_backward_qnorm", q, q_dt, subkeys, k_dt, T, H, n, S,
                                k, true, eps, idx, grad_scores, false, nullptr, grad_q,
                                grad_subkeys, nullptr, ws, ws_bytes, stream);
}

int mem_bag_forward(const void* values, pkmem_dtype v_dt, int64_t N, int D, const int64_t* idx,
                    const float* w, int64_t T, int bag, void* y_out, pkmem_stream_t stream) {
  const char* fn = "mem_bag_forward";
  int rc = check_bag_shapes(fn, v_dt, N, D, T, bag);
  if (rc) return rc;
  if (T > 0 && (!values || !idx || !w || !y_out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(values, 16) || !aligned(y_out, 16)) return fail(PKMEM_ERR_INVALID, "%s: values and y_out must be 16-byte aligned", fn);
  if (T == 0) return PKMEM_OK;
  rc = check_indices(fn, idx, T * bag, N, reinterpret_cast<hipStream_t>(stream));
  if (rc) return rc;
  hipError_t e = pk::launch_bag_forward(v_dt == PKMEM_BF16, values, D, idx, w, T, bag, y_out, nullptr, nullptr,
                                        reinterpret_cast<hipStream_t>(stream));
  return hip_status(e, fn);
}

int mem_bag_forward_gated(const void* values, pkmem_dtype v_dt, int64_t N, int D, const int64_t* idx,
                          const float* w, int64_t T, int bag, const void* gate, void* y_out,
                          void* out, pkmem_stream_t stream) {
  const char* fn = "mem_bag_forward_gated";
  int rc = check_bag_shapes(fn, v_dt, N, D, T, bag);
  if (rc) return rc;
  if (T > 0 && (!values || !idx || !w || !gate || !out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(values, 16) || !aligned(gate, 16) || !aligned(out, 16) || !aligned(y_out, 16))
    return fail(PKMEM_ERR_INVALID, "%s: values, gate, y_out and out must be 16-byte aligned", fn);
  if (T == 0) return PKMEM_OK;
  rc = check_indices(fn, idx, T * bag, N, reinterpret_cast<hipStream_t>(stream));
  if (rc) return rc;
  hipError_t e = pk::launch_bag_forward(v_dt == PKMEM_BF16, values, D, idx, w, T, bag, out, gate,
                                        y_out, reinterpret_cast<hipStream_t>(stream));
  return hip_status(e, fn);
}

int mem_gate_backward(const void* d_out, const void* gate, const void* y, pkmem_dtype v_dt, int64_t T,
                      int D, void* dy_out, float* grad_gate, pkmem_stream_t stream) {
  const char* fn = "mem_gate_backward";
  if (!dtype_ok(v_dt)) return fail(PKMEM_ERR_INVALID, "%s: unknown dtype %d", fn, (int)v_dt);
  if (T < 0) return fail(PKMEM_ERR_INVALID, "%s: T must be >= 0", fn);
  if (D < 8 || D % 8 != 0) return fail(PKMEM_ERR_UNSUPPORTED, "%s: D must be a positive multiple of 8 (got %d)", fn, D);
  if (T > 0 && (!d_out || !gate || !y || !dy_out || !grad_gate)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(d_out, 16) || !aligned(gate, 16) || !aligned(y, 16) || !aligned(dy_out, 16) || !aligned(grad_gate, 16))
    return fail(PKMEM_ERR_INVALID, "%s: every buffer must be 16-byte aligned", fn);
  if (T == 0) return PKMEM_OK;
  hipError_t e = pk::launch_gate_backward(v_dt == PKMEM_BF16, d_out, gate, y, T, D, dy_out, grad_gate,
                                          reinterpret_cast<hipStream_t>(stream));
  return hip_status(e, fn);
}

size_t mem_bag_backward_workspace_size(int64_t T, int H, int k, int64_t N, int D, int mode) {
  (void)N;
  if (T < 0 || H < 1 || k < 1) return 0;
  return bwd_ws_bytes(T, H, k, D, resolve_mode(mode, D, T * H * (int64_t)k));
}

int mem_bag_backward(const void* dy, const void* values, pkmem_dtype v_dt, int64_t N, int D,
                     const int64_t* idx, const float* w, int64_t T, int H, int k,
                     float* grad_values, float* grad_w, float* grad_scores, int mode, void* ws,
                     size_t ws_bytes, pkmem_stream_t stream) {
  const char* fn = "mem_bag_backward";
  return bag_backward_common(fn, dy, values, v_dt, N, D, idx, w, T, H, k, grad_values, nullptr,
                             nullptr, 0, nullptr, grad_w, grad_scores, mode, ws, ws_bytes,
                             reinterpret_cast<hipStream_t>(stream));
}

int mem_bag_backward_sparse(const void* dy, const void* values, pkmem_dtype v_dt, int64_t N, int D,
                            const int64_t* idx, const float* w, int64_t T, int H, int k,
                            int64_t* rows_out, float* grad_rows_out, int64_t cap,
                            int64_t* num_rows_out, float* grad_w, float* grad_scores, void* ws,
                            size_t ws_bytes, pkmem_stream_t stream) {
  const char* fn = "mem_bag_backward_sparse";
  if (!rows_out || !grad_rows_out || !num_rows_out)
    return fail(PKMEM_ERR_INVALID, "%s: rows_out, grad_rows_out and num_rows_out are required", fn);
  return bag_backward_common(fn, dy, values, v_dt, N, D, idx, w, T, H, k, nullptr, rows_out,
                             grad_rows_out, cap, num_rows_out, grad_w, grad_scores,
                             PKMEM_BWD_SORTED, ws, ws_bytes, reinterpret_cast<hipStream_t>(stream));
}

}  // extern "C"

// ---- norm and optimizer ------------------------------------------------------

namespace {

constexpr size_t NORM_ROW_BYTES = 32 << 10;  // a row fits the registers of one workgroup

struct Bytes {
  const void* p;
  size_t n;
};

bool share(const Bytes& a, const Bytes& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x && y && a.n && b.n && x < y + b.n && y < x + a.n;
}

// Does an output share bytes with one of the buffers `apart`, or with one of `in_place`
// that it is not itself?  Other workgroups may still read what it would overwrite.
bool over(const Bytes& out, std::initializer_list<Bytes> apart, std::initializer_list<Bytes> in_place = {}) {
  for (const Bytes& b : apart)
    if (share(out, b)) return true;
  for (const Bytes& b : in_place)
    if (share(out, b) && !(out.p == b.p && out.n == b.n)) return true;
  return false;
}

int check_rows_shape(const char* fn, pkmem_dtype dt, int64_t T, int D) {
  if (!dtype_ok(dt)) return fail(PKMEM_ERR_INVALID, "%s: unknown dtype %d", fn, (int)dt);
  if (T < 0) return fail(PKMEM_ERR_INVALID, "%s: the number of rows must be >= 0", fn);
  if (T > 0x7FFFFFFF) return fail(PKMEM_ERR_UNSUPPORTED, "%s: 2^31 rows or more", fn);
  if (D < 8 || D % 8 != 0)
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: rows must be a positive multiple of 8 wide (got %d)", fn, D);
  if ((size_t)D * esize(dt) > NORM_ROW_BYTES)
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: rows wider than 32 KiB are not supported (%d)", fn, D);
  return PKMEM_OK;
}

int check_adamw_opts(const char* fn, const pkmem_adamw_opts* o) {
  if (!o) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1))
    return fail(PKMEM_ERR_INVALID, "%s: betas must lie in [0, 1)", fn);
  if (!(o->lr >= 0 && o->lr <= 3e38 && o->eps >= 0 && o->eps <= 3e38 && o->weight_decay >= 0 &&
        o->weight_decay <= 3e38))
    return fail(PKMEM_ERR_INVALID, "%s: lr, eps and weight_decay must be finite and >= 0", fn);
  if (o->step < 1 && !o->step_dev) return fail(PKMEM_ERR_INVALID, "%s: step must be >= 1", fn);
  if (!aligned(o->lr_dev, 4) || !aligned(o->step_dev, 8) || !aligned(o->grad_scale, 4))
    return fail(PKMEM_ERR_INVALID, "%s: lr_dev, step_dev and grad_scale must be aligned to their size", fn);
  return PKMEM_OK;
}

// graded: gradients are there (a list of touched rows may be empty).
int check_adamw_tensor(const char* fn, const pkmem_adamw_tensor& t, int i, bool graded) {
  if (!dtype_ok(t.param_dt) || !dtype_ok(t.grad_dt) ||
      (t.state_dt != PKMEM_F32 && t.state_dt != PKMEM_E4M3))
    return fail(PKMEM_ERR_INVALID, "%s: tensor %d: unsupported dtype", fn, i);
  if (t.numel < 0) return fail(PKMEM_ERR_INVALID, "%s: tensor %d: numel must be >= 0", fn, i);
  if (t.numel > (int64_t(1) << 40)) return fail(PKMEM_ERR_UNSUPPORTED, "%s: tensor %d: more than 2^40 elements", fn, i);
  const bool s8 = t.state_dt == PKMEM_E4M3;
  if (t.numel > 0 && (!t.param || (graded && !t.grad) || !t.exp_avg || !t.exp_avg_sq ||
                      (s8 && (!t.exp_avg_scale || !t.exp_avg_sq_scale))))
    return fail(PKMEM_ERR_INVALID, "%s: tensor %d: null pointer", fn, i);
  const size_t se = s8 ? 1 : 4;
  if (!aligned(t.param, esize(t.param_dt)) || !aligned(t.grad, esize(t.grad_dt)) ||
      !aligned(t.exp_avg, se) || !aligned(t.exp_avg_sq, se) ||
      (s8 && (!aligned(t.exp_avg_scale, 4) || !aligned(t.exp_avg_sq_scale, 4))))
    return fail(PKMEM_ERR_INVALID, "%s: tensor %d: not aligned to its element size", fn, i);
  return PKMEM_OK;
}

// Does a buffer that a step writes overlap another that it writes or reads?  A
// parameter listed twice would be written by two workgroups at once, a state over a
// gradient be overwritten before another workgroup reads it.  rows: mem_adamw_rows's list.
int check_adamw_overlap(const char* fn, const pkmem_adamw_tensor* ts, int count, const pkmem_adamw_opts& o,
                        size_t grad_elems = 0, Bytes rows = {}) {
  struct Span { uintptr_t begin, end; int i; bool write; };
  constexpr int EACH = 6, MORE = 4, FEW = 16;
  Span few[EACH * FEW + MORE];
  Span* s = count <= FEW ? few : static_cast<Span*>(malloc(sizeof(Span) * (EACH * (size_t)count + MORE)));
  if (!s) return fail(PKMEM_ERR_UNSUPPORTED, "%s: no host memory for a list of %d", fn, count);
  size_t n = 0;
  auto add = [&](const void* p, size_t bytes, int i, bool write) {
    if (p && bytes) s[n++] = Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, i, write};
  };
  for (int i = 0; i < count; ++i) {
    const pkmem_adamw_tensor& t = ts[i];
    if (t.numel == 0) continue;
    const bool s8 = t.state_dt == PKMEM_E4M3;
    const size_t e = (size_t)t.numel, state = e * (s8 ? 1 : 4);
    const size_t scale = s8 ? (e + pk::ADAMW_STATE_BLOCK - 1) / pk::ADAMW_STATE_BLOCK * 4 : 0;
    add(t.param, e * esize(t.param_dt), i, true);
    add(t.exp_avg, state, i, true);
    add(t.exp_avg_sq, state, i, true);
    add(t.exp_avg_scale, scale, i, true);
    add(t.exp_avg_sq_scale, scale, i, true);
    add(t.grad, (rows.p ? grad_elems : e) * esize(t.grad_dt), i, false);
  }
  add(o.lr_dev, 4, -1, false);
  add(o.step_dev, 8, -1, false);
  add(o.grad_scale, 4, -1, false);
  add(rows.p, rows.n, -1, false);
  std::sort(s, s + n, [](const Span& a, const Span& b) { return a.begin < b.begin; });
  // the furthest ends of what is written and of what is read so far
  Span wrote{0, 0, -1, true}, read{0, 0, -1, false};
  int a = -2, b = -2;
  bool both = false;
  for (size_t i = 0; i < n && a == -2; ++i) {
    if (s[i].begin < wrote.end) a = wrote.i, b = s[i].i, both = s[i].write;
    else if (s[i].write && s[i].begin < read.end) a = s[i].i, b = read.i;
    Span& last = s[i].write ? wrote : read;
    if (s[i].end > last.end) last = s[i];
  }
  if (s != few) free(s);
  if (a == -2) return PKMEM_OK;
  if (both)
    return fail(PKMEM_ERR_INVALID, "%s: parameters or states of tensors %d and %d overlap", fn, a < b ? a : b, a < b ? b : a);
  return b < 0 ? fail(PKMEM_ERR_INVALID, "%s: a parameter or state of tensor %d overlaps a device scalar or the list of rows", fn, a)
               : fail(PKMEM_ERR_INVALID, "%s: a parameter or state of tensor %d overlaps the gradient of tensor %d", fn, a, b);
}

}  // namespace

extern "C" {

int mem_rmsnorm(const void* x, const void* res, const void* weight, pkmem_dtype dt, int64_t T,
                int D, float eps, void* sum_out, void* y_out, pkmem_dtype y_dt, float* scale_out,
                pkmem_stream_t stream) {
  const char* fn = "mem_rmsnorm";
  int rc = check_rows_shape(fn, dt, T, D);
  if (rc) return rc;
  if (y_dt != dt && y_dt != PKMEM_E4M3)
    return fail(PKMEM_ERR_INVALID, "%s: y_dt must be the row dtype or PKMEM_E4M3", fn);
  if (!(eps >= 0.f && eps <= 3.0e38f)) return fail(PKMEM_ERR_INVALID, "%s: eps must be finite and >= 0", fn);
  const bool q = y_dt == PKMEM_E4M3;
  if (T > 0 && (!x || !y_out || (q && !scale_out))) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!q && scale_out) return fail(PKMEM_ERR_INVALID, "%s: scale_out is for PKMEM_E4M3 only", fn);
  if (sum_out && sum_out == y_out) return fail(PKMEM_ERR_INVALID, "%s: sum_out and y_out are one buffer", fn);
  if (!aligned(x, 16) || !aligned(res, 16) || !aligned(weight, 16) || !aligned(sum_out, 16) ||
      !aligned(y_out, 16) || !aligned(scale_out, 4))
    return fail(PKMEM_ERR_INVALID, "%s: buffers must be 16-byte aligned (scale_out 4)", fn);
  if (T == 0) return PKMEM_OK;
  const size_t rows = (size_t)T * D * esize(dt);
  const Bytes bx{x, rows}, br{res, rows}, bw{weight, D * esize(dt)}, bs{sum_out, rows}, bc{scale_out, (size_t)T * 4},
      by{y_out, q ? (size_t)T * D : rows};
  if (over(bs, {bw, by, bc}, {bx, br}) || over(by, {bw, bc}, {bx, br}) || over(bc, {bx, br, bw}))
    return fail(PKMEM_ERR_INVALID, "%s: an output may not be weight or share bytes with another buffer (but be x or res itself, y_out in 8 bits not even that)", fn);
  return hip_status(pk::launch_rmsnorm(dt == PKMEM_BF16, x, res, weight, T, D, eps, sum_out, y_out,
                                       scale_out, reinterpret_cast<hipStream_t>(stream)), fn);
}

size_t mem_rmsnorm_backward_workspace_size(int64_t T, int D) {
  if (T < 0 || D < 1) return 0;
  return align256(pk::rmsnorm_backward_ws_bytes(T, D));
}

int mem_rmsnorm_backward(const void* dy, const void* h, const void* weight, pkmem_dtype dt,
                         int64_t T, int D, float eps, const void* dsum, void* dx_out,
                         float* grad_weight, void* ws, size_t ws_bytes, pkmem_stream_t stream) {
  const char* fn = "mem_rmsnorm_backward";
  int rc = check_rows_shape(fn, dt, T, D);
  if (rc) return rc;
  if (!(eps >= 0.f && eps <= 3.0e38f)) return fail(PKMEM_ERR_INVALID, "%s: eps must be finite and >= 0", fn);
  if (T > 0 && (!dy || !h || !dx_out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(dy, 16) || !aligned(h, 16) || !aligned(weight, 16) || !aligned(dsum, 16) ||
      !aligned(dx_out, 16) || !aligned(grad_weight, 4))
    return fail(PKMEM_ERR_INVALID, "%s: buffers must be 16-byte aligned (grad_weight 4)", fn);
  if (grad_weight) {
    const size_t need = mem_rmsnorm_backward_workspace_size(T, D);
    if (need > 0 && (!ws || ws_bytes < need))
      return fail(PKMEM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned(ws, 256)) return fail(PKMEM_ERR_INVALID, "%s: workspace must be 256-byte aligned", fn);
  }
  if (T == 0) return PKMEM_OK;
  const size_t rows = (size_t)T * D * esize(dt);
  const Bytes bdy{dy, rows}, bh{h, rows}, bd{dsum, rows}, bx{dx_out, rows}, bw{weight, D * esize(dt)},
      bg{grad_weight, (size_t)D * 4}, bws{grad_weight ? ws : nullptr, mem_rmsnorm_backward_workspace_size(T, D)};
  if (over(bx, {bw, bg, bws}, {bdy, bh, bd}) || over(bg, {bdy, bh, bd, bw, bws}) || over(bws, {bdy, bh, bd, bw}))
    return fail(PKMEM_ERR_INVALID, "%s: dx_out may be dy, h or dsum itself; outputs and workspace may share no other bytes", fn);
  return hip_status(pk::launch_rmsnorm_backward(dt == PKMEM_BF16, dy, h, weight, dsum, T, D, eps,
                                                dx_out, grad_weight, reinterpret_cast<float*>(ws),
                                                reinterpret_cast<hipStream_t>(stream)), fn);
}

int mem_quantize_rows(const void* x, pkmem_dtype dt, int64_t R, int C, void* q_out,
                      float* scale_out, pkmem_stream_t stream) {
  const char* fn = "mem_quantize_rows";
  int rc = check_rows_shape(fn, dt, R, C);
  if (rc) return rc;
  if (R > 0 && (!x || !q_out || !scale_out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(x, 16) || !aligned(q_out, 16) || !aligned(scale_out, 4))
    return fail(PKMEM_ERR_INVALID, "%s: x and q_out must be 16-byte aligned (scale_out 4)", fn);
  if (R == 0) return PKMEM_OK;
  const Bytes bx{x, (size_t)R * C * esize(dt)}, bq{q_out, (size_t)R * C}, bs{scale_out, (size_t)R * 4};
  if (over(bq, {bx, bs}) || over(bs, {bx}))
    return fail(PKMEM_ERR_INVALID, "%s: q_out may not be x, nor any two buffers share bytes", fn);
  return hip_status(pk::launch_quantize_rows(dt == PKMEM_BF16, x, R, C, q_out, scale_out,
                                             reinterpret_cast<hipStream_t>(stream)), fn);
}

int mem_adamw(const pkmem_adamw_tensor* tensors, int count, const pkmem_adamw_opts* opts,
              pkmem_stream_t stream) {
  const char* fn = "mem_adamw";
  int rc = check_adamw_opts(fn, opts);
  if (rc) return rc;
  if (count < 0) return fail(PKMEM_ERR_INVALID, "%s: count must be >= 0", fn);
  if (count > 0 && !tensors) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  for (int i = 0; i < count; ++i) {
    rc = check_adamw_tensor(fn, tensors[i], i, true);
    if (rc) return rc;
    if (tensors[i].numel > pk::ADAMW_MAX_NUMEL)
      return fail(PKMEM_ERR_UNSUPPORTED, "%s: tensor %d: more than 2^36 - 2^12 elements", fn, i);
  }
  rc = check_adamw_overlap(fn, tensors, count, *opts);
  if (rc) return rc;
  return hip_status(pk::launch_adamw(tensors, count, *opts, reinterpret_cast<hipStream_t>(stream)), fn);
}

int mem_adamw_rows(const pkmem_adamw_tensor* table, int64_t N, int D, const int64_t* rows,
                   int64_t U, const pkmem_adamw_opts* opts, pkmem_stream_t stream) {
  const char* fn = "mem_adamw_rows";
  int rc = check_adamw_opts(fn, opts);
  if (rc) return rc;
  if (!table) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  rc = check_adamw_tensor(fn, *table, 0, U > 0);
  if (rc) return rc;
  if (N < 1) return fail(PKMEM_ERR_INVALID, "%s: N must be >= 1", fn);
  if (D < 8 || D % 8 != 0) return fail(PKMEM_ERR_UNSUPPORTED, "%s: D must be a positive multiple of 8 (got %d)", fn, D);
  if (N > (int64_t(1) << 40) / D || table->numel != N * D)
    return fail(PKMEM_ERR_INVALID, "%s: numel must be N * D and at most 2^40", fn);
  if (table->grad_dt != PKMEM_F32) return fail(PKMEM_ERR_UNSUPPORTED, "%s: gradients of rows are fp32", fn);
  const bool s8 = table->state_dt == PKMEM_E4M3;
  if (s8 && D % pk::ADAMW_STATE_BLOCK != 0)
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: 8-bit states need D a multiple of %d (got %d)", fn, pk::ADAMW_STATE_BLOCK, D);
  if (!aligned(table->param, 16) || !aligned(table->grad, 16) || !aligned(table->exp_avg, 16) ||
      !aligned(table->exp_avg_sq, 16))
    return fail(PKMEM_ERR_INVALID, "%s: buffers must be 16-byte aligned", fn);
  if (U < 0) return fail(PKMEM_ERR_INVALID, "%s: U must be >= 0", fn);
  if (U > 0x7FFFFFFF || U * (int64_t)((D + 127) / 128) > 0x7FFFFFFF - 64)
    return fail(PKMEM_ERR_UNSUPPORTED, "%s: too many rows", fn);
  if (U > 0 && !rows) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(rows, 8)) return fail(PKMEM_ERR_INVALID, "%s: rows must be 8-byte aligned", fn);
  if (U == 0) return PKMEM_OK;
  rc = check_adamw_overlap(fn, table, 1, *opts, (size_t)U * D, {rows, (size_t)U * 8});
  if (rc) return rc;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (debug_checks()) {
    uint32_t* flag = nullptr;
    rc = debug_flag(fn, &flag);
    if (rc) return rc;
    rc = debug_outcome(fn, pk::launch_check_rows(rows, U, N, flag, st), flag, N, st);
    if (rc) return rc;
  }
  return hip_status(pk::launch_adamw_rows(*table, N, D, rows, U, *opts, st), fn);
}

}  // extern "C"

// ---- projections -------------------------------------------------------------

namespace {

// A product with rows x cols results, in 256-wide tiles of 512 threads: fewer than 2^32 a launch.
bool tiles_fit(int64_t rows, int cols) { return (rows + 255) / 256 * ((cols + 255) / 256) < (int64_t(1) << 23); }

int check_linear_shapes(const char* fn, pkmem_dtype dt, bool e4m3, int64_t T, int N, int K) {
  if (!dtype_ok(dt) && !(e4m3 && dt == PKMEM_E4M3)) return fail(PKMEM_ERR_INVALID, "%s: unknown dtype %d", fn, (int)dt);
  if (T < 0) return fail(PKMEM_ERR_INVALID, "%s: T must be >= 0", fn);
  if (T > 0x7FFFFFFF) return fail(PKMEM_ERR_UNSUPPORTED, "%s: T must be < 2^31", fn);
  const int ka = dt == PKMEM_E4M3 ? 16 : 8;
  if (N < 8 || N % 8 != 0) return fail(PKMEM_ERR_UNSUPPORTED, "%s: N must be a positive multiple of 8 (got %d)", fn, N);
  if (K < ka || K % ka != 0) return fail(PKMEM_ERR_UNSUPPORTED, "%s: K must be a positive multiple of %d (got %d)", fn, ka, K);
  if (N > (1 << 20) || K > (1 << 20)) return fail(PKMEM_ERR_UNSUPPORTED, "%s: N and K must be <= 2^20", fn);
  return PKMEM_OK;
}

}  // namespace

extern "C" {

int mem_linear(const void* x, const void* w, pkmem_dtype dt, const float* x_scale,
               const float* w_scale, const void* bias, const void* res, int64_t T, int N, int K,
               int act, void* z_out, void* y_out, pkmem_dtype y_dt, pkmem_stream_t stream) {
  const char* fn = "mem_linear";
  int rc = check_linear_shapes(fn, dt, true, T, N, K);
  if (rc) return rc;
  if (!tiles_fit(T, N)) return fail(PKMEM_ERR_UNSUPPORTED, "%s: 2^23 tiles of 256 x 256 or more", fn);
  if (!dtype_ok(y_dt) || (dt == PKMEM_F32 && y_dt != PKMEM_F32))
    return fail(PKMEM_ERR_INVALID, "%s: y_dt must be PKMEM_F32 or PKMEM_BF16 (PKMEM_F32 for fp32 operands)", fn);
  if (act < PKMEM_ACT_NONE || act > PKMEM_ACT_GELU) return fail(PKMEM_ERR_INVALID, "%s: unknown activation %d", fn, act);
  if (dt != PKMEM_E4M3 && (x_scale || w_scale))
    return fail(PKMEM_ERR_INVALID, "%s: scales belong to PKMEM_E4M3 operands", fn);
  if (T > 0 && (!x || !w || !y_out || (dt == PKMEM_E4M3 && (!x_scale || !w_scale))))
    return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 16) ||
      !aligned(bias, 16) || !aligned(res, 16) || !aligned(z_out, 16) || !aligned(y_out, 16))
    return fail(PKMEM_ERR_INVALID, "%s: buffers must be 16-byte aligned", fn);
  if (T == 0) return PKMEM_OK;
  const size_t e = dt == PKMEM_E4M3 ? 1 : esize(dt), ye = esize(y_dt), out = (size_t)T * N * ye;
  const Bytes bx{x, (size_t)T * K * e}, bw{w, (size_t)N * K * e}, bsx{x_scale, (size_t)T * 4}, bsw{w_scale, (size_t)N * 4},
      bb{bias, N * ye}, br{res, out}, bz{z_out, out}, by{y_out, out};
  if (over(by, {bx, bw, bsx, bsw, bb, bz}, {br}) || over(bz, {bx, bw, bsx, bsw, bb, br}))
    return fail(PKMEM_ERR_INVALID, "%s: an output may share no bytes with an operand or the other output (y_out may be res itself)", fn);
  const pk::LinearCall c{x, w, dt, x_scale, w_scale, bias, res, T, N, K, act, z_out, y_out, y_dt == PKMEM_BF16};
  return hip_status(pk::launch_linear(c, reinterpret_cast<hipStream_t>(stream)), fn);
}

int mem_act_backward(const void* dy, const void* z, pkmem_dtype dt, int act, int64_t T, int N,
                     void* dz_out, pkmem_stream_t stream) {
  const char* fn = "mem_act_backward";
  if (!dtype_ok(dt)) return fail(PKMEM_ERR_INVALID, "%s: unknown dtype %d", fn, (int)dt);
  if (act < PKMEM_ACT_NONE || act > PKMEM_ACT_GELU) return fail(PKMEM_ERR_INVALID, "%s: unknown activation %d", fn, act);
  if (T < 0) return fail(PKMEM_ERR_INVALID, "%s: T must be >= 0", fn);
  if (T > 0x7FFFFFFF) return fail(PKMEM_ERR_UNSUPPORTED, "%s: T must be < 2^31", fn);
  if (N < 8 || N % 8 != 0) return fail(PKMEM_ERR_UNSUPPORTED, "%s: N must be a positive multiple of 8 (got %d)", fn, N);
  if (T > 0 && (!dy || !z || !dz_out)) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(dy, 16) || !aligned(z, 16) || !aligned(dz_out, 16))
    return fail(PKMEM_ERR_INVALID, "%s: buffers must be 16-byte aligned", fn);
  if (T == 0) return PKMEM_OK;
  const size_t n = (size_t)T * N * esize(dt);
  if (over({dz_out, n}, {}, {{dy, n}, {z, n}}))
    return fail(PKMEM_ERR_INVALID, "%s: dz_out may be dy or z itself and share no other bytes with them", fn);
  return hip_status(pk::launch_act_backward(dt == PKMEM_BF16, dy, z, act, T * N, dz_out,
                                            reinterpret_cast<hipStream_t>(stream)), fn);
}

size_t mem_linear_backward_workspace_size(int64_t T, int N, int K, pkmem_dtype dt) {
  if (T < 1 || N < 1 || K < 1) return 0;
  return align256(pk::linear_backward_ws_bytes(dt == PKMEM_BF16, T, N, K));
}

int mem_linear_backward(const void* dz, const void* x, const void* w, pkmem_dtype dt, int64_t T,
                        int N, int K, const void* dx_add, void* dx_out, float* grad_w,
                        float* grad_bias, void* ws, size_t ws_bytes, pkmem_stream_t stream) {
  const char* fn = "mem_linear_backward";
  int rc = check_linear_shapes(fn, dt, false, T, N, K);
  if (rc) return rc;
  if (!tiles_fit(T, K) || !tiles_fit(N, K)) return fail(PKMEM_ERR_UNSUPPORTED, "%s: 2^23 tiles of 256 x 256 or more", fn);
  if (T > 0 && (!dz || (dx_out && !w) || (grad_w && !x))) return fail(PKMEM_ERR_INVALID, "%s: null pointer", fn);
  if (!aligned(dz, 16) || !aligned(x, 16) || !aligned(w, 16) || !aligned(dx_add, 16) ||
      !aligned(dx_out, 16) || !aligned(grad_w, 16) || !aligned(grad_bias, 4))
    return fail(PKMEM_ERR_INVALID, "%s: buffers must be 16-byte aligned (grad_bias 4)", fn);
  const size_t need = mem_linear_backward_workspace_size(T, N, K, dt);
  if ((grad_w || grad_bias) && need > 0 && (!ws || ws_bytes < need))
    return fail(PKMEM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
  if (!aligned(ws, 256)) return fail(PKMEM_ERR_INVALID, "%s: workspace must be 256-byte aligned", fn);
  if (T == 0 || (!dx_out && !grad_w && !grad_bias)) return PKMEM_OK;
  const size_t e = esize(dt);
  const Bytes bz{dz, (size_t)T * N * e}, bx{x, (size_t)T * K * e}, bw{w, (size_t)N * K * e}, ba{dx_add, bx.n}, bdx{dx_out, bx.n},
      bgw{grad_w, (size_t)N * K * 4}, bgb{grad_bias, (size_t)N * 4}, bws{grad_w || grad_bias ? ws : nullptr, need};
  if (over(bdx, {bz, bx, bw}, {ba}))
    return fail(PKMEM_ERR_INVALID, "%s: dx_out may be dx_add itself and share no other bytes with an input", fn);
  if (over(bgw, {bz, bx, bw, ba, bdx, bgb}) || over(bgb, {bz, bx, bw, ba, bdx}) || over(bws, {bz, bx, bw, ba, bdx, bgw, bgb}))
    return fail(PKMEM_ERR_INVALID, "%s: grad_w, grad_bias and workspace: each may share bytes with no other buffer", fn);
  return hip_status(pk::launch_linear_backward(dt == PKMEM_BF16, dz, x, w, T, N, K, dx_add, dx_out,
                                               grad_w, grad_bias, ws,
                                               reinterpret_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
