// C ABI of the WaveFilter filter+attend path: argument checks, workspace
// layout and the kernel sequence of every entry point (see wavefilter.h).
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <mutex>

#include "wf_kernels.hpp"
#include "wf_launch.hpp"

namespace wf {

static thread_local char g_last_error[512] = "";

static wf_status fail(wf_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
  va_end(ap);
  return s;
}

static wf_status ok() {
  g_last_error[0] = '\0';
  return WF_OK;
}

float effective_scale(const wf_params& p) {
  return p.scale != 0.f ? p.scale : (float)(1.0 / std::sqrt((double)p.head_dim));
}

int device_cu_count() {
  static thread_local int cached_dev = -1, cached_cus = 0;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (dev != cached_dev) {
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) !=
            hipSuccess ||
        cus <= 0)
      cus = 256;
    cached_dev = dev;
    cached_cus = cus;
  }
  return cached_cus;
}

// ------------------------------------------------------------ validation

#define WF_TRY_SHAPE(expr)           \
  do {                               \
    wf_status _s = (expr);           \
    if (_s != WF_OK) return _s;      \
  } while (0)

// Fields every entry point uses (not segments, budget).
static wf_status check_shape(const wf_params* p) {
  if (!p) return fail(WF_ERR_INVALID_ARG, "params is NULL");
  if (p->batch < 1 || p->heads < 1)
    return fail(WF_ERR_INVALID_ARG, "batch (%d) and heads (%d) must be >= 1",
                p->batch, p->heads);
  if ((long)p->batch * p->heads > (1L << 24))
    return fail(WF_ERR_UNSUPPORTED, "batch*heads = %ld exceeds 2^24",
                (long)p->batch * p->heads);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(WF_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are built",
                p->head_dim);
  if (p->q_len < 1) return fail(WF_ERR_INVALID_ARG, "q_len %d < 1", p->q_len);
  if (p->q_len > WF_MAX_Q_LEN)
    return fail(WF_ERR_UNSUPPORTED, "q_len %d exceeds %d", p->q_len,
                (int)WF_MAX_Q_LEN);
  if (p->gen_len < 0) return fail(WF_ERR_INVALID_ARG, "gen_len %d < 0", p->gen_len);
  if (p->levels < 1) return fail(WF_ERR_INVALID_ARG, "levels %d < 1", p->levels);
  if (p->levels > WF_MAX_LEVELS)
    return fail(WF_ERR_UNSUPPORTED, "levels %d exceeds %d", p->levels,
                (int)WF_MAX_LEVELS);
  if (p->ctx_len < (1 << p->levels))
    return fail(WF_ERR_INVALID_ARG, "ctx_len %d is shorter than 2^levels = %d",
                p->ctx_len, 1 << p->levels);
  if (p->ctx_len > (1 << 30))
    return fail(WF_ERR_UNSUPPORTED, "ctx_len %d exceeds 2^30", p->ctx_len);
  if (p->wavelet != WF_HAAR && p->wavelet != WF_DB2)
    return fail(WF_ERR_INVALID_ARG, "unknown wavelet %d", p->wavelet);
  if (p->boundary != WF_EXT_SYMMETRIC && p->boundary != WF_EXT_PERIODIC)
    return fail(WF_ERR_INVALID_ARG, "unknown boundary %d", p->boundary);
  if (p->dtype != WF_BF16 && p->dtype != WF_F32)
    return fail(WF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (!std::isfinite(p->scale))
    return fail(WF_ERR_INVALID_ARG, "scale is not finite");
  return WF_OK;
}

static wf_status check_params(const wf_params* p) {
  WF_TRY_SHAPE(check_shape(p));
  const int nJ = p->ctx_len >> p->levels;
  if (p->segments < 1 || p->segments > nJ)
    return fail(WF_ERR_INVALID_ARG, "segments %d outside [1, %d]", p->segments, nJ);
  if (p->budget < 1) return fail(WF_ERR_INVALID_ARG, "budget %d < 1", p->budget);
  if (p->dtype == WF_BF16 && plan_scan(*p, false, 0).nbuf < 2)
    return fail(WF_ERR_UNSUPPORTED, "query block and pool range do not fit the LDS ring");
  if ((long)p->batch * p->heads *
          (((long)p->budget < ((long)p->segments << p->levels)
                ? (long)p->budget
                : ((long)p->segments << p->levels)) +
           remainder_len(*p) + (long)p->gen_len) > (1L << 31))
    return fail(WF_ERR_UNSUPPORTED, "sparse cache too large");
  return WF_OK;
}

static wf_status check_ptr(const void* ptr, const char* name, bool nullable) {
  if (!ptr) {
    if (nullable) return WF_OK;
    return fail(WF_ERR_INVALID_ARG, "%s is NULL", name);
  }
  if (((uintptr_t)ptr & 15u) != 0)
    return fail(WF_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return WF_OK;
}

#define WF_TRY(expr)                 \
  do {                               \
    wf_status _s = (expr);           \
    if (_s != WF_OK) return _s;      \
  } while (0)

#define WF_HIP(expr, what)                                                  \
  do {                                                                      \
    hipError_t _e = (expr);                                                 \
    if (_e != hipSuccess)                                                   \
      return fail(WF_ERR_HIP, "%s: %s", what, hipGetErrorString(_e));      \
  } while (0)

// ------------------------------------------------------------ workspace

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct Layout {
  size_t logits = 0, sstats = 0, W = 0, seg = 0, cstats = 0,
         wpool = 0, tok = 0, part = 0, pstat = 0, wsum = 0, wpsum = 0, sseg = 0, total = 0;
};

static long keff_of(const wf_params& p) {
  const long pool = (long)p.segments << p.levels;
  return p.budget < pool ? p.budget : pool;
}

// Regions of the workspace, each 256-byte aligned.  The fused entry point on
// the token-level path keeps a log-sum-exp per (block, query) beside each
// coarse logit instead of the scan's per-workgroup statistics (the scan
// forms the pool normalisers from them on chip), and its attention keeps the
// selected tokens on chip.
static Layout layout_for(const wf_params& p, int op, long attn_rows, int fine) {
  Layout l;
  const size_t U = (size_t)p.batch * p.heads, B = p.q_len;
  const size_t nJ = (size_t)p.ctx_len >> p.levels;
  const size_t P = (size_t)p.segments << p.levels;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up256(bytes);
    return at;
  };
  const bool shared = op == WF_OP_SHARED;
  if (shared) op = WF_OP_FUSED;  // the fused regions, then the sums
  const bool fast = op == WF_OP_FUSED && fast_path(p);
  const bool whole = op == WF_OP_FUSED || op == WF_OP_CACHED;  // a whole step
  const bool skim = op == WF_OP_SKIM || whole;
  const bool scan = op == WF_OP_SCAN || whole;
  const bool attn = op == WF_OP_ATTN || whole;
  if (fast) {
    const FastPlan fp = plan_fast(p);
    l.logits = take(U * nJ * 2 * B * sizeof(float));  // block rows: logits, log-sum-exps
    l.sstats = take(U * fp.R * 2 * B * sizeof(float));
  } else if (skim) {
    const SkimPlan sp = plan_skim(p, op == WF_OP_FUSED, fine);  // from A_J otherwise
    l.logits = take(U * B * nJ * sizeof(float));
    l.sstats = take(U * sp.ntiles * 2 * B * sizeof(float));
  }
  // On the coefficient-tile path, and with fp32 keys, the attention's partials
  // take the place of the coarse logits and their statistics, whose last reader
  // (the W kernel) has ended when the attention starts: the tiles and fp32
  // splits of small calls, finer than a CU needs for large ones, then fit the
  // workspaces that coarser ones did.  (On the token-level path they stay
  // apart: sharing took 84.1 us instead of 82.3 for 64 units of 8K keys.)
  const bool overlay = whole && (p.dtype != WF_BF16 || (op == WF_OP_FUSED && !fast));
  size_t part_bytes = 0, pstat_bytes = 0;
  if (attn) {
    const AttnPlan ap = plan_attn(p, attn_rows, fine);
    part_bytes = up256(U * ap.splits * B * p.head_dim * sizeof(float));
    pstat_bytes = up256(U * ap.splits * 2 * B * sizeof(float));
  }
  if (overlay) {
    l.part = l.logits;  // the first region
    l.pstat = l.part + part_bytes;
    off = std::max(off, l.pstat + pstat_bytes);
  }
  if (whole) {
    l.W = take(U * nJ * sizeof(float));
    l.seg = take(U * p.segments * sizeof(int32_t));
  }
  if (scan) {
    // the token-level path forms the pool normalisers inside the scan
    const ScanPlan cp = plan_scan(p, false, fine);
    if (!fast) l.cstats = take(U * cp.chunks * 2 * B * sizeof(float));
    l.wpool = take(U * P * sizeof(float));
  }
  // a selecting attention keeps its selected tokens on chip
  const bool attn_selects = fast || (op == WF_OP_CACHED && attn_can_select(p, attn_rows));
  if (whole && !attn_selects) l.tok = take(U * keff_of(p) * sizeof(int32_t));
  if (attn && !overlay) {
    l.part = take(part_bytes);
    l.pstat = take(pstat_bytes);
  }
  if (shared) {
    // W and W' of each sequence, summed over its heads; its shared regions
    const size_t nb = (size_t)p.batch;
    l.wsum = take(nb * nJ * sizeof(float));
    l.wpsum = take(nb * P * sizeof(float));
    l.sseg = take(nb * p.segments * sizeof(int32_t));
  }
  l.total = off;
  return l;
}

// Whether the finer Haar tiles' statistics fit where the attention's coarsest
// partials share their place, so that the workspace is no larger than with coarse
// tiles and both apart.
static int fine_tiles(const wf_params& p, int op, long attn_rows) {
  if (p.wavelet != WF_HAAR || (op != WF_OP_FUSED && op != WF_OP_SHARED) || fast_path(p)) return 0;
  const long more = plan_skim(p, true, kFineTiles).ntiles - plan_skim(p, true, 0).ntiles;
  return more == 0 || 2 * more <= plan_attn(p, attn_rows, 0).splits * (p.head_dim + 2L) ? kFineTiles
                                                                                        : 0;
}

// fp32 calls take the fine splits where these fit the bytes that they have (and,
// in all, a small workspace), else the coarse ones, which fit the bytes that were
// enough before the splits became finer.
constexpr size_t kFineBytes = (size_t)32 << 20;
template <class Of>
static auto layout_in(const wf_params& p, size_t have, int tiles, int* fine, const Of& of) {
  *fine = tiles | kFineSplits;
  const auto f = of(*fine);
  if (p.dtype == WF_BF16 || (f.total <= have && f.total <= kFineBytes)) return f;
  const auto c = of(tiles);
  if (f.total <= c.total) return f;
  *fine = tiles;
  return c;
}
static Layout layout_in(const wf_params& p, int op, long attn_rows, size_t have, int* fine) {
  return layout_in(p, have, fine_tiles(p, op, attn_rows), fine,
                   [&](int f) { return layout_for(p, op, attn_rows, f); });
}

static wf_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return WF_OK;
  if (!ws) return fail(WF_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
  if (((uintptr_t)ws & 255u) != 0)
    return fail(WF_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (have < need)
    return fail(WF_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
  return WF_OK;
}

static inline char* at(void* ws, size_t off) { return static_cast<char*>(ws) + off; }

// ------------------------------------------------------------ fused sequence

// Kernel sequences of the fused entry point.  The general path scores the
// coarse coefficients and runs both passes of the token scan; the token-level
// path (bf16, Haar, 3..5 levels, <= 64 query rows) derives the scan's
// normalisers from the skim's block statistics.
static const char* const kGeneralNames[] = {
    "skim_tile", "skim_select", "scan_stats", "scan_weights",
    "scan_select", "sparse_attn", "attn_combine"};
// W over all CUs, the top-S in the statistics pass, and when the attention's
// rows allow it the top-k in the attention (scan_selects).  One workgroup per
// unit for W and the top-S took 30.6 us of 107.9 with 16 units of 128 query
// rows and 1024 coefficients; W over all CUs takes 8.1.
static const char* const kGeneralWideNames[] = {
    "skim_tile", "skim_weights", "scan_stats", "scan_weights",
    "scan_select", "sparse_attn", "attn_combine"};
static const char* const kGeneralWideSelectNames[] = {
    "skim_tile", "skim_weights", "scan_stats", "scan_weights", "sparse_attn", "attn_combine"};
static const char* const kFastNames[] = {
    "token_skim", "block_weights", "scan_weights", "sparse_attn", "attn_combine"};
constexpr int kMaxFusedKernels = 7;

// Where W is formed over all CUs and the statistics pass takes the top-S
static bool scan_selects(const wf_params& p) {
  return scan_can_select(p) &&
         (wide_weights(p) || (p.dtype == WF_BF16 && p.q_len <= 64 &&
                              (((long)p.ctx_len >> p.levels) & 3) == 0));
}

static long fused_rows(const wf_params& p) {
  return keff_of(p) + remainder_len(p) + p.gen_len;
}
// the general sequence with its selections in their consumers
static bool general_wide(const wf_params& p) {
  return !fast_path(p) && scan_selects(p);
}
static bool general_attn_selects(const wf_params& p) {
  const bool small = p.dtype == WF_BF16 && p.q_len <= 64 && ((p.ctx_len >> p.levels) & 3) == 0;
  return general_wide(p) && attn_can_select(p, fused_rows(p)) && (small || pool_on_chip(p));
}
static int fused_kernels(const wf_params& p) {
  return fast_path(p) ? 5 : general_attn_selects(p) ? 6 : 7;
}
static const char* const* fused_names(const wf_params& p) {
  if (fast_path(p)) return kFastNames;
  if (general_wide(p)) return general_attn_selects(p) ? kGeneralWideSelectNames : kGeneralWideNames;
  return kGeneralNames;
}

static wf_status fused_impl(const wf_params* p, const void* Q, const void* K,
                            const void* V, const void* Kg, const void* Vg,
                            void* O, int32_t* tok_idx, int32_t* seg_idx,
                            void* ws, size_t ws_bytes, void* stream,
                            void** events, int n_events) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_ptr(O, "O", false));
  WF_TRY(check_ptr(tok_idx, "tok_idx", true));
  WF_TRY(check_ptr(seg_idx, "seg_idx", true));
  if (p->gen_len > 0) {
    WF_TRY(check_ptr(Kg, "Kg", false));
    WF_TRY(check_ptr(Vg, "Vg", false));
  }
  const int nk = fused_kernels(*p);
  const char* const* names = fused_names(*p);
  if (events && n_events < nk + 1)
    return fail(WF_ERR_INVALID_ARG, "n_events %d < %d", n_events, nk + 1);
  const long keff = keff_of(*p);
  const long nrows = keff + remainder_len(*p) + p->gen_len;
  int fine;
  const Layout l = layout_in(*p, WF_OP_FUSED, nrows, ws_bytes, &fine);
  WF_TRY(check_workspace(ws, ws_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  float* logits = reinterpret_cast<float*>(at(ws, l.logits));
  float* sstats = reinterpret_cast<float*>(at(ws, l.sstats));
  float* W = reinterpret_cast<float*>(at(ws, l.W));
  int32_t* seg = seg_idx ? seg_idx : reinterpret_cast<int32_t*>(at(ws, l.seg));
  float* cstats = reinterpret_cast<float*>(at(ws, l.cstats));
  float* wpool = reinterpret_cast<float*>(at(ws, l.wpool));
  int32_t* tok = tok_idx ? tok_idx : reinterpret_cast<int32_t*>(at(ws, l.tok));
  float* part = reinterpret_cast<float*>(at(ws, l.part));
  float* pstat = reinterpret_cast<float*>(at(ws, l.pstat));
  int k = 0;
  auto mark = [&]() -> hipError_t {
    if (!events) return hipSuccess;
    return hipEventRecord(static_cast<hipEvent_t>(events[k]), s);
  };
  // launch one kernel of the sequence, bracketed by events when timed
  auto step = [&](hipError_t launched) -> wf_status {
    if (launched != hipSuccess)
      return fail(WF_ERR_HIP, "%s: %s", names[k], hipGetErrorString(launched));
    ++k;
    hipError_t e = mark();
    if (e != hipSuccess) return fail(WF_ERR_HIP, "hipEventRecord: %s", hipGetErrorString(e));
    return WF_OK;
  };
  WF_HIP(mark(), "hipEventRecord");
  if (fast_path(*p)) {
    // token logits -> block rows; W of every block; the scan takes the top-S
    // regions and the attention the top-k tokens themselves
    WF_TRY(step(launch_token_skim(*p, Q, K, logits, sstats, s)));
    WF_TRY(step(launch_block_weights(*p, logits, sstats, W, s)));
    WF_TRY(step(launch_scan_select_weights(*p, Q, K, W, logits, seg, wpool, s)));
    WF_TRY(step(launch_attn_select(*p, Q, K, V, wpool, seg, tok_idx, Kg, Vg, nrows, part,
                                   pstat, fine, s)));
  } else {
    const SkimPlan sp = plan_skim(*p, true, fine);
    WF_TRY(step(launch_skim_tiles(*p, true, Q, K, nullptr, logits, sstats, fine, s)));
    if (general_wide(*p)) {
      WF_TRY(step(launch_skim_weights(*p, sp.ntiles, logits, sstats, W, s)));
      WF_TRY(step(launch_scan_select_stats(*p, Q, K, W, seg, cstats, fine, s)));
    } else {
      WF_TRY(step(launch_skim_select(*p, sp.ntiles, logits, sstats, W, seg, s)));
      WF_TRY(step(launch_scan_chunks(*p, 0, Q, K, seg, cstats, wpool, fine, s)));
    }
    WF_TRY(step(launch_scan_chunks(*p, 1, Q, K, seg, cstats, wpool, fine, s)));
    if (general_attn_selects(*p)) {
      WF_TRY(step(launch_attn_select(*p, Q, K, V, wpool, seg, tok_idx, Kg, Vg, nrows, part,
                                     pstat, fine, s)));
    } else {
      WF_TRY(step(launch_scan_select(*p, wpool, seg, tok, s)));
      WF_TRY(step(launch_attn(*p, Q, K, V, tok, (int)keff, Kg, Vg, p->gen_len, nrows,
                              part, pstat, fine, s)));
    }
  }
  WF_TRY(step(launch_attn_combine(*p, nrows, part, pstat, O, fine, s)));
  return ok();
}

// ------------------------------------------------------------ no allocation
//
// wf_filter_attend_noalloc runs the fused sequence on a workspace that the
// library owns: a file-scope device array, one copy per device, present from
// the load of the code object until the process ends.  Host code never
// passes `scratch` itself (in host code the name is a host-side stand-in, not
// a device address); it passes the address hipGetSymbolAddress reports for
// the current device, looked up once per device.
constexpr size_t kScratchBytes = (size_t)WF_NOALLOC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char scratch[kScratchBytes];

constexpr int kMaxDevices = 64;
static std::mutex g_scratch_mu;
static void* g_scratch_ptr[kMaxDevices] = {};

static wf_status scratch_of_current_device(void** out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail(WF_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
  if (dev < 0 || dev >= kMaxDevices)
    return fail(WF_ERR_UNSUPPORTED, "device %d: at most %d devices", dev, kMaxDevices);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* ptr = nullptr;
    e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !ptr)
      return fail(WF_ERR_HIP, "hipGetSymbolAddress(scratch): %s", hipGetErrorString(e));
    g_scratch_ptr[dev] = ptr;
  }
  *out = g_scratch_ptr[dev];
  return WF_OK;
}

static wf_status noalloc_impl(const wf_params* p, const void* Q, const void* K,
                              const void* V, const void* Kg, const void* Vg, void* O,
                              int32_t* tok_idx, int32_t* seg_idx, void* stream) {
  WF_TRY(check_params(p));
  const long nrows = keff_of(*p) + remainder_len(*p) + p->gen_len;
  int fine;
  const size_t need = layout_in(*p, WF_OP_FUSED, nrows, kScratchBytes, &fine).total;
  if (need > kScratchBytes)
    return fail(WF_ERR_WORKSPACE,
                "these parameters need %zu bytes of scratch; the allocation-free entry "
                "point holds %zu (use wf_filter_attend with a workspace)",
                need, kScratchBytes);
  void* ws = nullptr;
  WF_TRY(scratch_of_current_device(&ws));
  return fused_impl(p, Q, K, V, Kg, Vg, O, tok_idx, seg_idx, ws, kScratchBytes, stream,
                    nullptr, 0);
}

// ------------------------------------------------------------ cached A_J

static const char* const kCachedNames[] = {
    "skim_tile", "skim_select", "scan_stats", "scan_weights",
    "scan_select", "sparse_attn", "attn_combine"};
constexpr int kCachedKernels = 7;
// with bf16 keys the attention takes the top-k of W' itself
static const char* const kCachedSelectNames[] = {
    "skim_tile", "skim_select", "scan_stats", "scan_weights", "sparse_attn", "attn_combine"};
// W is formed over all CUs and the statistics pass takes the top-S of W
// itself (scan_selects)
static const char* const kCachedWideNames[] = {
    "skim_tile", "skim_weights", "scan_stats", "scan_weights",
    "scan_select", "sparse_attn", "attn_combine"};
static const char* const kCachedWideSelectNames[] = {
    "skim_tile", "skim_weights", "scan_stats", "scan_weights", "sparse_attn", "attn_combine"};

static long cached_rows(const wf_params& p) {
  return keff_of(p) + remainder_len(p) + p.gen_len;
}
static bool cached_attn_selects(const wf_params& p) {
  return attn_can_select(p, cached_rows(p));
}
static bool cached_scan_selects(const wf_params& p) {
  return scan_selects(p);
}
static int cached_kernels(const wf_params& p) {
  return cached_attn_selects(p) ? kCachedKernels - 1 : kCachedKernels;
}
static const char* const* cached_names(const wf_params& p) {
  if (cached_scan_selects(p))
    return cached_attn_selects(p) ? kCachedWideSelectNames : kCachedWideNames;
  return cached_attn_selects(p) ? kCachedSelectNames : kCachedNames;
}

static wf_status cached_impl(const wf_params* p, const void* Q, const float* approx,
                             const void* K, const void* V, const void* Kg, const void* Vg,
                             void* O, int32_t* tok_idx, int32_t* seg_idx, void* ws,
                             size_t ws_bytes, void* stream, void** events, int n_events) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(approx, "approx", false));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_ptr(O, "O", false));
  WF_TRY(check_ptr(tok_idx, "tok_idx", true));
  WF_TRY(check_ptr(seg_idx, "seg_idx", true));
  if (p->gen_len > 0) {
    WF_TRY(check_ptr(Kg, "Kg", false));
    WF_TRY(check_ptr(Vg, "Vg", false));
  }
  const int nk = cached_kernels(*p);
  const char* const* names = cached_names(*p);
  if (events && n_events < nk + 1)
    return fail(WF_ERR_INVALID_ARG, "n_events %d < %d", n_events, nk + 1);
  const long keff = keff_of(*p);
  const long nrows = cached_rows(*p);
  int fine;
  const Layout l = layout_in(*p, WF_OP_CACHED, nrows, ws_bytes, &fine);
  WF_TRY(check_workspace(ws, ws_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  float* logits = reinterpret_cast<float*>(at(ws, l.logits));
  float* sstats = reinterpret_cast<float*>(at(ws, l.sstats));
  float* W = reinterpret_cast<float*>(at(ws, l.W));
  int32_t* seg = seg_idx ? seg_idx : reinterpret_cast<int32_t*>(at(ws, l.seg));
  float* cstats = reinterpret_cast<float*>(at(ws, l.cstats));
  float* wpool = reinterpret_cast<float*>(at(ws, l.wpool));
  int32_t* tok = tok_idx ? tok_idx : reinterpret_cast<int32_t*>(at(ws, l.tok));
  float* part = reinterpret_cast<float*>(at(ws, l.part));
  float* pstat = reinterpret_cast<float*>(at(ws, l.pstat));
  int k = 0;
  auto mark = [&]() -> hipError_t {
    if (!events) return hipSuccess;
    return hipEventRecord(static_cast<hipEvent_t>(events[k]), s);
  };
  auto step = [&](hipError_t launched) -> wf_status {
    if (launched != hipSuccess)
      return fail(WF_ERR_HIP, "%s: %s", names[k], hipGetErrorString(launched));
    ++k;
    hipError_t e = mark();
    if (e != hipSuccess) return fail(WF_ERR_HIP, "hipEventRecord: %s", hipGetErrorString(e));
    return WF_OK;
  };
  WF_HIP(mark(), "hipEventRecord");
  const SkimPlan sp = plan_skim(*p, false, fine);
  WF_TRY(step(launch_skim_tiles(*p, false, Q, nullptr, approx, logits, sstats, fine, s)));
  if (cached_scan_selects(*p)) {
    WF_TRY(step(launch_skim_weights(*p, sp.ntiles, logits, sstats, W, s)));
    WF_TRY(step(launch_scan_select_stats(*p, Q, K, W, seg, cstats, fine, s)));
  } else {
    WF_TRY(step(launch_skim_select(*p, sp.ntiles, logits, sstats, W, seg, s)));
    WF_TRY(step(launch_scan_chunks(*p, 0, Q, K, seg, cstats, wpool, fine, s)));
  }
  WF_TRY(step(launch_scan_chunks(*p, 1, Q, K, seg, cstats, wpool, fine, s)));
  if (cached_attn_selects(*p)) {
    WF_TRY(step(launch_attn_select(*p, Q, K, V, wpool, seg, tok_idx, Kg, Vg, nrows, part,
                                   pstat, fine, s)));
  } else {
    WF_TRY(step(launch_scan_select(*p, wpool, seg, tok, s)));
    WF_TRY(step(launch_attn(*p, Q, K, V, tok, (int)keff, Kg, Vg, p->gen_len, nrows, part,
                            pstat, fine, s)));
  }
  WF_TRY(step(launch_attn_combine(*p, nrows, part, pstat, O, fine, s)));
  return ok();
}

// ------------------------------------------------------------ shared selection

// One selection per sequence, shared by its heads: the token-level sequence
// with W and W' added over the heads before each top-k.
static const char* const kSharedNames[] = {
    "token_skim", "block_weights", "head_sum_w", "scan_weights",
    "head_sum_wpool", "sparse_attn", "attn_combine"};
// the general path: W per unit from the skim select (whose own regions are
// not used), the heads' sum, one select per sequence; the scan's two passes
// per unit over the sequence's regions, the heads' sum of W', one token
// select per sequence; attention per unit
static const char* const kSharedGeneralNames[] = {
    "skim_tile", "skim_select", "head_sum_w", "select_regions", "scan_stats",
    "scan_weights", "head_sum_wpool", "scan_select", "sparse_attn", "attn_combine"};
// each head's W alone, over all CUs
static const char* const kSharedGeneralWideNames[] = {
    "skim_tile", "skim_weights", "head_sum_w", "select_regions", "scan_stats",
    "scan_weights", "head_sum_wpool", "scan_select", "sparse_attn", "attn_combine"};
constexpr int kSharedMaxKernels = 10;
static bool shared_w_only(const wf_params& p) {
  return wide_weights(p) || (((long)p.ctx_len >> p.levels) & 3) == 0;
}
static int shared_kernels(const wf_params& p) { return fast_path(p) ? 7 : 10; }
static const char* const* shared_names(const wf_params& p) {
  if (fast_path(p)) return kSharedNames;
  return shared_w_only(p) ? kSharedGeneralWideNames : kSharedGeneralNames;
}

static wf_status shared_impl(const wf_params* p, const void* Q, const void* K,
                             const void* V, const void* Kg, const void* Vg, void* O,
                             int32_t* tok_idx, int32_t* seg_idx, void* ws, size_t ws_bytes,
                             void* stream, void** events, int n_events) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_ptr(O, "O", false));
  WF_TRY(check_ptr(tok_idx, "tok_idx", true));
  WF_TRY(check_ptr(seg_idx, "seg_idx", true));
  if (p->gen_len > 0) {
    WF_TRY(check_ptr(Kg, "Kg", false));
    WF_TRY(check_ptr(Vg, "Vg", false));
  }
  const int nk = shared_kernels(*p);
  const char* const* names = shared_names(*p);
  if (events && n_events < nk + 1)
    return fail(WF_ERR_INVALID_ARG, "n_events %d < %d", n_events, nk + 1);
  const long keff = keff_of(*p);
  const long nrows = keff + remainder_len(*p) + p->gen_len;
  int fine;
  const Layout l = layout_in(*p, WF_OP_SHARED, nrows, ws_bytes, &fine);
  WF_TRY(check_workspace(ws, ws_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  float* logits = reinterpret_cast<float*>(at(ws, l.logits));
  float* sstats = reinterpret_cast<float*>(at(ws, l.sstats));
  float* W = reinterpret_cast<float*>(at(ws, l.W));
  float* cstats = reinterpret_cast<float*>(at(ws, l.cstats));
  float* wpool = reinterpret_cast<float*>(at(ws, l.wpool));
  float* part = reinterpret_cast<float*>(at(ws, l.part));
  float* pstat = reinterpret_cast<float*>(at(ws, l.pstat));
  float* wsum = reinterpret_cast<float*>(at(ws, l.wsum));
  float* wpsum = reinterpret_cast<float*>(at(ws, l.wpsum));
  int32_t* seg = seg_idx ? seg_idx : reinterpret_cast<int32_t*>(at(ws, l.sseg));
  const int H = p->heads;
  const long nJ = (long)p->ctx_len >> p->levels;
  const long P = (long)p->segments << p->levels;
  int k = 0;
  auto mark = [&]() -> hipError_t {
    if (!events) return hipSuccess;
    return hipEventRecord(static_cast<hipEvent_t>(events[k]), s);
  };
  auto step = [&](hipError_t launched) -> wf_status {
    if (launched != hipSuccess)
      return fail(WF_ERR_HIP, "%s: %s", names[k], hipGetErrorString(launched));
    ++k;
    hipError_t e = mark();
    if (e != hipSuccess) return fail(WF_ERR_HIP, "hipEventRecord: %s", hipGetErrorString(e));
    return WF_OK;
  };
  WF_HIP(mark(), "hipEventRecord");
  if (fast_path(*p)) {
    WF_TRY(step(launch_token_skim(*p, Q, K, logits, sstats, s)));
    WF_TRY(step(launch_block_weights(*p, logits, sstats, W, s)));
    WF_TRY(step(launch_head_sum(W, wsum, nJ, H, p->batch, s)));
    WF_TRY(step(launch_scan_select_weights(*p, Q, K, wsum, logits, seg, wpool, s, H)));
    WF_TRY(step(launch_head_sum(wpool, wpsum, P, H, p->batch, s)));
    WF_TRY(step(launch_attn_select(*p, Q, K, V, wpsum, seg, tok_idx, Kg, Vg, nrows, part,
                                   pstat, fine, s, H)));
  } else {
    // one "unit" per sequence for the two selections over the heads' sums
    wf_params pg = *p;
    pg.heads = 1;
    int32_t* tok = tok_idx ? tok_idx : reinterpret_cast<int32_t*>(at(ws, l.tok));
    int32_t* unit_seg = reinterpret_cast<int32_t*>(at(ws, l.seg));  // not used after
    const SkimPlan sp = plan_skim(*p, true, fine);
    WF_TRY(step(launch_skim_tiles(*p, true, Q, K, nullptr, logits, sstats, fine, s)));
    if (shared_w_only(*p))
      WF_TRY(step(launch_skim_weights(*p, sp.ntiles, logits, sstats, W, s)));
    else  // the per-unit select's regions are not used
      WF_TRY(step(launch_skim_select(*p, sp.ntiles, logits, sstats, W, unit_seg, s)));
    WF_TRY(step(launch_head_sum(W, wsum, nJ, H, p->batch, s)));
    WF_TRY(step(launch_select_w(pg, p->batch, wsum, seg, s)));
    WF_TRY(step(launch_scan_chunks(*p, 0, Q, K, seg, cstats, wpool, fine, s, H)));
    WF_TRY(step(launch_scan_chunks(*p, 1, Q, K, seg, cstats, wpool, fine, s, H)));
    WF_TRY(step(launch_head_sum(wpool, wpsum, P, H, p->batch, s)));
    WF_TRY(step(launch_scan_select(pg, wpsum, seg, tok, s)));
    WF_TRY(step(launch_attn(*p, Q, K, V, tok, (int)keff, Kg, Vg, p->gen_len, nrows, part,
                            pstat, fine, s, H)));
  }
  WF_TRY(step(launch_attn_combine(*p, nrows, part, pstat, O, fine, s)));
  return ok();
}

// ------------------------------------------------------------ recursion

// Validates the recursion's parameters and fills counts[b - 1] = c_b.
static wf_status check_recursion(const wf_params* p, const float* prop, int32_t* counts) {
  WF_TRY(check_shape(p));
  if (!prop) return fail(WF_ERR_INVALID_ARG, "proportions is NULL");
  long n = (long)p->ctx_len >> p->levels;
  for (int b = p->levels; b >= 1; --b) {
    const float m = prop[b - 1];
    if (!(m > 0.f && m <= 1.f))
      return fail(WF_ERR_INVALID_ARG, "proportion m_%d = %g outside (0, 1]", b, (double)m);
    long c = (long)std::ceil((double)m * (double)n);
    c = std::max(1L, std::min(c, n));
    counts[b - 1] = (int32_t)c;
    n = 2 * c;
  }
  if ((long)p->batch * p->heads * (2L * counts[0] + remainder_len(*p) + p->gen_len) >
      (1L << 31))
    return fail(WF_ERR_UNSUPPORTED, "sparse cache too large");
  return WF_OK;
}

struct RecLayout {
  size_t logits = 0, stats = 0, W = 0, sel[2] = {0, 0}, tok = 0, part = 0, pstat = 0,
         total = 0;
};

static RecLayout rec_layout(const wf_params& p, const int32_t* counts, int fine) {
  RecLayout l;
  const RecPlan rp = plan_recursion(p, counts);
  const size_t U = (size_t)p.batch * p.heads, B = p.q_len;
  const long nrows = 2L * counts[0] + remainder_len(p) + p.gen_len;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += up256(bytes);
    return at;
  };
  l.logits = take(U * B * rp.max_n * sizeof(float));
  l.stats = take(U * rp.max_tiles * 2 * B * sizeof(float));
  const AttnPlan ap = plan_attn(p, nrows, fine);
  const size_t part_bytes = up256(U * ap.splits * B * p.head_dim * sizeof(float));
  const size_t pstat_bytes = up256(U * ap.splits * 2 * B * sizeof(float));
  // fp32: the partials in the place of the last scale's logits and statistics
  const bool overlay = p.dtype != WF_BF16;
  if (overlay) {
    l.part = l.logits;
    l.pstat = l.part + part_bytes;
    off = std::max(off, l.pstat + pstat_bytes);
  }
  l.W = take(U * rp.max_n * sizeof(float));
  l.sel[0] = take(U * rp.max_keep * sizeof(int32_t));
  l.sel[1] = take(U * rp.max_keep * sizeof(int32_t));
  l.tok = take(U * 2 * counts[0] * sizeof(int32_t));
  if (!overlay) {
    l.part = take(part_bytes);
    l.pstat = take(pstat_bytes);
  }
  l.total = off;
  return l;
}

static RecLayout rec_layout_in(const wf_params& p, const int32_t* counts, size_t have, int* fine) {
  return layout_in(p, have, 0, fine, [&](int f) { return rec_layout(p, counts, f); });
}

static const char* const kRecTileNames[WF_MAX_LEVELS] = {
    "rec_tiles_b1", "rec_tiles_b2", "rec_tiles_b3", "rec_tiles_b4", "rec_tiles_b5",
    "rec_tiles_b6", "rec_tiles_b7", "rec_tiles_b8", "rec_tiles_b9", "rec_tiles_b10"};
static const char* const kRecSelectNames[WF_MAX_LEVELS] = {
    "rec_select_b1", "rec_select_b2", "rec_select_b3", "rec_select_b4", "rec_select_b5",
    "rec_select_b6", "rec_select_b7", "rec_select_b8", "rec_select_b9", "rec_select_b10"};

static int rec_kernels(const wf_params& p) { return 2 * p.levels + 2; }

static const char* rec_kernel_name(const wf_params& p, int i) {
  if (i < 2 * p.levels) {
    const int b = p.levels - i / 2;
    return (i % 2 == 0 ? kRecTileNames : kRecSelectNames)[b - 1];
  }
  return i == 2 * p.levels ? "sparse_attn" : "attn_combine";
}

static wf_status recursive_impl(const wf_params* p, const float* prop, const void* Q,
                                const void* K, const void* V, const void* Kg,
                                const void* Vg, void* O, int32_t* tok_idx,
                                int32_t* kept_idx, void* ws, size_t ws_bytes,
                                void* stream, void** events, int n_events) {
  int32_t counts[WF_MAX_LEVELS];
  WF_TRY(check_recursion(p, prop, counts));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_ptr(O, "O", false));
  WF_TRY(check_ptr(tok_idx, "tok_idx", true));
  if (kept_idx && ((uintptr_t)kept_idx & 3u) != 0)
    return fail(WF_ERR_INVALID_ARG, "kept_idx is not 4-byte aligned");
  if (p->gen_len > 0) {
    WF_TRY(check_ptr(Kg, "Kg", false));
    WF_TRY(check_ptr(Vg, "Vg", false));
  }
  const int nk = rec_kernels(*p);
  if (events && n_events < nk + 1)
    return fail(WF_ERR_INVALID_ARG, "n_events %d < %d", n_events, nk + 1);
  int fine;
  const RecLayout l = rec_layout_in(*p, counts, ws_bytes, &fine);
  WF_TRY(check_workspace(ws, ws_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  float* logits = reinterpret_cast<float*>(at(ws, l.logits));
  float* stats = reinterpret_cast<float*>(at(ws, l.stats));
  float* W = reinterpret_cast<float*>(at(ws, l.W));
  int32_t* sel[2] = {reinterpret_cast<int32_t*>(at(ws, l.sel[0])),
                     reinterpret_cast<int32_t*>(at(ws, l.sel[1]))};
  int32_t* tok = tok_idx ? tok_idx : reinterpret_cast<int32_t*>(at(ws, l.tok));
  float* part = reinterpret_cast<float*>(at(ws, l.part));
  float* pstat = reinterpret_cast<float*>(at(ws, l.pstat));
  int k = 0;
  auto mark = [&]() -> hipError_t {
    if (!events) return hipSuccess;
    return hipEventRecord(static_cast<hipEvent_t>(events[k]), s);
  };
  auto step = [&](hipError_t launched) -> wf_status {
    if (launched != hipSuccess)
      return fail(WF_ERR_HIP, "%s: %s", rec_kernel_name(*p, k), hipGetErrorString(launched));
    ++k;
    hipError_t e = mark();
    if (e != hipSuccess) return fail(WF_ERR_HIP, "hipEventRecord: %s", hipGetErrorString(e));
    return WF_OK;
  };
  WF_HIP(mark(), "hipEventRecord");
  long n = (long)p->ctx_len >> p->levels;
  const int32_t* parent = nullptr;
  int npar = 0;
  const long U = (long)p->batch * p->heads;
  long kept_at = 0;  // element offset of this scale's ids in kept_idx
  for (int b = p->levels; b >= 1; --b) {
    int32_t* out = b == 1 ? tok : kept_idx ? kept_idx + kept_at : sel[b & 1];
    kept_at += U * counts[b - 1];
    if (rec_token_path(*p) && b <= 5) {
      // the scale's coarse logits as sums of token logits (of the kept
      // blocks' tokens below the first scale)
      const long rows = parent ? (long)npar << (b + 1) : filtered_len(*p);
      WF_TRY(step(launch_rec_token_skim(*p, b, n, parent, npar, Q, K, logits, stats, s)));
      WF_TRY(step(launch_rec_select_slices(*p, b, n, counts[b - 1], parent, npar,
                                           plan_rec_token(*p, b, rows, parent != nullptr).R,
                                           logits, stats, W, out, s)));
    } else {
      WF_TRY(step(launch_rec_tiles(*p, b, n, parent, npar, Q, K, logits, stats, s)));
      WF_TRY(step(launch_rec_select(*p, b, n, counts[b - 1], parent, npar, logits, stats, W,
                                    out, s)));
    }
    parent = out;
    npar = counts[b - 1];
    n = 2L * counts[b - 1];
  }
  const int nsel = 2 * counts[0];
  const long nrows = (long)nsel + remainder_len(*p) + p->gen_len;
  WF_TRY(step(launch_attn(*p, Q, K, V, tok, nsel, Kg, Vg, p->gen_len, nrows, part, pstat,
                          fine, s)));
  WF_TRY(step(launch_attn_combine(*p, nrows, part, pstat, O, fine, s)));
  return ok();
}

// ------------------------------------------------------------ quantised cache

static wf_status check_cache(const wf_cache_params* p) {
  if (!p) return fail(WF_ERR_INVALID_ARG, "params is NULL");
  if (p->batch < 1 || p->heads < 1)
    return fail(WF_ERR_INVALID_ARG, "batch (%d) and heads (%d) must be >= 1", p->batch, p->heads);
  if (p->capacity < 1) return fail(WF_ERR_INVALID_ARG, "capacity %d < 1", p->capacity);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(WF_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are built", p->head_dim);
  if (p->rows < 0) return fail(WF_ERR_INVALID_ARG, "rows %d < 0", p->rows);
  if (p->dtype != WF_BF16 && p->dtype != WF_F32)
    return fail(WF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (p->format != WF_CACHE_E4M3 && p->format != WF_CACHE_E2M1)
    return fail(WF_ERR_INVALID_ARG, "unknown cache format %d", p->format);
  if ((long)p->batch * p->heads > (1L << 24))
    return fail(WF_ERR_UNSUPPORTED, "batch*heads = %ld exceeds 2^24", (long)p->batch * p->heads);
  if (cache_groups(*p) * kBlock > UINT32_MAX)  // a launch has fewer than 2^32 threads
    return fail(WF_ERR_UNSUPPORTED, "%ld rows in one call are too many",
                (long)p->batch * p->heads * p->rows);
  return WF_OK;
}

static wf_status cache_impl(const wf_cache_params* p, bool store, const void* K, const void* V,
                            const int32_t* row_idx, const void* Kc, const void* Kx,
                            const void* Vc, const void* Vx, void* stream) {
  WF_TRY(check_cache(p));
  if (p->rows == 0) return ok();
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_ptr(row_idx, "row_idx", true));
  WF_TRY(check_ptr(Kc, "Kc", false));
  WF_TRY(check_ptr(Kx, "Kx", false));
  WF_TRY(check_ptr(Vc, "Vc", false));
  WF_TRY(check_ptr(Vx, "Vx", false));
  if (!row_idx && (p->first < 0 || (long)p->first + p->rows > p->capacity))
    return fail(WF_ERR_INVALID_ARG, "rows %d .. %ld are outside the capacity %d", p->first,
                (long)p->first + p->rows, p->capacity);
  (void)hipGetLastError();
  WF_HIP(launch_cache(*p, store, K, V, row_idx, Kc, Kx, Vc, Vx, static_cast<hipStream_t>(stream)),
         store ? "cache_store" : "cache_load");
  return ok();
}

// ------------------------------------------------------------ a cache in pages

// Arrays of 32-bit words, which the kernels read one at a time.
static wf_status check_words(const void* ptr, const char* name, bool nullable) {
  if (!ptr) return nullable ? WF_OK : fail(WF_ERR_INVALID_ARG, "%s is NULL", name);
  if (((uintptr_t)ptr & 3u) != 0)
    return fail(WF_ERR_INVALID_ARG, "%s is not 4-byte aligned", name);
  return WF_OK;
}

static wf_status check_rows(int dtype, int head_dim) {
  if (head_dim != 64 && head_dim != 128)
    return fail(WF_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are built", head_dim);
  if (dtype != WF_BF16 && dtype != WF_F32)
    return fail(WF_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  return WF_OK;
}

// The pool of a params struct that begins with it.
template <typename P>
static wf_status check_pool(const P* p) {
  if (!p) return fail(WF_ERR_INVALID_ARG, "params is NULL");
  if (p->pages < 1 || p->heads < 1)
    return fail(WF_ERR_INVALID_ARG, "pages (%d) and heads (%d) must be >= 1", p->pages, p->heads);
  if (p->page_rows < 16 || p->page_rows > 1024 || (p->page_rows & (p->page_rows - 1)) != 0)
    return fail(WF_ERR_UNSUPPORTED, "page_rows %d: powers of two from 16 to 1024 are built",
                p->page_rows);
  WF_TRY(check_rows(p->dtype, p->head_dim));
  if (p->format != WF_CACHE_PLAIN && p->format != WF_CACHE_E4M3 && p->format != WF_CACHE_E2M1)
    return fail(WF_ERR_INVALID_ARG, "unknown cache format %d", p->format);
  if ((long)p->pages * p->page_rows > (1L << 30))
    return fail(WF_ERR_UNSUPPORTED, "more than 2^30 rows in the pool");
  if (p->heads > (1 << 20)) return fail(WF_ERR_UNSUPPORTED, "heads %d exceeds 2^20", p->heads);
  return WF_OK;
}

template <typename P>
static wf_status check_pool_ptrs(const P* p, const void* Kc, const void* Kx, const void* Vc,
                                 const void* Vx) {
  WF_TRY(check_ptr(Kc, "Kc", false));
  WF_TRY(check_ptr(Vc, "Vc", false));
  WF_TRY(check_ptr(Kx, "Kx", p->format == WF_CACHE_PLAIN));
  WF_TRY(check_ptr(Vx, "Vx", p->format == WF_CACHE_PLAIN));
  return WF_OK;
}

template <typename P>
static wf_status check_rotation(const P* p) {
  if (p->rot_dim < 16 || p->rot_dim > p->head_dim || p->rot_dim % 16 != 0)
    return fail(WF_ERR_UNSUPPORTED, "rot_dim %d: multiples of 16 up to head_dim are built",
                p->rot_dim);
  if (p->layout != WF_ROPE_HALVES && p->layout != WF_ROPE_PAIRS)
    return fail(WF_ERR_INVALID_ARG, "unknown layout of pairs %d", p->layout);
  if (p->axes < 1 || p->axes > WF_MAX_ROPE_AXES)
    return fail(WF_ERR_INVALID_ARG, "axes %d outside [1, %d]", p->axes, WF_MAX_ROPE_AXES);
  if (!std::isfinite(p->factor)) return fail(WF_ERR_INVALID_ARG, "factor is not finite");
  for (int i = 0; i < p->rot_dim / 2; ++i)
    if (p->axis[i] >= p->axes)
      return fail(WF_ERR_INVALID_ARG, "axis %d of pair %d: there are %d", p->axis[i], i, p->axes);
  return WF_OK;
}

// A stride of n > 1 places, in elements, of which 16 bytes have `unit`.
static wf_status check_stride(const char* name, int64_t stride, int64_t least, int unit) {
  if (stride < least || stride > (1L << 40) || stride % unit != 0)
    return fail(WF_ERR_INVALID_ARG, "%s %ld: a multiple of %d, at least %ld", name, (long)stride,
                unit, (long)least);
  return WF_OK;
}

static wf_status rope_impl(const wf_rope_params* p, const void* X, const int32_t* pos,
                           const float* freq, void* Y, void* stream) {
  if (!p) return fail(WF_ERR_INVALID_ARG, "params is NULL");
  if (p->batch < 1 || p->heads < 1 || p->rows < 0)
    return fail(WF_ERR_INVALID_ARG, "batch (%d) and heads (%d) must be >= 1, rows (%d) >= 0",
                p->batch, p->heads, p->rows);
  WF_TRY(check_rows(p->dtype, p->head_dim));
  WF_TRY(check_rotation(p));
  if (p->heads > (1 << 20) || (long)p->batch * p->rows > (1L << 30))
    return fail(WF_ERR_UNSUPPORTED, "heads above 2^20 or batch*rows above 2^30");
  const int unit = p->dtype == WF_BF16 ? 8 : 4;
  long xs[3], ys[3];
  const long n[3] = {p->batch, p->heads, p->rows};
  static const char* const xn[3] = {"x_strides[0]", "x_strides[1]", "x_strides[2]"};
  static const char* const yn[3] = {"y_strides[0]", "y_strides[1]", "y_strides[2]"};
  auto whole = [&](const int64_t* s) { return s[0] == 0 && s[1] == 0 && s[2] == 0; };
  const long dense[3] = {(long)p->heads * p->rows * p->head_dim, (long)p->rows * p->head_dim,
                         p->head_dim};
  const bool xw = whole(p->x_strides), yw = whole(p->y_strides);
  for (int i = 0; i < 3; ++i) {
    xs[i] = xw ? dense[i] : n[i] > 1 ? p->x_strides[i] : 0;
    ys[i] = yw ? dense[i] : n[i] > 1 ? p->y_strides[i] : 0;
    if (!xw && n[i] > 1) WF_TRY(check_stride(xn[i], xs[i], 0, unit));
    if (!yw && n[i] > 1) WF_TRY(check_stride(yn[i], ys[i], p->head_dim, unit));
    if (n[i] <= 1) xs[i] = ys[i] = 0;
  }
  if (p->rows == 0) return ok();
  if (rope_groups(*p) * kBlock > UINT32_MAX)
    return fail(WF_ERR_UNSUPPORTED, "too many rows in one call");
  WF_TRY(check_ptr(X, "X", false));
  WF_TRY(check_words(pos, "pos", false));
  WF_TRY(check_words(freq, "inv_freq", false));
  WF_TRY(check_ptr(Y, "Y", false));
  if (X == Y && (xs[0] != ys[0] || xs[1] != ys[1] || xs[2] != ys[2]))
    return fail(WF_ERR_INVALID_ARG, "Y is X, with other strides");
  (void)hipGetLastError();
  WF_HIP(launch_rope(*p, X, pos, freq, Y, xs, ys, static_cast<hipStream_t>(stream)), "rope");
  return ok();
}

static wf_status append_impl(const wf_append_params* p, const void* Q, const void* K,
                             const void* V, const int32_t* pos, const float* freq,
                             const int32_t* slot, void* Kc, void* Kx, void* Vc, void* Vx, void* Qr,
                             void* stream) {
  WF_TRY(check_pool(p));
  if (p->tokens < 0 || p->group < 0)
    return fail(WF_ERR_INVALID_ARG, "tokens (%d) and group (%d) must be >= 0", p->tokens, p->group);
  if (p->rot_dim != 0) WF_TRY(check_rotation(p));
  if (p->tokens > (1 << 30) || (long)p->heads * ((long)p->group + 2) > (1L << 20))
    return fail(WF_ERR_UNSUPPORTED, "tokens above 2^30 or heads*(group + 2) above 2^20");
  const int unit = p->dtype == WF_BF16 ? 8 : 4;
  const long kv = (long)p->heads * p->head_dim, hq = kv * p->group;
  AppendArgs a{};
  auto stride = [&](const char* name, int64_t given, long least, long& out) {
    out = given ? given : least;
    return check_stride(name, out, least, unit);
  };
  WF_TRY(stride("k_row", p->k_row, kv, a.ks));
  WF_TRY(stride("v_row", p->v_row, kv, a.vs));
  WF_TRY(stride("q_row", p->q_row, hq, a.qs));
  WF_TRY(stride("qr_row", p->qr_row, hq, a.os));
  if (p->tokens == 0) return ok();
  if (append_groups(*p) * kBlock > UINT32_MAX)
    return fail(WF_ERR_UNSUPPORTED, "too many rows in one call");
  WF_TRY(check_ptr(Q, "Q", p->group == 0));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_words(pos, "pos", p->rot_dim == 0));
  WF_TRY(check_words(freq, "inv_freq", p->rot_dim == 0));
  WF_TRY(check_words(slot, "slot", false));
  WF_TRY(check_pool_ptrs(p, Kc, Kx, Vc, Vx));
  WF_TRY(check_ptr(Qr, "Qr", p->group == 0));
  if (p->group > 0 && Q == Qr && a.qs != a.os)
    return fail(WF_ERR_INVALID_ARG, "Qr is Q, with another stride");
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.Qr = Qr;
  a.slot = slot;
  a.Kc = Kc;
  a.Kx = static_cast<uint8_t*>(Kx);
  a.Vc = Vc;
  a.Vx = static_cast<uint8_t*>(Vx);
  (void)hipGetLastError();
  WF_HIP(launch_append(*p, a, pos, freq, static_cast<hipStream_t>(stream)), "page_append");
  return ok();
}

static wf_status move_impl(const wf_move_params* p, const int32_t* table, const int32_t* first,
                           const int32_t* source, void* Kc, void* Kx, void* Vc, void* Vx,
                           void* stream) {
  WF_TRY(check_pool(p));
  if (p->batch < 1 || p->table_pages < 1 || p->moves < 0)
    return fail(WF_ERR_INVALID_ARG,
                "batch (%d) and table_pages (%d) must be >= 1, moves (%d) >= 0", p->batch,
                p->table_pages, p->moves);
  if (p->moves > WF_MAX_Q_LEN)
    return fail(WF_ERR_UNSUPPORTED, "moves %d exceeds %d", p->moves, (int)WF_MAX_Q_LEN);
  if (p->moves == 0) return ok();
  if ((long)p->batch * p->heads > (1L << 24) || move_groups(*p) * kBlock > UINT32_MAX)
    return fail(WF_ERR_UNSUPPORTED, "too many sequences and heads in one call");
  WF_TRY(check_words(table, "table", false));
  WF_TRY(check_words(first, "first", false));
  WF_TRY(check_words(source, "source", false));
  WF_TRY(check_pool_ptrs(p, Kc, Kx, Vc, Vx));
  (void)hipGetLastError();
  WF_HIP(launch_move(*p, table, first, source, Kc, Kx, Vc, Vx, static_cast<hipStream_t>(stream)),
         "page_move");
  return ok();
}

static wf_status check_tree(const wf_tree_params* p, size_t have, TreePlan* plan) {
  WF_TRY(check_pool(p));
  if (p->group < 1 || p->batch < 1 || p->tokens < 1 || p->table_pages < 1 || p->max_rows < 1)
    return fail(WF_ERR_INVALID_ARG,
                "group (%d), batch (%d), tokens (%d), table_pages (%d) and max_rows (%d) must be "
                ">= 1",
                p->group, p->batch, p->tokens, p->table_pages, p->max_rows);
  if (p->max_rows > WF_MAX_Q_LEN)
    return fail(WF_ERR_UNSUPPORTED, "max_rows %d exceeds %d", p->max_rows, (int)WF_MAX_Q_LEN);
  if (p->max_len < 0 || p->max_len > (long)p->table_pages * p->page_rows)
    return fail(WF_ERR_INVALID_ARG, "max_len %d outside [0, %ld], the rows of a table", p->max_len,
                (long)p->table_pages * p->page_rows);
  if (p->causal != 0 && p->causal != 1)
    return fail(WF_ERR_INVALID_ARG, "causal %d is neither 0 nor 1", p->causal);
  // as for the prefix: an infinite factor would make a score of 0 NaN
  if (!std::isfinite(p->scale * 1.44269504f))
    return fail(WF_ERR_INVALID_ARG, "scale times log2(e) is not finite in fp32");
  if (p->max_len > (1 << 30)) return fail(WF_ERR_UNSUPPORTED, "more than 2^30 rows");
  // every product below stays in 64 bits: each factor is held to 2^31 in turn
  const long hq = (long)p->heads * p->group;
  if (hq > (1L << 20) || (long)p->tokens * hq > (1L << 30) ||
      (long)p->batch * p->max_rows * hq > (1L << 30))
    return fail(WF_ERR_UNSUPPORTED, "more than 2^20 query heads or 2^30 query rows in one call");
  const int unit = p->dtype == WF_BF16 ? 8 : 4;
  if (p->q_row) WF_TRY(check_stride("q_row", p->q_row, hq * p->head_dim, unit));
  if (p->o_row) WF_TRY(check_stride("o_row", p->o_row, hq * p->head_dim, unit));
  *plan = plan_tree(*p, have);
  // a launch has fewer than 2^32 threads
  if ((plan->items + 7) * 64 * plan->nw > UINT32_MAX || plan->merges * p->batch * kBlock > UINT32_MAX)
    return fail(WF_ERR_UNSUPPORTED, "too many workgroups in one call");
  return WF_OK;
}

static wf_status tree_impl(const wf_tree_params* p, const void* Q, const void* Kc, const void* Kx,
                           const void* Vc, const void* Vx, const int32_t* table,
                           const int32_t* len, const int32_t* row_start, const void* mask, void* O,
                           float* lse, void* ws, size_t ws_bytes, void* stream) {
  TreePlan plan;
  WF_TRY(check_tree(p, ws ? ws_bytes : 0, &plan));
  if (!row_start && p->tokens != (long)p->batch * p->max_rows)
    return fail(WF_ERR_INVALID_ARG, "tokens %d are not batch * max_rows = %ld, without row_start",
                p->tokens, (long)p->batch * p->max_rows);
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_pool_ptrs(p, Kc, Kx, Vc, Vx));
  WF_TRY(check_words(table, "table", false));
  WF_TRY(check_words(len, "len", false));
  WF_TRY(check_words(row_start, "row_start", true));
  WF_TRY(check_words(mask, "mask", true));
  WF_TRY(check_ptr(O, "O", false));
  WF_TRY(check_words(lse, "lse", true));
  if (Q == O) return fail(WF_ERR_INVALID_ARG, "O is Q");
  WF_TRY(check_workspace(ws, ws_bytes, plan.part_bytes + plan.pstat_bytes));
  TreeArgs a{};
  a.Q = Q;
  a.K = Kc;
  a.V = Vc;
  a.Kx = static_cast<const uint8_t*>(Kx);
  a.Vx = static_cast<const uint8_t*>(Vx);
  a.table = table;
  a.len = len;
  a.start = row_start;
  a.mask = static_cast<const uint32_t*>(mask);
  a.O = O;
  a.lse = lse;
  a.part = static_cast<float*>(ws);
  a.pstat = ws ? reinterpret_cast<float*>(at(ws, plan.part_bytes)) : nullptr;
  const long row = (long)p->heads * p->group * p->head_dim;
  a.qs = p->q_row ? p->q_row : row;
  a.os = p->o_row ? p->o_row : row;
  (void)hipGetLastError();
  WF_HIP(launch_tree(*p, plan, a, static_cast<hipStream_t>(stream)), "tree_attn");
  return ok();
}

// ------------------------------------------------------------ shared prefix

static wf_status check_prefix(const wf_prefix_params* p, size_t have, PrefixPlan* plan) {
  if (!p) return fail(WF_ERR_INVALID_ARG, "params is NULL");
  if (p->prefixes < 1 || p->share < 1 || p->heads < 1 || p->group < 1 || p->q_len < 1)
    return fail(WF_ERR_INVALID_ARG,
                "prefixes (%d), share (%d), heads (%d), group (%d) and q_len (%d) must be >= 1",
                p->prefixes, p->share, p->heads, p->group, p->q_len);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(WF_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128 are built", p->head_dim);
  if (p->prefix_cap < 0 || p->prefix_rows < 0 || p->tail_cap < 0)
    return fail(WF_ERR_INVALID_ARG, "prefix_cap (%d), prefix_rows (%d) and tail_cap (%d) must be >= 0",
                p->prefix_cap, p->prefix_rows, p->tail_cap);
  if (p->prefix_rows == 0 && p->tail_cap == 0)
    return fail(WF_ERR_INVALID_ARG, "neither prefix rows nor own rows");
  if (p->prefix_rows > 0 && p->prefix_cap == 0)
    return fail(WF_ERR_INVALID_ARG, "prefix_rows %d of an empty prefix", p->prefix_rows);
  if (p->prefix_cap > (1 << 30) || p->prefix_rows > (1 << 30) || p->tail_cap > (1 << 30))
    return fail(WF_ERR_UNSUPPORTED, "more than 2^30 rows");
  if (p->dtype != WF_BF16 && p->dtype != WF_F32)
    return fail(WF_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
  if (p->format != WF_CACHE_PLAIN && p->format != WF_CACHE_E4M3 && p->format != WF_CACHE_E2M1)
    return fail(WF_ERR_INVALID_ARG, "unknown cache format %d", p->format);
  // the kernels scale scores in log2 units: an infinite factor would make a score of 0 NaN
  if (!std::isfinite(p->scale * 1.44269504f))
    return fail(WF_ERR_INVALID_ARG, "scale times log2(e) is not finite in fp32");
  // every product below stays in 64 bits: each factor is held to 2^31 in turn
  long rows = 1;
  for (long f : {(long)p->prefixes, (long)p->share, (long)p->heads, (long)p->group, (long)p->q_len}) {
    rows *= f;
    if (rows > (1L << 30))
      return fail(WF_ERR_UNSUPPORTED, "more than 2^30 query rows in one call");
  }
  *plan = plan_prefix(*p, have);
  // a launch has fewer than 2^32 threads
  if ((plan->items + 7) * 64 * plan->nw > UINT32_MAX || plan->titems * kBlock > UINT32_MAX)
    return fail(WF_ERR_UNSUPPORTED, "too many workgroups in one call");
  return WF_OK;
}

static wf_status prefix_impl(const wf_prefix_params* p, const void* Q, const void* K,
                             const void* Kx, const void* V, const void* Vx,
                             const int32_t* row_idx, const int32_t* prefix_len, const void* Kt,
                             const void* Vt, const int32_t* tail_len, void* O, float* lse,
                             void* ws, size_t ws_bytes, void* stream) {
  PrefixPlan plan;
  WF_TRY(check_prefix(p, ws ? ws_bytes : 0, &plan));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(O, "O", false));
  WF_TRY(check_ptr(lse, "lse", true));
  WF_TRY(check_ptr(row_idx, "row_idx", true));
  WF_TRY(check_ptr(prefix_len, "prefix_len", true));
  WF_TRY(check_ptr(tail_len, "tail_len", true));
  if (p->prefix_rows > 0) {
    WF_TRY(check_ptr(K, "K", false));
    WF_TRY(check_ptr(V, "V", false));
    if (p->format != WF_CACHE_PLAIN) {
      WF_TRY(check_ptr(Kx, "Kx", false));
      WF_TRY(check_ptr(Vx, "Vx", false));
    }
    if (!row_idx && p->prefix_rows > p->prefix_cap)
      return fail(WF_ERR_INVALID_ARG, "prefix_rows %d exceeds prefix_cap %d", p->prefix_rows,
                  p->prefix_cap);
  }
  if (p->tail_cap > 0) {
    WF_TRY(check_ptr(Kt, "Kt", false));
    WF_TRY(check_ptr(Vt, "Vt", false));
  }
  WF_TRY(check_workspace(ws, ws_bytes, plan.part_bytes + plan.pstat_bytes));
  (void)hipGetLastError();
  PrefixArgs a{};
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.Kx = static_cast<const uint8_t*>(Kx);
  a.Vx = static_cast<const uint8_t*>(Vx);
  a.list = row_idx;
  a.plen = prefix_len;
  a.Kt = Kt;
  a.Vt = Vt;
  a.tlen = tail_len;
  a.O = O;
  a.lse = lse;
  a.part = static_cast<float*>(ws);
  a.pstat = ws ? reinterpret_cast<float*>(at(ws, plan.part_bytes)) : nullptr;
  WF_HIP(launch_prefix(*p, plan, a, static_cast<hipStream_t>(stream)), "prefix_attn");
  return ok();
}

}  // namespace wf

using namespace wf;

extern "C" {

size_t wf_workspace_bytes(const wf_params* p, int32_t op) {
  if (check_params(p) != WF_OK) return 0;
  if (op < WF_OP_SKIM || op > WF_OP_SHARED) return 0;
  const long rows = keff_of(*p) + remainder_len(*p) + p->gen_len;
  int fine;
  const size_t total = layout_in(*p, op, rows, SIZE_MAX, &fine).total;
  if (op != WF_OP_ATTN) return total;
  // enough for a call with fewer rows too
  const size_t splits = (size_t)p->batch * p->heads * most_attn_splits(*p, rows) * p->q_len;
  return std::max(total, up256(splits * p->head_dim * sizeof(float)) +
                             up256(splits * 2 * sizeof(float)));
}

int32_t wf_effective_budget(const wf_params* p) {
  if (check_params(p) != WF_OK) return -1;
  return (int32_t)keff_of(*p);
}

wf_status wf_dwt_keys(const wf_params* p, const void* K, float* approx,
                      float* details, void* stream) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(approx, "approx", false));
  WF_TRY(check_ptr(details, "details", true));
  (void)hipGetLastError();
  WF_HIP(launch_dwt(*p, K, approx, details, static_cast<hipStream_t>(stream)),
         "dwt");
  return ok();
}

wf_status wf_skim_score(const wf_params* p, const void* Q, const float* approx,
                        float* seg_score, int32_t* seg_idx, void* workspace,
                        size_t workspace_bytes, void* stream) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(approx, "approx", false));
  WF_TRY(check_ptr(seg_score, "seg_score", false));
  WF_TRY(check_ptr(seg_idx, "seg_idx", false));
  int fine;
  const Layout l = layout_in(*p, WF_OP_SKIM, 0, workspace_bytes, &fine);
  WF_TRY(check_workspace(workspace, workspace_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const SkimPlan sp = plan_skim(*p, false, fine);
  float* logits = reinterpret_cast<float*>(at(workspace, l.logits));
  float* sstats = reinterpret_cast<float*>(at(workspace, l.sstats));
  (void)hipGetLastError();
  WF_HIP(launch_skim_tiles(*p, false, Q, nullptr, approx, logits, sstats, fine, s),
         "skim_tile");
  WF_HIP(launch_skim_select(*p, sp.ntiles, logits, sstats, seg_score, seg_idx, s),
         "skim_select");
  return ok();
}

wf_status wf_scan_select(const wf_params* p, const void* Q, const void* K,
                         const int32_t* seg_idx, float* tok_score,
                         int32_t* tok_idx, void* workspace,
                         size_t workspace_bytes, void* stream) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(seg_idx, "seg_idx", false));
  WF_TRY(check_ptr(tok_score, "tok_score", true));
  WF_TRY(check_ptr(tok_idx, "tok_idx", false));
  int fine;
  const Layout l = layout_in(*p, WF_OP_SCAN, 0, workspace_bytes, &fine);
  WF_TRY(check_workspace(workspace, workspace_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* cstats = reinterpret_cast<float*>(at(workspace, l.cstats));
  float* wpool = tok_score ? tok_score : reinterpret_cast<float*>(at(workspace, l.wpool));
  (void)hipGetLastError();
  WF_HIP(launch_scan_chunks(*p, 0, Q, K, seg_idx, cstats, wpool, fine, s), "scan_stats");
  WF_HIP(launch_scan_chunks(*p, 1, Q, K, seg_idx, cstats, wpool, fine, s), "scan_weights");
  WF_HIP(launch_scan_select(*p, wpool, seg_idx, tok_idx, s), "scan_select");
  return ok();
}

wf_status wf_gather_kv(const wf_params* p, const void* K, const void* V,
                       const int32_t* tok_idx, const void* Kg, const void* Vg,
                       void* Ks, void* Vs, void* stream) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(K, "K", false));
  WF_TRY(check_ptr(V, "V", false));
  WF_TRY(check_ptr(tok_idx, "tok_idx", false));
  WF_TRY(check_ptr(Ks, "Ks", false));
  WF_TRY(check_ptr(Vs, "Vs", false));
  if (p->gen_len > 0) {
    WF_TRY(check_ptr(Kg, "Kg", false));
    WF_TRY(check_ptr(Vg, "Vg", false));
  }
  (void)hipGetLastError();
  WF_HIP(launch_gather(*p, K, V, tok_idx, Kg, Vg, Ks, Vs,
                       static_cast<hipStream_t>(stream)),
         "gather");
  return ok();
}

wf_status wf_sparse_attn(const wf_params* p, const void* Q, const void* Ks,
                         const void* Vs, int32_t n_kv, void* O,
                         void* workspace, size_t workspace_bytes,
                         void* stream) {
  WF_TRY(check_params(p));
  WF_TRY(check_ptr(Q, "Q", false));
  WF_TRY(check_ptr(Ks, "Ks", false));
  WF_TRY(check_ptr(Vs, "Vs", false));
  WF_TRY(check_ptr(O, "O", false));
  if (n_kv < 1) return fail(WF_ERR_INVALID_ARG, "n_kv %d < 1", n_kv);
  int fine;
  const Layout l = layout_in(*p, WF_OP_ATTN, n_kv, workspace_bytes, &fine);
  WF_TRY(check_workspace(workspace, workspace_bytes, l.total));
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* part = reinterpret_cast<float*>(at(workspace, l.part));
  float* pstat = reinterpret_cast<float*>(at(workspace, l.pstat));
  (void)hipGetLastError();
  WF_HIP(launch_attn(*p, Q, Ks, Vs, nullptr, n_kv, nullptr, nullptr, 0, n_kv,
                     part, pstat, fine, s),
         "sparse_attn");
  WF_HIP(launch_attn_combine(*p, n_kv, part, pstat, O, fine, s), "attn_combine");
  return ok();
}

wf_status wf_filter_attend(const wf_params* p, const void* Q, const void* K,
                           const void* V, const void* Kg, const void* Vg,
                           void* O, int32_t* tok_idx, int32_t* seg_idx,
                           void* workspace, size_t workspace_bytes,
                           void* stream) {
  return fused_impl(p, Q, K, V, Kg, Vg, O, tok_idx, seg_idx, workspace,
                    workspace_bytes, stream, nullptr, 0);
}

wf_status wf_filter_attend_timed(const wf_params* p, const void* Q,
                                 const void* K, const void* V, const void* Kg,
                                 const void* Vg, void* O, int32_t* tok_idx,
                                 int32_t* seg_idx, void* workspace,
                                 size_t workspace_bytes, void* stream,
                                 void** events, int32_t n_events) {
  if (!events) return fail(WF_ERR_INVALID_ARG, "events is NULL");
  for (int i = 0; i < n_events && i <= kMaxFusedKernels; ++i)
    if (!events[i]) return fail(WF_ERR_INVALID_ARG, "events[%d] is NULL", i);
  return fused_impl(p, Q, K, V, Kg, Vg, O, tok_idx, seg_idx, workspace,
                    workspace_bytes, stream, events, n_events);
}

wf_status wf_filter_attend_noalloc(const wf_params* p, const void* Q, const void* K,
                                   const void* V, const void* Kg, const void* Vg, void* O,
                                   int32_t* tok_idx, int32_t* seg_idx, void* stream) {
  return noalloc_impl(p, Q, K, V, Kg, Vg, O, tok_idx, seg_idx, stream);
}

int32_t wf_filter_attend_kernels(const wf_params* p) {
  if (check_params(p) != WF_OK) return -1;
  return fused_kernels(*p);
}

const char* wf_filter_attend_kernel_name(const wf_params* p, int32_t i) {
  if (check_params(p) != WF_OK || i < 0 || i >= fused_kernels(*p)) return nullptr;
  return fused_names(*p)[i];
}

wf_status wf_filter_attend_shared(const wf_params* p, const void* Q, const void* K,
                                  const void* V, const void* Kg, const void* Vg, void* O,
                                  int32_t* tok_idx, int32_t* seg_idx, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  return shared_impl(p, Q, K, V, Kg, Vg, O, tok_idx, seg_idx, workspace, workspace_bytes,
                     stream, nullptr, 0);
}

wf_status wf_filter_attend_shared_timed(const wf_params* p, const void* Q, const void* K,
                                        const void* V, const void* Kg, const void* Vg,
                                        void* O, int32_t* tok_idx, int32_t* seg_idx,
                                        void* workspace, size_t workspace_bytes,
                                        void* stream, void** events, int32_t n_events) {
  if (!events) return fail(WF_ERR_INVALID_ARG, "events is NULL");
  for (int i = 0; i < n_events && i <= kSharedMaxKernels; ++i)
    if (!events[i]) return fail(WF_ERR_INVALID_ARG, "events[%d] is NULL", i);
  return shared_impl(p, Q, K, V, Kg, Vg, O, tok_idx, seg_idx, workspace, workspace_bytes,
                     stream, events, n_events);
}

int32_t wf_filter_attend_shared_kernels(const wf_params* p) {
  if (check_params(p) != WF_OK) return -1;
  return shared_kernels(*p);
}

const char* wf_filter_attend_shared_kernel_name(const wf_params* p, int32_t i) {
  if (check_params(p) != WF_OK || i < 0 || i >= shared_kernels(*p)) return nullptr;
  return shared_names(*p)[i];
}

wf_status wf_filter_attend_cached(const wf_params* p, const void* Q, const float* approx,
                                  const void* K, const void* V, const void* Kg,
                                  const void* Vg, void* O, int32_t* tok_idx,
                                  int32_t* seg_idx, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  return cached_impl(p, Q, approx, K, V, Kg, Vg, O, tok_idx, seg_idx, workspace,
                     workspace_bytes, stream, nullptr, 0);
}

wf_status wf_filter_attend_cached_timed(const wf_params* p, const void* Q,
                                        const float* approx, const void* K, const void* V,
                                        const void* Kg, const void* Vg, void* O,
                                        int32_t* tok_idx, int32_t* seg_idx, void* workspace,
                                        size_t workspace_bytes, void* stream, void** events,
                                        int32_t n_events) {
  if (!events) return fail(WF_ERR_INVALID_ARG, "events is NULL");
  for (int i = 0; i < n_events && i <= cached_kernels(*p); ++i)
    if (!events[i]) return fail(WF_ERR_INVALID_ARG, "events[%d] is NULL", i);
  return cached_impl(p, Q, approx, K, V, Kg, Vg, O, tok_idx, seg_idx, workspace,
                     workspace_bytes, stream, events, n_events);
}

int32_t wf_filter_attend_cached_kernels(const wf_params* p) {
  if (check_params(p) != WF_OK) return -1;
  return cached_kernels(*p);
}

const char* wf_filter_attend_cached_kernel_name(const wf_params* p, int32_t i) {
  if (check_params(p) != WF_OK || i < 0 || i >= cached_kernels(*p)) return nullptr;
  return cached_names(*p)[i];
}

wf_status wf_recursion_counts(const wf_params* p, const float* proportions,
                              int32_t* counts) {
  int32_t c[WF_MAX_LEVELS];
  if (!counts) return fail(WF_ERR_INVALID_ARG, "counts is NULL");
  WF_TRY(check_recursion(p, proportions, c));
  for (int b = 0; b < p->levels; ++b) counts[b] = c[b];
  return ok();
}

size_t wf_recursive_workspace_bytes(const wf_params* p, const float* proportions) {
  int32_t c[WF_MAX_LEVELS];
  if (check_recursion(p, proportions, c) != WF_OK) return 0;
  int fine;
  return rec_layout_in(*p, c, SIZE_MAX, &fine).total;
}

wf_status wf_filter_attend_recursive(const wf_params* p, const float* proportions,
                                     const void* Q, const void* K, const void* V,
                                     const void* Kg, const void* Vg, void* O,
                                     int32_t* tok_idx, int32_t* kept_idx, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  return recursive_impl(p, proportions, Q, K, V, Kg, Vg, O, tok_idx, kept_idx, workspace,
                        workspace_bytes, stream, nullptr, 0);
}

wf_status wf_filter_attend_recursive_timed(const wf_params* p, const float* proportions,
                                           const void* Q, const void* K, const void* V,
                                           const void* Kg, const void* Vg, void* O,
                                           int32_t* tok_idx, int32_t* kept_idx,
                                           void* workspace, size_t workspace_bytes,
                                           void* stream, void** events, int32_t n_events) {
  if (!events) return fail(WF_ERR_INVALID_ARG, "events is NULL");
  WF_TRY(check_shape(p));
  for (int i = 0; i < n_events && i <= rec_kernels(*p); ++i)
    if (!events[i]) return fail(WF_ERR_INVALID_ARG, "events[%d] is NULL", i);
  return recursive_impl(p, proportions, Q, K, V, Kg, Vg, O, tok_idx, kept_idx, workspace,
                        workspace_bytes, stream, events, n_events);
}

int32_t wf_filter_attend_recursive_kernels(const wf_params* p) {
  if (check_shape(p) != WF_OK) return -1;
  return rec_kernels(*p);
}

const char* wf_filter_attend_recursive_kernel_name(const wf_params* p, int32_t i) {
  if (check_shape(p) != WF_OK || i < 0 || i >= rec_kernels(*p)) return nullptr;
  return rec_kernel_name(*p, i);
}

wf_status wf_cache_store(const wf_cache_params* p, const void* K, const void* V,
                         const int32_t* row_idx, void* Kc, void* Kx, void* Vc, void* Vx,
                         void* stream) {
  return cache_impl(p, true, K, V, row_idx, Kc, Kx, Vc, Vx, stream);
}

wf_status wf_cache_load(const wf_cache_params* p, const void* Kc, const void* Kx, const void* Vc,
                        const void* Vx, const int32_t* row_idx, void* K, void* V, void* stream) {
  return cache_impl(p, false, K, V, row_idx, Kc, Kx, Vc, Vx, stream);
}

wf_status wf_rope(const wf_rope_params* p, const void* X, const int32_t* pos,
                  const float* inv_freq, void* Y, void* stream) {
  return rope_impl(p, X, pos, inv_freq, Y, stream);
}

wf_status wf_page_append(const wf_append_params* p, const void* Q, const void* K, const void* V,
                         const int32_t* pos, const float* inv_freq, const int32_t* slot, void* Kc,
                         void* Kx, void* Vc, void* Vx, void* Qr, void* stream) {
  return append_impl(p, Q, K, V, pos, inv_freq, slot, Kc, Kx, Vc, Vx, Qr, stream);
}

wf_status wf_page_move(const wf_move_params* p, const int32_t* table, const int32_t* first,
                       const int32_t* source, void* Kc, void* Kx, void* Vc, void* Vx,
                       void* stream) {
  return move_impl(p, table, first, source, Kc, Kx, Vc, Vx, stream);
}

size_t wf_tree_workspace_bytes(const wf_tree_params* p) {
  TreePlan plan;
  if (check_tree(p, SIZE_MAX, &plan) != WF_OK) return 0;
  return plan.part_bytes + plan.pstat_bytes;
}

wf_status wf_tree_plan(const wf_tree_params* p, size_t workspace_bytes, wf_prefix_split* split) {
  TreePlan plan;
  WF_TRY(check_tree(p, workspace_bytes, &plan));
  if (!split) return fail(WF_ERR_INVALID_ARG, "split is NULL");
  const int wave = plan.few ? plan.few : 32 * plan.qw;
  *split = wf_prefix_split{plan.splits, plan.rps, plan.nw / plan.kw * wave, wave, plan.kw};
  return ok();
}

wf_status wf_tree_attn(const wf_tree_params* p, const void* Q, const void* Kc, const void* Kx,
                       const void* Vc, const void* Vx, const int32_t* table, const int32_t* len,
                       const int32_t* row_start, const void* mask, void* O, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream) {
  return tree_impl(p, Q, Kc, Kx, Vc, Vx, table, len, row_start, mask, O, lse, workspace,
                   workspace_bytes, stream);
}

size_t wf_prefix_workspace_bytes(const wf_prefix_params* p) {
  PrefixPlan plan;
  if (check_prefix(p, SIZE_MAX, &plan) != WF_OK) return 0;
  return plan.part_bytes + plan.pstat_bytes;
}

wf_status wf_prefix_plan(const wf_prefix_params* p, size_t workspace_bytes,
                         wf_prefix_split* split) {
  PrefixPlan plan;
  WF_TRY(check_prefix(p, workspace_bytes, &plan));
  if (!split) return fail(WF_ERR_INVALID_ARG, "split is NULL");
  *split = wf_prefix_split{};
  if (p->prefix_rows > 0)
    *split = wf_prefix_split{plan.splits, plan.rps, plan.nw / plan.kw * 32 * plan.qw,
                             32 * plan.qw, plan.kw};
  return ok();
}

wf_status wf_prefix_attn(const wf_prefix_params* p, const void* Q, const void* K, const void* Kx,
                         const void* V, const void* Vx, const int32_t* row_idx,
                         const int32_t* prefix_len, const void* Kt, const void* Vt,
                         const int32_t* tail_len, void* O, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
  return prefix_impl(p, Q, K, Kx, V, Vx, row_idx, prefix_len, Kt, Vt, tail_len, O, lse, workspace,
                     workspace_bytes, stream);
}

wf_status wf_init(void) {
  WF_HIP(load_fast_kernels(), "loading the token-skim kernels");
  WF_HIP(load_scan_kernels(), "loading the scan kernels");
  WF_HIP(load_attn_kernels(), "loading the attention kernels");
  WF_HIP(load_skim_kernels(), "loading the skim kernels");
  WF_HIP(load_dwt_kernels(), "loading the DWT kernels");
  WF_HIP(load_cache_kernels(), "loading the cache kernels");
  WF_HIP(load_prefix_kernels(), "loading the prefix-attention kernels");
  WF_HIP(load_page_kernels(), "loading the kernels of a cache in pages");
  WF_HIP(load_tree_kernels(), "loading the attention over a cache in pages");
  void* scratch_ptr = nullptr;  // this file's code object and its scratch array
  WF_TRY(scratch_of_current_device(&scratch_ptr));
  return ok();
}

const char* wf_status_str(wf_status s) {
  switch (s) {
    case WF_OK: return "WF_OK";
    case WF_ERR_INVALID_ARG: return "WF_ERR_INVALID_ARG";
    case WF_ERR_UNSUPPORTED: return "WF_ERR_UNSUPPORTED";
    case WF_ERR_WORKSPACE: return "WF_ERR_WORKSPACE";
    case WF_ERR_HIP: return "WF_ERR_HIP";
  }
  return "WF_ERR_UNKNOWN";
}

const char* wf_last_error(void) { return g_last_error; }

}  // extern "C"
