// C ABI of libstepprune (include/stepprune.h): host-side validation, workspace
// layout and launch order.  Every entry point validates its arguments before
// touching the device and never throws.
#include <float.h>
#include <string.h>

#include <mutex>

#include <rocprofiler-sdk-roctx/roctx.h>

#include "sp_internal.h"

using namespace sp;

namespace {

// A roctx range named after the entry point around each call (host-side
// enqueue), so a marker trace shows the three stages of Algorithm 1.
struct TraceRange {
  explicit TraceRange(const char* name) { roctxRangePushA(name); }
  ~TraceRange() { roctxRangePop(); }
  TraceRange(const TraceRange&) = delete;
  TraceRange& operator=(const TraceRange&) = delete;
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

sp_status check_dims(const sp_dims* d) {
  if (!d) return SP_EINVAL;
  if (d->d <= 0 || d->d_text <= 0 || d->h <= 0) return SP_EINVAL;
  if (d->d % 64 || d->d_text % 64 || d->h % 64) return SP_EINVAL;
  if (d->dtype != SP_F32 && d->dtype != SP_BF16) return SP_EUNSUPPORTED;
  if (d->h > 1024) return SP_EUNSUPPORTED;
  if (d->dtype == SP_F32 && d->h > 512) return SP_EUNSUPPORTED;
  return SP_OK;
}

int elem_bytes(const sp_dims* d) { return d->dtype == SP_F32 ? 4 : 2; }

struct SelectWs {
  size_t gram, kept, count, total;
  int64_t gstride;
  int gram_ld;
};

// Header; Gram blocks [G][2 (max_group + 1) + 3][ld] float32; group-local kept
// lists; group counts.
SelectWs select_ws_layout(int G, int max_group, int max_cap) {
  SelectWs w;
  w.gram_ld = (int)align_up((size_t)max_group + 2, 4);
  w.gstride = (int64_t)(2 * (max_group + 1) + kGramExtraRows) * w.gram_ld;
  size_t off = kWsHeaderBytes;
  w.gram = off;
  off = align_up(off + (size_t)G * w.gstride * 4, 256);
  w.kept = off;
  off = align_up(off + (size_t)G * (max_cap > 0 ? max_cap : 1) * 4, 256);
  w.count = off;
  off = align_up(off + (size_t)G * 4, 256);
  w.total = off;
  return w;
}

// Header, then the text projection's K-split partial products [split][T_txt][h].
size_t project_ws_bytes(const sp_dims* d, int64_t T_txt) {
  const size_t split = (size_t)text_split(d->dtype, T_txt, d->h, d->d_text);
  return kWsHeaderBytes + align_up(split * (size_t)T_txt * d->h * 4, 256);
}

sp_status hip_status(hipError_t e) { return e == hipSuccess ? SP_OK : SP_EHIP; }

// Header, then the gate and denoiser's intermediates: x~ / h float32 [T, d],
// two bfloat16 [T, d] buffers and the bfloat16 [T, 4d] hidden activations.
struct GateWs {
  size_t xt, p, q, hid, total;
};
GateWs gate_ws_layout(const sp_dims* d, int64_t T) {
  GateWs w;
  const size_t td = (size_t)T * d->d;
  w.xt = kWsHeaderBytes;
  w.p = align_up(w.xt + td * 4, 256);
  w.q = align_up(w.p + td * 2, 256);
  w.hid = align_up(w.q + td * 2, 256);
  w.total = align_up(w.hid + td * 4 * 2, 256);
  return w;
}

// Header, then the encoder's buffers (sp_internal.h, EncodeArgs).
struct EncodeWs {
  size_t R, L, A, QKV, HID, total;
};
EncodeWs encode_ws_layout(const sp_dims* d, int64_t T_vis, int64_t T_txt) {
  EncodeWs w;
  const size_t S = (size_t)(T_vis + T_txt), dd = (size_t)d->d;
  w.R = kWsHeaderBytes;
  w.L = align_up(w.R + S * dd * 4, 256);
  w.A = align_up(w.L + S * dd * 2, 256);
  w.QKV = align_up(w.A + S * dd * 2, 256);
  w.HID = align_up(w.QKV + S * dd * 3 * 2, 256);
  w.total = align_up(w.HID + S * dd * 4 * 2, 256);
  return w;
}

// The encoder takes bfloat16, d a multiple of 128 (heads of width 128) up to
// 4096 (the row kernels keep a row in one wave's registers).
sp_status check_encode_dims(const sp_dims* d) {
  sp_status st = check_dims(d);
  if (st != SP_OK) return st;
  if (d->dtype != SP_BF16 || d->d % 128 || d->d > 4096) return SP_EUNSUPPORTED;
  return SP_OK;
}

// The cache's structs, checked into the kernels' form.
sp_status check_cache_dims(const sp_cache_dims* d, CacheShape& s) {
  if (!d) return SP_EINVAL;
  if (d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads || d->head_dim < 1 ||
      d->page_size < 1 || d->pages < 1)
    return SP_EINVAL;
  if (d->dtype != SP_F32 && d->dtype != SP_BF16) return SP_EUNSUPPORTED;
  if (d->head_dim != 64 && d->head_dim != 128) return SP_EUNSUPPORTED;
  if (d->q_heads > kMaxCacheHeads) return SP_EUNSUPPORTED;
  s.page_shift = 4;
  while (s.page_shift < 8 && (1 << s.page_shift) != d->page_size) ++s.page_shift;
  if ((1 << s.page_shift) != d->page_size) return SP_EUNSUPPORTED;
  s.q_heads = d->q_heads;
  s.kv_heads = d->kv_heads;
  s.head_dim = d->head_dim;
  s.dtype = d->dtype;
  s.pages = d->pages;
  return SP_OK;
}

// Device pointers are looked at only with `pointers` (the workspace query has none).
sp_status check_cache_runs(const sp_cache_runs* r, const CacheShape& s, bool pointers, CacheRuns& o) {
  if (!r) return SP_EINVAL;
  if (r->count < 0 || r->table_width < 0 || r->max_len < 0) return SP_EINVAL;
  if (r->max_len > (int64_t)r->table_width << s.page_shift) return SP_EINVAL;
  if (r->max_len > kMaxCacheTokens || r->count > kMaxCacheRuns) return SP_EUNSUPPORTED;
  if (pointers && r->count > 0 && (!r->len || (r->max_len > 0 && !r->table))) return SP_EINVAL;
  o.table = r->table;
  o.len = r->len;
  o.count = r->count;
  o.width = r->max_len > 0 ? r->table_width : 0;     // (runs of no tokens need no table)
  o.max_len = r->max_len;
  return SP_OK;
}

sp_status check_cache_rows(const sp_cache_rows* r, const CacheShape& s, int S, bool pointers, CacheRows& o) {
  if (!r) return SP_EINVAL;
  if (r->rows < 0 || r->max_rows < 0) return SP_EINVAL;
  if (r->layout != SP_LAYOUT_PADDED && r->layout != SP_LAYOUT_PACKED) return SP_EINVAL;
  o.padded = r->layout == SP_LAYOUT_PADDED;
  if (o.padded && (r->rows_per_seq < 0 || (int64_t)r->rows_per_seq * S > r->rows)) return SP_EINVAL;
  if (pointers && S > 0 && !r->seq_info) return SP_EINVAL;
  if (r->rows > (int64_t)kMaxCacheRows / (s.q_heads / s.kv_heads)) return SP_EUNSUPPORTED;
  o.rows = r->rows;
  o.rows_per_seq = o.padded ? r->rows_per_seq : 0;
  o.info = r->seq_info;
  // no sequence is longer than its slice or the arrays, however large a bound is passed
  const int64_t most = o.padded ? o.rows_per_seq : o.rows;
  o.max_rows = r->max_rows < most ? r->max_rows : (int)most;
  return SP_OK;
}

sp_status check_attend(const sp_cache_dims* dims, const sp_cache_rows* rows, const sp_cache_runs* runs,
                       const sp_cache_runs* prefix, bool pointers, AttendArgs& a) {
  sp_status st = check_cache_dims(dims, a.shape);
  if (st == SP_OK) st = check_cache_runs(runs, a.shape, pointers, a.runs);
  if (st == SP_OK) st = check_cache_rows(rows, a.shape, a.runs.count, pointers, a.rows);
  a.prefix = CacheRuns{};
  if (st == SP_OK && prefix) st = check_cache_runs(prefix, a.shape, pointers, a.prefix);
  if (st != SP_OK) return st;
  a.plan = plan_cache_attend(a.shape, a.rows, a.runs, a.prefix);
  return cache_attend_fits(a) ? SP_OK : SP_EUNSUPPORTED;
}

// Header; parts of every row; the parts' maxima and sums, and their outputs (none where
// a row has one part at most, which is its output).
struct AttendWs {
  size_t row_parts, ml[3], o[3], total;              // short, prefix, tall
};
AttendWs attend_ws_layout(const AttendArgs& a) {
  const AttendPlan& p = a.plan;
  const size_t brief = (size_t)short_slots(a);
  const bool joined = p.prefix_parts > 0 || p.short_parts > 1;
  const size_t n[3] = {joined ? brief * p.short_parts : 0, brief * p.prefix_parts,
                       p.tall_parts > 1 ? (size_t)a.rows.rows * a.shape.q_heads * p.tall_parts : 0};
  AttendWs w;
  w.row_parts = kWsHeaderBytes;
  w.total = align_up(w.row_parts + (size_t)a.rows.rows * sizeof(int2), 256);
  for (int i = 0; i < 3; ++i) {
    w.ml[i] = w.total;
    w.o[i] = align_up(w.ml[i] + n[i] * 2 * 4, 256);
    w.total = align_up(w.o[i] + n[i] * a.shape.head_dim * 4, 256);
  }
  return w;
}

}  // namespace

extern "C" {

const char* stepprune_status_string(sp_status s) {
  // A C caller may pass any int: read its bytes, since loading an enumeration
  // outside its enumerators' range is undefined in C++.
  static_assert(sizeof(sp_status) == sizeof(int32_t), "sp_status is int-sized");
  int32_t v;
  memcpy(&v, &s, sizeof(v));
  switch (v) {
    case SP_OK: return "ok";
    case SP_EINVAL: return "invalid argument";
    case SP_EUNSUPPORTED: return "unsupported argument";
    case SP_EWORKSPACE: return "workspace too small";
    case SP_EHIP: return "HIP runtime error";
    case SP_EDEVICE: return "device-side error (see stepprune_read_device_error)";
  }
  return "unknown status";
}

size_t stepprune_workspace_bytes(int32_t which, const sp_dims* dims, int64_t T_vis, int64_t T_txt,
                                 int32_t B, int32_t G, int32_t max_group, int32_t max_cap) {
  if (check_dims(dims) != SP_OK || T_vis < 0 || T_txt < 0 || B < 0 || G < 0) return 0;
  switch (which) {
    case 0: return project_ws_bytes(dims, T_txt);
    case 1:
      if (max_group < 0 || max_group > kMaxGroup || max_cap < 0) return 0;
      return select_ws_layout(G, max_group, max_cap).total;
    case 2: return kWsHeaderBytes;
    case 3:
      if (dims->dtype != SP_BF16 || dims->d > 4096) return 0;
      return gate_ws_layout(dims, T_vis).total;
    case 4:
      if (check_encode_dims(dims) != SP_OK || B < 1 || max_group < 1) return 0;
      return encode_ws_layout(dims, T_vis, T_txt).total;
  }
  return 0;
}

sp_status stepprune_project(const sp_dims* dims, const void* X, int64_t T_vis, const void* s_start,
                            const void* s_stop, const void* W_kqv, const void* E_text,
                            const int32_t* text_off, int32_t B, int64_t T_txt, const void* W_text,
                            float g_text, float ln_eps, void* KQV, float* ctx, void* ws,
                            size_t ws_bytes, const hipEvent_t* events, hipStream_t stream) {
  const TraceRange range("stepprune_project");
  sp_status st = check_dims(dims);
  if (st != SP_OK) return st;
  if (T_vis < 0 || T_txt < 0 || B < 1) return SP_EINVAL;
  if (!s_start || !s_stop || !W_kqv || !KQV || !ctx || !text_off || !W_text || !ws) return SP_EINVAL;
  if ((T_vis > 0 && !X) || (T_txt > 0 && !E_text)) return SP_EINVAL;
  if (!aligned16(X) || !aligned16(s_start) || !aligned16(s_stop) || !aligned16(W_kqv) ||
      !aligned16(E_text) || !aligned16(W_text) || !aligned16(KQV) || !aligned16(ctx) ||
      !aligned16(ws))
    return SP_EINVAL;
  if (!(ln_eps >= 0.0f)) return SP_EINVAL;
  if (ws_bytes < project_ws_bytes(dims, T_txt)) return SP_EWORKSPACE;

  int32_t* err = reinterpret_cast<int32_t*>(ws);
  float* tproj = reinterpret_cast<float*>(static_cast<char*>(ws) + kWsHeaderBytes);
  record_event(events, 0, stream);
  hipError_t e = launch_project_gemm(dims->dtype, X, T_vis, s_start, s_stop, W_kqv, dims->d,
                                     3 * dims->h, KQV, E_text, T_txt, W_text, dims->d_text,
                                     dims->h, tproj, stream);
  record_event(events, 1, stream);
  if (e == hipSuccess)
    e = launch_text_pool(tproj, text_split(dims->dtype, T_txt, dims->h, dims->d_text), text_off, B,
                         T_txt, dims->h, g_text, ln_eps, ctx, err, stream);
  return hip_status(e);
}

}  // extern "C"

namespace {

// ------------------------------------------------------------ fixed scratch
// The scratch of stepprune_select_noalloc: one array in device memory, a copy
// per GPU, held until the process ends.  In host code the array's name is a
// stand-in, not a device address: host code uses only the address that
// hipGetSymbolAddress returns for the current device, fetched once per device
// and kept in scratch_ptr.
static __device__ __align__(256) char scratch[STEPPRUNE_NOALLOC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex scratch_mu;
void* scratch_ptr[kMaxDevices];

// The scratch address on the device that owns `stream` (it must be the
// current device: the symbol is looked up with that device current).
sp_status device_scratch(hipStream_t stream, void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return SP_EHIP;
  if (stream) {
    hipDevice_t sdev = -1;
    if (hipStreamGetDevice(stream, &sdev) != hipSuccess) return SP_EHIP;
    if (sdev != dev) return SP_EINVAL;
  }
  if (dev < 0 || dev >= kMaxDevices) return SP_EUNSUPPORTED;
  std::lock_guard<std::mutex> lock(scratch_mu);
  if (!scratch_ptr[dev]) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return SP_EHIP;
    scratch_ptr[dev] = p;
  }
  *out = scratch_ptr[dev];
  return SP_OK;
}

// Shared body of stepprune_select, stepprune_select_trajectory (traj may be
// null for the others) and stepprune_select_noalloc (use_scratch: the
// workspace is the device's fixed scratch and the error word is err_word).
sp_status select_impl(const sp_dims* dims, const void* KQV, const float* ctx, int64_t T_vis,
                      const int32_t* img_off, int32_t B, const int32_t* grp_off,
                      const int32_t* grp_img, const int32_t* grp_cap, int32_t G,
                      int32_t max_group, int32_t max_cap, const int32_t* kept_off, float b_stop,
                      int32_t g, uint32_t flags, int32_t* kept_idx, int32_t* kept_cnt,
                      int32_t* grp_cnt, float* trace, int32_t trace_steps,
                      const sp_trajectory* traj, void* ws, size_t ws_bytes,
                      const hipEvent_t* events, hipStream_t stream,
                      bool use_scratch = false, int32_t* err_word = nullptr) {
  sp_status st = check_dims(dims);
  if (st != SP_OK) return st;
  if (T_vis < 0 || B < 1 || G < 0 || max_group < 0 || max_cap < 0 || trace_steps < 0)
    return SP_EINVAL;
  if (g < 1) return SP_EINVAL;
  if (g > kGMax) return SP_EUNSUPPORTED;
  if (max_group > kMaxGroup) return SP_EUNSUPPORTED;
  if (flags & ~(uint32_t)(SP_TRACE | SP_NO_HISTORY | SP_FULL_ROLLOUT | SP_GRAM_ONLY | SP_REUSE_GRAM |
                          SP_LOGITS))
    return SP_EINVAL;
  if ((flags & SP_LOGITS) && !(flags & SP_TRACE)) return SP_EINVAL;
  if ((flags & SP_GRAM_ONLY) && (flags & SP_REUSE_GRAM)) return SP_EINVAL;
  if ((flags & SP_GRAM_ONLY) && traj) return SP_EINVAL;
  if (!KQV || !ctx || !img_off || !kept_off || !kept_cnt) return SP_EINVAL;
  if (use_scratch ? !err_word || (reinterpret_cast<uintptr_t>(err_word) & 3u) : !ws)
    return SP_EINVAL;
  if (G > 0 && (!grp_off || !grp_img || !grp_cap || !kept_idx)) return SP_EINVAL;
  if ((flags & SP_TRACE) && trace_steps > 0 && !trace) return SP_EINVAL;
  if (b_stop != b_stop) return SP_EINVAL;   // NaN
  if (traj) {
    if (!(traj->tau > 0.0f) || !(traj->beta > 0.0f && traj->beta <= 1.0f)) return SP_EINVAL;
    if (traj->pstop_steps < 0 || (traj->pstop_steps > 0 && !traj->pstop)) return SP_EINVAL;
    if ((G > 0 && !traj->kbar) || (T_vis > 0 && !traj->s)) return SP_EINVAL;
    if (g != 1) return SP_EUNSUPPORTED;
  }
  if (!aligned16(KQV) || !aligned16(ctx) || (!use_scratch && !aligned16(ws))) return SP_EINVAL;
  const SelectWs lay = select_ws_layout(G, max_group, max_cap);
  if (use_scratch) {
    if (lay.total > (size_t)STEPPRUNE_NOALLOC_SCRATCH_BYTES) return SP_EWORKSPACE;
    const sp_status sst = device_scratch(stream, &ws);
    if (sst != SP_OK) return sst;
    ws_bytes = STEPPRUNE_NOALLOC_SCRATCH_BYTES;
  }
  if (ws_bytes < lay.total) return SP_EWORKSPACE;

  char* wsb = static_cast<char*>(ws);
  SelectArgs a;
  a.dtype = dims->dtype;
  a.KQV = KQV;
  a.ctx = ctx;
  a.T_vis = T_vis;
  a.h = dims->h;
  a.img_off = img_off;
  a.B = B;
  a.grp_off = grp_off;
  a.grp_img = grp_img;
  a.grp_cap = grp_cap;
  a.G = G;
  a.max_group = max_group;
  a.max_cap = max_cap > 0 ? max_cap : 1;
  a.kept_off = kept_off;
  a.b_stop = b_stop;
  a.g = g;
  a.flags = flags;
  a.kept_idx = kept_idx;
  a.kept_cnt = kept_cnt;
  a.grp_cnt = grp_cnt;
  a.trace = trace;
  a.trace_steps = trace_steps;
  a.traj_tau = traj ? traj->tau : 0.0f;
  a.traj_beta = traj ? traj->beta : 0.0f;
  a.traj_s = traj ? traj->s : nullptr;
  a.traj_kbar = traj ? traj->kbar : nullptr;
  a.traj_pstop = traj && traj->pstop_steps > 0 ? traj->pstop : nullptr;
  a.traj_pstop_steps = traj && traj->pstop ? traj->pstop_steps : 0;
  a.gram = reinterpret_cast<float*>(wsb + lay.gram);
  a.gram_group_stride = lay.gstride;
  a.gram_ld = lay.gram_ld;
  a.grp_kept = reinterpret_cast<int32_t*>(wsb + lay.kept);
  a.grp_count = reinterpret_cast<int32_t*>(wsb + lay.count);
  a.err = use_scratch ? err_word : reinterpret_cast<int32_t*>(wsb);
  a.events = events;
  return hip_status(launch_select(a, stream));
}

}  // namespace

extern "C" {

sp_status stepprune_select(const sp_dims* dims, const void* KQV, const float* ctx, int64_t T_vis,
                           const int32_t* img_off, int32_t B, const int32_t* grp_off,
                           const int32_t* grp_img, const int32_t* grp_cap, int32_t G,
                           int32_t max_group, int32_t max_cap, const int32_t* kept_off,
                           float b_stop, int32_t g, uint32_t flags, int32_t* kept_idx,
                           int32_t* kept_cnt, int32_t* grp_cnt, float* trace, int32_t trace_steps,
                           void* ws, size_t ws_bytes, const hipEvent_t* events,
                           hipStream_t stream) {
  const TraceRange range("stepprune_select");
  return select_impl(dims, KQV, ctx, T_vis, img_off, B, grp_off, grp_img, grp_cap, G, max_group,
                     max_cap, kept_off, b_stop, g, flags, kept_idx, kept_cnt, grp_cnt, trace,
                     trace_steps, nullptr, ws, ws_bytes, events, stream);
}

sp_status stepprune_select_trajectory(const sp_dims* dims, const void* KQV, const float* ctx,
                                      int64_t T_vis, const int32_t* img_off, int32_t B,
                                      const int32_t* grp_off, const int32_t* grp_img,
                                      const int32_t* grp_cap, int32_t G, int32_t max_group,
                                      int32_t max_cap, const int32_t* kept_off, float b_stop,
                                      int32_t g, uint32_t flags, int32_t* kept_idx,
                                      int32_t* kept_cnt, int32_t* grp_cnt, float* trace,
                                      int32_t trace_steps, const sp_trajectory* traj, void* ws,
                                      size_t ws_bytes, const hipEvent_t* events,
                                      hipStream_t stream) {
  const TraceRange range("stepprune_select_trajectory");
  if (!traj) return SP_EINVAL;
  return select_impl(dims, KQV, ctx, T_vis, img_off, B, grp_off, grp_img, grp_cap, G, max_group,
                     max_cap, kept_off, b_stop, g, flags, kept_idx, kept_cnt, grp_cnt, trace,
                     trace_steps, traj, ws, ws_bytes, events, stream);
}

sp_status stepprune_select_noalloc(const sp_dims* dims, const void* KQV, const float* ctx,
                                   int64_t T_vis, const int32_t* img_off, int32_t B,
                                   const int32_t* grp_off, const int32_t* grp_img,
                                   const int32_t* grp_cap, int32_t G, int32_t max_group,
                                   int32_t max_cap, const int32_t* kept_off, float b_stop,
                                   int32_t g, uint32_t flags, int32_t* kept_idx,
                                   int32_t* kept_cnt, int32_t* grp_cnt, float* trace,
                                   int32_t trace_steps, int32_t* err,
                                   const hipEvent_t* events, hipStream_t stream) {
  const TraceRange range("stepprune_select_noalloc");
  return select_impl(dims, KQV, ctx, T_vis, img_off, B, grp_off, grp_img, grp_cap, G, max_group,
                     max_cap, kept_off, b_stop, g, flags, kept_idx, kept_cnt, grp_cnt, trace,
                     trace_steps, nullptr, nullptr, 0, events, stream, true, err);
}

sp_status stepprune_compact(const sp_dims* dims, const void* X, const int32_t* img_off,
                            const void* E_text, const int32_t* text_off, const int32_t* kept_idx,
                            const int32_t* kept_off, const int32_t* kept_cnt, int32_t B,
                            int32_t layout, int32_t rows_per_image, int64_t out_rows, void* out,
                            int32_t* seq_info, void* ws, size_t ws_bytes,
                            const hipEvent_t* events, hipStream_t stream) {
  const TraceRange range("stepprune_compact");
  sp_status st = check_dims(dims);
  if (st != SP_OK) return st;
  if (dims->d_text != dims->d) return SP_EUNSUPPORTED;
  if (B < 1 || out_rows < 0) return SP_EINVAL;
  if (layout != SP_LAYOUT_PADDED && layout != SP_LAYOUT_PACKED) return SP_EINVAL;
  if (layout == SP_LAYOUT_PADDED && (rows_per_image < 0 || (int64_t)rows_per_image * B > out_rows))
    return SP_EINVAL;
  if (!X || !img_off || !E_text || !text_off || !kept_idx || !kept_off || !kept_cnt || !out ||
      !seq_info || !ws)
    return SP_EINVAL;
  if (!aligned16(X) || !aligned16(E_text) || !aligned16(out) || !aligned16(ws)) return SP_EINVAL;
  if (ws_bytes < kWsHeaderBytes) return SP_EWORKSPACE;
  CompactArgs a;
  a.elem_bytes = elem_bytes(dims);
  a.d = dims->d;
  a.X = X;
  a.img_off = img_off;
  a.E = E_text;
  a.text_off = text_off;
  a.kept_idx = kept_idx;
  a.kept_off = kept_off;
  a.kept_cnt = kept_cnt;
  a.B = B;
  a.layout = layout;
  a.rows_per_image = rows_per_image;
  a.out_rows = out_rows;
  a.out = out;
  a.seq_info = seq_info;
  a.err = reinterpret_cast<int32_t*>(ws);
  record_event(events, 0, stream);
  hipError_t e = launch_compact(a, stream);
  record_event(events, 1, stream);
  return hip_status(e);
}

sp_status stepprune_compact_positions(const int32_t* vis_pos, int64_t T_vis, const int32_t* img_off,
                                      const int32_t* text_pos, int64_t T_txt, const int32_t* text_off,
                                      int32_t axes, const int32_t* kept_idx, const int32_t* kept_off,
                                      const int32_t* kept_cnt, int32_t B, int32_t layout,
                                      int32_t rows_per_image, int64_t out_rows, int32_t* pos,
                                      void* ws, size_t ws_bytes, hipStream_t stream) {
  const TraceRange range("stepprune_compact_positions");
  if (B < 1 || T_vis < 0 || T_txt < 0 || out_rows < 0 || axes < 1 || axes > 3) return SP_EINVAL;
  if (layout != SP_LAYOUT_PADDED && layout != SP_LAYOUT_PACKED) return SP_EINVAL;
  if (layout == SP_LAYOUT_PADDED && (rows_per_image < 0 || (int64_t)rows_per_image * B > out_rows))
    return SP_EINVAL;
  if ((T_vis > 0 && !vis_pos) || (T_txt > 0 && !text_pos) || (out_rows > 0 && !pos)) return SP_EINVAL;
  if (!img_off || !text_off || !kept_idx || !kept_off || !kept_cnt || !ws || !aligned16(ws))
    return SP_EINVAL;
  if (ws_bytes < kWsHeaderBytes) return SP_EWORKSPACE;
  PositionsArgs a;
  a.vis_pos = vis_pos;
  a.T_vis = T_vis;
  a.img_off = img_off;
  a.text_pos = text_pos;
  a.T_txt = T_txt;
  a.text_off = text_off;
  a.axes = axes;
  a.kept_idx = kept_idx;
  a.kept_off = kept_off;
  a.kept_cnt = kept_cnt;
  a.B = B;
  a.layout = layout;
  a.rows_per_image = rows_per_image;
  a.out_rows = out_rows;
  a.pos = pos;
  a.err = reinterpret_cast<int32_t*>(ws);
  return hip_status(launch_compact_positions(a, stream));
}

sp_status stepprune_cache_append(const sp_cache_dims* dims, const void* Q, int64_t ldq,
                                 const void* K, int64_t ldk, const void* V, int64_t ldv,
                                 const sp_cache_rows* rows, const sp_cache_runs* runs,
                                 const sp_cache_rotation* rot, void* Q_out, void* k_cache,
                                 void* v_cache, void* ws, size_t ws_bytes, hipStream_t stream) {
  const TraceRange range("stepprune_cache_append");
  AppendArgs a;
  sp_status st = check_cache_dims(dims, a.shape);
  if (st == SP_OK) st = check_cache_runs(runs, a.shape, true, a.runs);
  if (st == SP_OK) st = check_cache_rows(rows, a.shape, a.runs.count, true, a.rows);
  if (st != SP_OK) return st;
  const int e = a.shape.dtype == SP_F32 ? 4 : 2;
  const int64_t q_cols = (int64_t)a.shape.q_heads * a.shape.head_dim;
  const int64_t kv_cols = (int64_t)a.shape.kv_heads * a.shape.head_dim;
  if (!k_cache || !v_cache || !ws || !Q != !Q_out) return SP_EINVAL;
  if (a.rows.rows > 0 && (!K || !V)) return SP_EINVAL;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(Q_out) || !aligned16(k_cache) ||
      !aligned16(v_cache) || !aligned16(ws))
    return SP_EINVAL;
  if ((Q && (ldq < q_cols || ldq * e % 16)) || ldk < kv_cols || ldk * e % 16 || ldv < kv_cols || ldv * e % 16)
    return SP_EINVAL;
  if (Q && Q == Q_out && ldq != q_cols) return SP_EINVAL;
  a.cos_sin = nullptr;
  a.pos = nullptr;
  a.positions = a.rot_dim = a.interleaved = a.sec1 = a.sec2 = 0;
  a.axes = 1;
  if (rot) {
    if (!rot->cos_sin || !aligned16(rot->cos_sin) || rot->positions < 1) return SP_EINVAL;
    if (rot->rot_dim < 16 || rot->rot_dim % 16 || rot->rot_dim > a.shape.head_dim) return SP_EINVAL;
    if (rot->interleaved != 0 && rot->interleaved != 1) return SP_EINVAL;
    if (rot->axes < 1 || rot->axes > (rot->pos ? 3 : 1)) return SP_EINVAL;
    int64_t pairs = 0;
    for (int i = 0; i < rot->axes; ++i) {
      if (rot->section[i] < 0) return SP_EINVAL;
      pairs += rot->section[i];
    }
    if (pairs != rot->rot_dim / 2) return SP_EINVAL;
    a.cos_sin = rot->cos_sin;
    a.pos = rot->pos;
    a.positions = rot->positions;
    a.rot_dim = rot->rot_dim;
    a.interleaved = rot->interleaved;
    a.axes = rot->axes;
    a.sec1 = rot->axes > 1 ? rot->section[0] : (int)pairs;
    a.sec2 = rot->axes > 2 ? rot->section[0] + rot->section[1] : (int)pairs;
  }
  if (ws_bytes < kWsHeaderBytes) return SP_EWORKSPACE;
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldv = ldv;
  a.Q_out = Q_out;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.err = reinterpret_cast<int32_t*>(ws);
  return hip_status(launch_cache_append(a, stream));
}

size_t stepprune_cache_workspace_bytes(const sp_cache_dims* dims, const sp_cache_rows* rows,
                                       const sp_cache_runs* runs, const sp_cache_runs* prefix) {
  AttendArgs a;
  if (check_attend(dims, rows, runs, prefix, false, a) != SP_OK) return 0;
  return attend_ws_layout(a).total;
}

sp_status stepprune_cache_attend(const sp_cache_dims* dims, const void* Q, int64_t ldq,
                                 const sp_cache_rows* rows, const sp_cache_runs* runs,
                                 const sp_cache_runs* prefix, const int32_t* grp_off, float scale,
                                 uint32_t flags, const void* k_cache, const void* v_cache, void* O,
                                 float* lse, void* ws, size_t ws_bytes, const hipEvent_t* events,
                                 hipStream_t stream) {
  const TraceRange range("stepprune_cache_attend");
  AttendArgs a;
  const sp_status st = check_attend(dims, rows, runs, prefix, true, a);
  if (st != SP_OK) return st;
  if (flags & ~(uint32_t)SP_ATTEND_ALL) return SP_EINVAL;
  // -inf, a masked score, stays -inf times the scale
  const float c2 = scale * 1.4426950408889634f;
  if (!(c2 >= FLT_MIN && c2 <= FLT_MAX)) return SP_EINVAL;
  if (!k_cache || !v_cache || !ws || !prefix != !grp_off) return SP_EINVAL;
  if (a.rows.rows > 0 && (!Q || !O || Q == O)) return SP_EINVAL;
  if (!aligned16(Q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(O) || !aligned16(ws))
    return SP_EINVAL;
  if (ldq < (int64_t)a.shape.q_heads * a.shape.head_dim || ldq * (a.shape.dtype == SP_F32 ? 4 : 2) % 16)
    return SP_EINVAL;
  const AttendWs w = attend_ws_layout(a);
  if (ws_bytes < w.total) return SP_EWORKSPACE;
  char* base = static_cast<char*>(ws);
  a.grp_off = grp_off;
  a.Q = Q;
  a.ldq = ldq;
  a.c2 = c2;
  a.c2_low = (float)((double)scale * 1.4426950408889634 - (double)c2);
  a.all = (flags & SP_ATTEND_ALL) != 0;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.O = O;
  a.lse = lse;
  a.row_parts = reinterpret_cast<int2*>(base + w.row_parts);
  a.short_ml = reinterpret_cast<float*>(base + w.ml[0]);
  a.short_o = reinterpret_cast<float*>(base + w.o[0]);
  a.prefix_ml = reinterpret_cast<float*>(base + w.ml[1]);
  a.prefix_o = reinterpret_cast<float*>(base + w.o[1]);
  a.tall_ml = reinterpret_cast<float*>(base + w.ml[2]);
  a.tall_o = reinterpret_cast<float*>(base + w.o[2]);
  a.err = reinterpret_cast<int32_t*>(base);
  record_event(events, 0, stream);
  const hipError_t e = launch_cache_attend(a, stream);
  record_event(events, 1, stream);
  return hip_status(e);
}

sp_status stepprune_read_device_error(void* ws, hipStream_t stream, int32_t* code) {
  if (!ws || !code) return SP_EINVAL;
  if (hipStreamSynchronize(stream) != hipSuccess) return SP_EHIP;
  int32_t v = 0;
  if (hipMemcpy(&v, ws, sizeof(v), hipMemcpyDeviceToHost) != hipSuccess) return SP_EHIP;
  *code = v;
  if (v != 0) {
    const int32_t zero = 0;
    if (hipMemcpy(ws, &zero, sizeof(zero), hipMemcpyHostToDevice) != hipSuccess) return SP_EHIP;
    return SP_EDEVICE;
  }
  return SP_OK;
}

sp_status stepprune_encode(const sp_dims* dims, const void* X, int64_t T_vis,
                           const int32_t* img_off, int32_t B, const void* E_text,
                           const int32_t* text_off, int64_t T_txt, const void* W_p, float g_text,
                           const sp_encoder_block* blocks, int32_t max_seq, uint32_t flags,
                           void* H, void* ws, size_t ws_bytes, const hipEvent_t* events,
                           hipStream_t stream) {
  const TraceRange range("stepprune_encode");
  sp_status st = check_encode_dims(dims);
  if (st != SP_OK) return st;
  if (T_vis < 0 || T_txt < 0 || B < 1 || max_seq < 1 || !blocks) return SP_EINVAL;
  if (flags & ~(uint32_t)SP_ENC_CAUSAL) return SP_EINVAL;
  if (!img_off || !text_off || !W_p || !ws || (T_vis > 0 && (!X || !H)) || (T_txt > 0 && !E_text))
    return SP_EINVAL;
  if (!aligned16(X) || !aligned16(E_text) || !aligned16(W_p) || !aligned16(H) || !aligned16(ws))
    return SP_EINVAL;
  if (!(g_text == g_text)) return SP_EINVAL;   // NaN
  for (int k = 0; k < kEncoderBlocks; ++k) {
    const sp_encoder_block& p = blocks[k];
    const void* ptrs[] = {p.ln1_g, p.ln1_b, p.W_qkv, p.b_qkv, p.W_o, p.b_o,
                          p.ln2_g, p.ln2_b, p.W_1, p.b_1, p.W_2, p.b_2};
    for (const void* q : ptrs)
      if (!q || !aligned16(q)) return SP_EINVAL;
  }
  const EncodeWs w = encode_ws_layout(dims, T_vis, T_txt);
  if (ws_bytes < w.total) return SP_EWORKSPACE;
  char* base = static_cast<char*>(ws);
  EncodeArgs a;
  a.d = dims->d;
  a.d_text = dims->d_text;
  a.T_vis = T_vis;
  a.T_txt = T_txt;
  a.B = B;
  a.max_seq = max_seq;
  a.causal = (flags & SP_ENC_CAUSAL) != 0;
  a.g_text = g_text;
  a.X = static_cast<const uint16_t*>(X);
  a.img_off = img_off;
  a.E = static_cast<const uint16_t*>(E_text);
  a.text_off = text_off;
  a.W_p = static_cast<const uint16_t*>(W_p);
  for (int k = 0; k < kEncoderBlocks; ++k) {
    const sp_encoder_block& p = blocks[k];
    EncoderBlockArgs& q = a.blk[k];
    q.ln1_g = p.ln1_g;
    q.ln1_b = p.ln1_b;
    q.W_qkv = static_cast<const uint16_t*>(p.W_qkv);
    q.b_qkv = p.b_qkv;
    q.W_o = static_cast<const uint16_t*>(p.W_o);
    q.b_o = p.b_o;
    q.ln2_g = p.ln2_g;
    q.ln2_b = p.ln2_b;
    q.W_1 = static_cast<const uint16_t*>(p.W_1);
    q.b_1 = p.b_1;
    q.W_2 = static_cast<const uint16_t*>(p.W_2);
    q.b_2 = p.b_2;
  }
  a.H = static_cast<uint16_t*>(H);
  a.R = reinterpret_cast<float*>(base + w.R);
  a.L = reinterpret_cast<uint16_t*>(base + w.L);
  a.A = reinterpret_cast<uint16_t*>(base + w.A);
  a.QKV = reinterpret_cast<uint16_t*>(base + w.QKV);
  a.HID = reinterpret_cast<uint16_t*>(base + w.HID);
  a.err = reinterpret_cast<int32_t*>(base);
  record_event(events, 0, stream);
  const hipError_t e = launch_encode(a, stream);
  record_event(events, 1, stream);
  return hip_status(e);
}

sp_status stepprune_gate_denoise(const sp_dims* dims, const void* X, int64_t T,
                                 const float* alpha, const void* eps, const sp_denoiser* p,
                                 void* out, void* ws, size_t ws_bytes,
                                 const hipEvent_t* events, hipStream_t stream) {
  const TraceRange range("stepprune_gate_denoise");
  sp_status st = check_dims(dims);
  if (st != SP_OK) return st;
  if (dims->dtype != SP_BF16 || dims->d > 4096) return SP_EUNSUPPORTED;
  if (T < 0 || !p || !out || !ws) return SP_EINVAL;
  if (T > 0 && (!X || !alpha || !eps)) return SP_EINVAL;
  if (!p->ln1_g || !p->ln1_b || !p->W_v || !p->b_v || !p->W_o || !p->b_o || !p->ln2_g ||
      !p->ln2_b || !p->W_1 || !p->b_1 || !p->W_2 || !p->b_2)
    return SP_EINVAL;
  if (!aligned16(X) || !aligned16(eps) || !aligned16(out) || !aligned16(ws) ||
      !aligned16(p->W_v) || !aligned16(p->W_o) || !aligned16(p->W_1) || !aligned16(p->W_2) ||
      !aligned16(p->ln1_g) || !aligned16(p->ln1_b) || !aligned16(p->b_v) || !aligned16(p->b_o) ||
      !aligned16(p->ln2_g) || !aligned16(p->ln2_b) || !aligned16(p->b_1) || !aligned16(p->b_2))
    return SP_EINVAL;
  if (out == X || out == eps) return SP_EINVAL;
  const GateWs w = gate_ws_layout(dims, T);
  if (ws_bytes < w.total) return SP_EWORKSPACE;
  char* base = static_cast<char*>(ws);
  DenoiseArgs a;
  a.T = T;
  a.d = dims->d;
  a.X = static_cast<const uint16_t*>(X);
  a.alpha = alpha;
  a.eps = static_cast<const uint16_t*>(eps);
  a.ln1_g = p->ln1_g;
  a.ln1_b = p->ln1_b;
  a.W_v = static_cast<const uint16_t*>(p->W_v);
  a.b_v = p->b_v;
  a.W_o = static_cast<const uint16_t*>(p->W_o);
  a.b_o = p->b_o;
  a.ln2_g = p->ln2_g;
  a.ln2_b = p->ln2_b;
  a.W_1 = static_cast<const uint16_t*>(p->W_1);
  a.b_1 = p->b_1;
  a.W_2 = static_cast<const uint16_t*>(p->W_2);
  a.b_2 = p->b_2;
  a.out = static_cast<uint16_t*>(out);
  a.xt = reinterpret_cast<float*>(base + w.xt);
  a.buf_p = reinterpret_cast<uint16_t*>(base + w.p);
  a.buf_q = reinterpret_cast<uint16_t*>(base + w.q);
  a.hid = reinterpret_cast<uint16_t*>(base + w.hid);
  record_event(events, 0, stream);
  const hipError_t e = launch_gate_denoise(a, stream);
  record_event(events, 1, stream);
  return hip_status(e);
}

}  // extern "C"
