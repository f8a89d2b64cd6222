// Host side of include/catekv_cache.h: argument checks and launches.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "cache.h"

namespace {

using namespace catekv;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return host_error(code, buf);
}

int hip_fail(hipError_t e, const char* what) { return fail(CATEKV_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

int check_types(int format, int dtype) {
  if (format != CATEKV_I8 && format != CATEKV_E4M3) return fail(CATEKV_ERR_UNSUPPORTED, "8-bit format %d unsupported", format);
  if (dtype != CATEKV_F32 && dtype != CATEKV_BF16) return fail(CATEKV_ERR_UNSUPPORTED, "dtype %d unsupported", dtype);
  return CATEKV_OK;
}

int check_block(int block) {
  if (block != 32 && block != 64) return fail(CATEKV_ERR_INVALID_ARG, "block of %d rows (32 or 64)", block);
  return CATEKV_OK;
}

int check_rows(int n_views, int64_t max_rows, int d) {
  if (n_views < 1) return fail(CATEKV_ERR_INVALID_ARG, "n_views=%d must be >= 1", n_views);
  if (max_rows < 1) return fail(CATEKV_ERR_INVALID_ARG, "max_rows=%lld must be >= 1", (long long)max_rows);
  if (max_rows > INT32_MAX) return fail(CATEKV_ERR_UNSUPPORTED, "max_rows=%lld above 2^31 - 1", (long long)max_rows);
  if (d != kD) return fail(CATEKV_ERR_UNSUPPORTED, "head dimension %d unsupported (only %d)", d, kD);
  return CATEKV_OK;
}

// Addresses that the kernels read or write 16 bytes at a time.
int check_aligned(const void* p, const char* name) {
  if (reinterpret_cast<uintptr_t>(p) % 16) return fail(CATEKV_ERR_INVALID_ARG, "%s is not on a 16-byte border", name);
  return CATEKV_OK;
}

// The checks of both conversions, and their launch sizes.
int check_convert(int format, int dtype, int block, const void* kv, const void* lens, const void* views, int n_views,
                  int64_t max_rows, int d) {
  int rc = check_types(format, dtype);
  if (!rc && (!kv || !lens || !views)) rc = fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  if (!rc) rc = check_block(block);
  if (!rc) rc = check_rows(n_views, max_rows, d);
  if (!rc && !launch_fits(q8_groups(max_rows, block) * n_views, kQ8Threads))
    rc = fail(CATEKV_ERR_UNSUPPORTED, "n_views=%d of max_rows=%lld: too many blocks for one launch", n_views, (long long)max_rows);
  return rc;
}

// Fills what both attention calls share, after their checks.
int attend_args(const catekv_decode_plan_t* plan, const void* q, const void* views, const int64_t* lens, int batch,
                int hq, int hkv, int d, float scale, float* out, float* lse, float* const* acc, float decay, void* ws,
                size_t ws_bytes, void* wws, size_t wws_bytes, AttendArgs& a) {
  if (!host_plan_valid(plan)) return fail(CATEKV_ERR_INVALID_ARG, "plan missing or not built by catekv_decode_plan");
  if (!q || !views || !lens || !out) return fail(CATEKV_ERR_INVALID_ARG, "null tensor pointer");
  int rc = check_aligned(q, "q");
  if (!rc) rc = check_aligned(out, "out");
  if (!rc) rc = host_check_heads(hq, hkv, d);
  if (rc) return rc;
  if (plan->batch != batch || plan->hq != hq || plan->hkv != hkv)
    return fail(CATEKV_ERR_INVALID_ARG, "shapes (batch=%d hq=%d hkv=%d) differ from the plan (%d, %d, %d)", batch, hq,
                hkv, plan->batch, plan->hq, plan->hkv);
  if (!(scale > 0.f) || !std::isfinite(scale))
    return fail(CATEKV_ERR_INVALID_ARG, "scale=%g must be positive and finite", (double)scale);
  const int64_t joins = plan->n_multi > 0 ? (int64_t)batch * hq : 0;   // a workgroup per view and head of its group
  if (!launch_fits(plan->n_workers, kAttendThreads) || !launch_fits(joins + (acc ? plan->n_workers : 0), kAttendThreads))
    return fail(CATEKV_ERR_UNSUPPORTED, "batch=%d hq=%d, a plan of %d shares: too many workgroups for one launch", batch, hq,
                plan->n_workers);
  rc = host_check_ws(ws, ws_bytes, plan->ws_bytes);
  if (rc) return rc;
  if (acc) {
    if (!(decay >= 0.f && decay <= 1.f)) return fail(CATEKV_ERR_INVALID_ARG, "decay=%g outside [0, 1]", (double)decay);
    rc = host_check_ws(wws, wws_bytes, catekv_weights_workspace(plan));
    if (rc) return rc;
  }
  const DecodeArgs p = host_plan_args(plan, ws);
  a.q = q;
  a.views = views;
  a.lens = lens;
  a.items = p.items;
  a.worker_seg = p.worker_seg;
  a.v2items = p.v2items;
  a.infos = p.views;
  a.slots = p.slots;
  a.scores = reinterpret_cast<float*>(wws);
  a.score_rows = attend_score_rows(plan);
  a.acc = acc;
  a.decay = decay;
  a.n_workers = p.n_workers;
  a.n_views = p.n_views;
  a.n_multi = p.n_multi;
  a.hkv = hkv;
  a.variant = p.variant;
  a.scale = scale;
  a.out = out;
  a.lse = lse;
  return CATEKV_OK;
}

int check_evict(const void* views, const void* lens, const void* acc, const void* budget, int n_views, int64_t max_rows,
                int cs, int recent, int d, const void* ws, size_t ws_bytes) {
  if (!views || !lens || !acc || !budget) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  int rc = check_rows(n_views, max_rows, d);
  if (rc) return rc;
  if (cs < 1) return fail(CATEKV_ERR_INVALID_ARG, "chunk size %d must be >= 1", cs);
  if (!evict_fits(n_views, max_rows, cs))
    return fail(CATEKV_ERR_UNSUPPORTED, "n_views=%d, max_rows=%lld, cs=%d: too large for one eviction", n_views,
                (long long)max_rows, cs);
  if (recent < 0) return fail(CATEKV_ERR_INVALID_ARG, "recent=%d must be >= 0", recent);
  return host_check_ws(ws, ws_bytes, evict_workspace_bytes(n_views, max_rows, cs));
}

}  // namespace

namespace catekv {

// A worker's share is at most ceil(U / W) units of kDecodeQuantum rows, U the
// units of all views; a view wastes less than one unit.
int64_t attend_score_rows(const catekv_decode_plan_t* plan) {
  const int64_t views = (int64_t)plan->batch * plan->hkv, W = plan->n_workers;
  const int64_t units = (plan->max_len_total + views * (kDecodeQuantum - 1)) / kDecodeQuantum;
  return (units + W - 1) / W * kDecodeQuantum;
}

}  // namespace catekv

extern "C" {

int catekv_q8_quantize(int format, int dtype, int block, const catekv_kv_ptrs* kv, const int64_t* lens,
                       const catekv_q8_view* views, int n_views, int64_t max_rows, int d, void* stream) {
  const int rc = check_convert(format, dtype, block, kv, lens, views, n_views, max_rows, d);
  if (rc) return rc;
  Q8Args a{};
  a.block = block;
  a.kv = kv;
  a.lens = lens;
  a.views = views;
  a.n_views = n_views;
  a.max_rows = max_rows;
  const hipError_t e = launch_q8_quantize(format, dtype, a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "q8_quantize launch");
}

int catekv_q8_dequantize(int format, int dtype, int block, const catekv_q8_view* views, const int64_t* lens,
                         const catekv_kv_ptrs* kv_out, int n_views, int64_t max_rows, int d, void* stream) {
  const int rc = check_convert(format, dtype, block, kv_out, lens, views, n_views, max_rows, d);
  if (rc) return rc;
  Q8Args a{};
  a.block = block;
  a.kv = kv_out;
  a.lens = lens;
  a.views = views;
  a.n_views = n_views;
  a.max_rows = max_rows;
  const hipError_t e = launch_q8_dequantize(format, dtype, a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "q8_dequantize launch");
}

int catekv_q8_append(int format, int dtype, int block, const catekv_q8_view* views, const int64_t* capacity,
                     int64_t* lens, const void* k_new, const void* v_new, int batch, int hkv, int d,
                     int32_t* overflow, void* stream) {
  int rc = check_types(format, dtype);
  if (rc) return rc;
  if (!views || !capacity || !lens || !k_new || !v_new) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  rc = check_block(block);
  if (rc) return rc;
  if (batch < 1 || hkv < 1) return fail(CATEKV_ERR_INVALID_ARG, "batch=%d hkv=%d must be >= 1", batch, hkv);
  if (d != kD) return fail(CATEKV_ERR_UNSUPPORTED, "head dimension %d unsupported (only %d)", d, kD);
  if (!launch_fits((int64_t)batch * hkv, kAppendThreads)) return fail(CATEKV_ERR_INVALID_ARG, "batch * hkv too large");
  rc = check_aligned(k_new, "k_new");
  if (!rc) rc = check_aligned(v_new, "v_new");
  if (rc) return rc;
  Q8Args a{};
  a.block = block;
  a.views = views;
  a.capacity = capacity;
  a.lens_rw = lens;
  a.k_new = k_new;
  a.v_new = v_new;
  a.overflow = overflow;
  a.n_views = batch * hkv;
  const hipError_t e = launch_q8_append(format, dtype, a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "q8_append launch");
}

size_t catekv_weights_workspace(const catekv_decode_plan_t* plan) {
  if (!host_plan_valid(plan)) return 0;
  return (size_t)attend_score_rows(plan) * (size_t)plan->n_workers * (size_t)(plan->hq / plan->hkv) * sizeof(float);
}

int catekv_q8_decode_attn(int format, int dtype, int block, const catekv_decode_plan_t* plan, const void* q,
                          const catekv_q8_view* views, const int64_t* lens, int batch, int hq, int hkv, int d,
                          float scale, float* out, float* lse, float* const* acc, float decay, void* ws,
                          size_t ws_bytes, void* wws, size_t wws_bytes, void* stream) {
  int rc = check_types(format, dtype);
  if (!rc) rc = check_block(block);
  if (rc) return rc;
  AttendArgs a{};
  rc = attend_args(plan, q, views, lens, batch, hq, hkv, d, scale, out, lse, acc, decay, ws, ws_bytes, wws, wws_bytes, a);
  if (rc) return rc;
  a.block = block;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const hipError_t e = format == CATEKV_I8 ? launch_attend_i8(dtype, hq / hkv, a, s) : launch_attend_e4m3(dtype, hq / hkv, a, s);
  return e == hipSuccess ? host_ok() : hip_fail(e, "q8_decode_attn launch");
}

int catekv_decode_attn_weights(int dtype, const catekv_decode_plan_t* plan, const void* q, const catekv_kv_ptrs* kv,
                               const int64_t* lens, int batch, int hq, int hkv, int d, float scale, float* out,
                               float* lse, float* const* acc, float decay, void* ws, size_t ws_bytes, void* wws,
                               size_t wws_bytes, void* stream) {
  int rc = check_types(CATEKV_I8, dtype);
  if (rc) return rc;
  if (!acc) return fail(CATEKV_ERR_INVALID_ARG, "acc is null (catekv_decode_attn adds no weights up)");
  AttendArgs a{};
  rc = attend_args(plan, q, kv, lens, batch, hq, hkv, d, scale, out, lse, acc, decay, ws, ws_bytes, wws, wws_bytes, a);
  if (rc) return rc;
  const hipError_t e = launch_attend_dense(dtype, hq / hkv, a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "decode_attn_weights launch");
}

size_t catekv_evict_workspace(int n_views, int64_t max_rows, int cs) {
  if (n_views < 1 || max_rows < 1 || cs < 1 || !evict_fits(n_views, max_rows, cs)) return 0;
  return evict_workspace_bytes(n_views, max_rows, cs);
}

int catekv_evict_kv(int dtype, const catekv_kv_ptrs* kv, int64_t* lens, float* const* acc, const int32_t* budget,
                    int n_views, int64_t max_rows, int cs, int recent, int d, void* ws, size_t ws_bytes,
                    void* stream) {
  int rc = check_types(CATEKV_I8, dtype);
  if (!rc) rc = check_evict(kv, lens, acc, budget, n_views, max_rows, cs, recent, d, ws, ws_bytes);
  if (rc) return rc;
  EvictArgs a{};
  a.kv = kv;
  a.lens = lens;
  a.acc = acc;
  a.budget = budget;
  a.n_views = n_views;
  a.row_bytes = kD * (dtype == CATEKV_BF16 ? 2 : 4);
  a.cs = cs;
  a.recent = recent;
  a.max_rows = max_rows;
  a.ws = ws;
  const hipError_t e = launch_evict(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "evict_kv launch");
}

int catekv_q8_evict(int block, const catekv_q8_view* views, int64_t* lens, float* const* acc, const int32_t* budget,
                    int n_views, int64_t max_rows, int cs, int recent, int d, void* ws, size_t ws_bytes,
                    void* stream) {
  int rc = check_block(block);
  if (!rc) rc = check_evict(views, lens, acc, budget, n_views, max_rows, cs, recent, d, ws, ws_bytes);
  if (rc) return rc;
  if (cs % block) return fail(CATEKV_ERR_INVALID_ARG, "chunk size %d is not a multiple of the block's %d rows", cs, block);
  EvictArgs a{};
  a.q8 = views;
  a.lens = lens;
  a.acc = acc;
  a.budget = budget;
  a.n_views = n_views;
  a.row_bytes = kD;
  a.block = block;
  a.cs = cs;
  a.recent = recent;
  a.max_rows = max_rows;
  a.ws = ws;
  const hipError_t e = launch_evict(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "q8_evict launch");
}

}  // extern "C"
