// Internal interface of the 8-bit caches, of attention that adds its weights
// up, and of eviction: what cache_api.cpp passes to the kernels.
#pragma once

#include "catekv_cache.h"
#include "internal.h"

namespace catekv {

// ---- host side, shared with api.cpp ----------------------------------------
int host_error(int code, const char* msg);         // sets catekv_last_error()
int host_ok();
int host_check_heads(int hq, int hkv, int d);
int host_check_ws(const void* ws, size_t ws_bytes, size_t need);
bool host_plan_valid(const catekv_decode_plan_t* plan);
// The plan's tables in its workspace; the other fields are the caller's.
DecodeArgs host_plan_args(const catekv_decode_plan_t* plan, void* ws);

// HIP takes launches of less than 2^32 threads.
inline bool launch_fits(int64_t workgroups, int threads) { return workgroups * threads < (int64_t)1 << 32; }

// ---- 8-bit caches ------------------------------------------------------------
struct Q8Args {
  int block;                       // rows of a block: 32 or 64
  const catekv_q8_view* views;
  const catekv_kv_ptrs* kv;        // rows in the cache's own type
  const int64_t* lens;
  int64_t* lens_rw;                // append
  const int64_t* capacity;
  const void* k_new;
  const void* v_new;
  int32_t* overflow;
  int n_views;
  int64_t max_rows;
};
// Workgroups per view (K or V) of the first two, of kQ8Threads threads.
constexpr int kQ8Threads = 256;
constexpr int kAppendThreads = 512;   // of the append's one workgroup per view
int64_t q8_groups(int64_t max_rows, int block);
hipError_t launch_q8_quantize(int fmt, int dtype, const Q8Args& a, hipStream_t stream);
hipError_t launch_q8_dequantize(int fmt, int dtype, const Q8Args& a, hipStream_t stream);
hipError_t launch_q8_append(int fmt, int dtype, const Q8Args& a, hipStream_t stream);

// ---- attention -----------------------------------------------------------------
constexpr int kAttendThreads = 512;   // of a workgroup of either kernel
struct AttendArgs {
  const void* q;
  const void* views;               // catekv_kv_ptrs or catekv_q8_view, one per view
  const int64_t* lens;
  const DecodeItem* items;
  const int32_t* worker_seg;
  const V2Item* v2items;
  const ViewInfo* infos;
  float* slots;
  float* scores;                   // [worker][segments: head-major planes], with acc
  int64_t score_rows;              // rows of scores per worker
  float* const* acc;               // one array per view; null without weights
  float decay;
  int n_workers, n_views, n_multi, hkv, variant, block;
  bool staged;                     // the stream kernel keeps its scores in LDS until its end
  float scale;
  float* out;
  float* lse;
};
// Rows of scores that a worker of this plan holds at most.
int64_t attend_score_rows(const catekv_decode_plan_t* plan);
hipError_t launch_attend_dense(int dtype, int G, const AttendArgs& a, hipStream_t stream);
hipError_t launch_attend_i8(int dtype, int G, const AttendArgs& a, hipStream_t stream);
hipError_t launch_attend_e4m3(int dtype, int G, const AttendArgs& a, hipStream_t stream);

// ---- eviction ----------------------------------------------------------------
struct EvictArgs {
  const catekv_kv_ptrs* kv;        // rows of row_bytes, or
  const catekv_q8_view* q8;        // codes in blocks of `block`
  int64_t* lens;
  float* const* acc;
  const int32_t* budget;
  int n_views, row_bytes, block, cs, recent;
  int64_t max_rows;
  void* ws;
};
// Sizes whose element numbers fit 32 bits and whose launches HIP takes.
bool evict_fits(int n_views, int64_t max_rows, int cs);
size_t evict_workspace_bytes(int n_views, int64_t max_rows, int cs);
hipError_t launch_evict(const EvictArgs& a, hipStream_t stream);

}  // namespace catekv
