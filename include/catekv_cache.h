/*
 * catekv_cache.h -- caches held in 8 bits, attention that adds its weights up
 * per cached row, and eviction of the rows that gathered least (MI355X, gfx950).
 *
 *   catekv_q8_quantize          a cache's rows into 8 bits with a scale per block of rows
 *   catekv_q8_dequantize        and back
 *   catekv_q8_append            the newest token of each step into every 8-bit view
 *   catekv_q8_decode_attn       one decode step over 8-bit views, its weights added up on request
 *   catekv_decode_attn_weights  one decode step over catekv_decode_attn's views, its weights added up
 *   catekv_evict_kv             drops the chunks of rows that gathered least weight
 *   catekv_q8_evict             the same for 8-bit views
 *
 * The conventions of catekv.h hold: caller-owned device pointers, checks before
 * any work is enqueued, caller-owned workspaces, d == 128, asynchronous work on
 * `stream`.  Every address below lies on a 16-byte border, except the scales,
 * the arrays of accumulated weights, lse and the tables, which lie on a border of
 * their own type (q, out, k_new and v_new are checked: INVALID_ARG).  No two views
 * that a call writes share memory, nor do two arrays of weights.
 *
 * An 8-bit view of L rows in blocks of `block` rows (32 or 64; K and V alike):
 *   rows [0, nb block), nb = L / block rounded down, as codes [row][d] with one
 *     fp32 scale per block: row t is code[t] * scale[t / block];
 *   rows [nb block, L) in the cache's own dtype in the tail [block][d], row
 *     t - nb block.
 * A block's scale and codes come from its rows x alone, once, when it is full:
 *   CATEKV_I8    scale = fp32(m * fp32(1/127)), m = max |x|;
 *                code = x / scale rounded to the nearest integer, ties to even
 *   CATEKV_E4M3  (OCP e4m3fn) scale = the least power of two with m <= 448 scale;
 *                code = x / scale rounded to the nearest e4m3 value, ties to even
 *   m < 2^-100 gives scale 0 and codes 0; a value that is not finite gives a NaN
 *   scale and codes 0, so that every row of the block reads as NaN.
 */
#ifndef CATEKV_CACHE_H
#define CATEKV_CACHE_H

#include "catekv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CATEKV_I8 = 0, CATEKV_E4M3 = 1 } catekv_q8_format;

/* One (sequence, KV head) view.  For a capacity of C rows: k, v hold
 * C / block * block rows (rounded down) of 128 bytes, k_scale, v_scale as many
 * floats as those are blocks, k_tail, v_tail `block` rows of the cache's dtype. */
typedef struct catekv_q8_view {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  void* k_tail;
  void* v_tail;
} catekv_q8_view;

/* Brings the first lens[bh] rows of every view kv[bh] into views[bh].
 * kv     [n_views] device, rows in dtype
 * lens   [n_views] int64, device; a view with lens outside [0, max_rows] is left
 *        alone
 * views  [n_views] device
 * max_rows  a bound on lens (sizes the launch)
 * Errors: INVALID_ARG for null pointers, n_views < 1, max_rows < 1 or a block
 * other than 32 or 64; UNSUPPORTED for an unknown format or dtype, d != 128,
 * max_rows above 2^31 - 1 or sizes that would take a launch of 2^32 threads (64
 * for each block and each tail, in fours: 2^26 of all views together). */
int catekv_q8_quantize(int format, int dtype, int block, const catekv_kv_ptrs* kv, const int64_t* lens,
                       const catekv_q8_view* views, int n_views, int64_t max_rows, int d, void* stream);

/* The rows of every view in dtype: code * scale in fp32, rounded to dtype, and
 * the tail's rows as they are.  Writes the first lens[bh] rows of kv_out[bh].
 * Errors: as above. */
int catekv_q8_dequantize(int format, int dtype, int block, const catekv_q8_view* views, const int64_t* lens,
                         const catekv_kv_ptrs* kv_out, int n_views, int64_t max_rows, int d, void* stream);

/* Appends the newest token to every view (catekv_append_kv on 8-bit views): its
 * K and V rows go into the tail, lens[bh] grows by one, and a tail that is full
 * then becomes the view's next block.  A view with lens[bh] outside
 * [0, capacity[bh]) is left unchanged and sets *overflow = 1 when overflow is
 * not NULL.  The result is that of catekv_q8_quantize on the longer rows.
 * k_new, v_new  [batch][hkv][d] (dtype)
 * Errors: INVALID_ARG for null pointers, batch < 1, hkv < 1, batch * hkv of 2^23
 * or more or a bad block; UNSUPPORTED for an unknown format or dtype or d != 128. */
int catekv_q8_append(int format, int dtype, int block, const catekv_q8_view* views, const int64_t* capacity,
                     int64_t* lens, const void* k_new, const void* v_new, int batch, int hkv, int d,
                     int32_t* overflow, void* stream);

/* Workspace bytes of a decode step of this plan that adds its weights up; 0
 * for a plan that catekv_decode_plan has not filled. */
size_t catekv_weights_workspace(const catekv_decode_plan_t* plan);

/* One decode step over 8-bit views: catekv_decode_attn with K and V read as
 * their codes times their scales.  dtype is that of q and of the tails.  With
 * acc, the step's softmax weights are added up per row,
 *   acc[bh][t] = decay * acc[bh][t] + (1/G) sum_g softmax_g(t),  t < L,
 * over the G query heads of the view's group; rows from L on are not touched.  A head
 * whose rows all score -inf (out 0, lse -inf) adds nothing; one whose output is NaN
 * adds NaN.
 * views   [batch][hkv] device
 * lens    [batch][hkv] int64, device; L = min(lens, planned max_len).  The tail
 *         starts at lens / block * block whatever the plan says
 * out, lse  as in catekv_decode_attn
 * acc     [batch][hkv] device pointers to fp32 arrays of at least L values, in
 *         device memory, or NULL for no weights
 * decay   in [0, 1]; 1 sums all steps, 0 leaves this step's weights alone
 *         whatever acc held (ignored without acc)
 * ws      the plan's workspace
 * wws     catekv_weights_workspace() bytes (ignored without acc); calls that
 *         overlap in time must not share it
 * Errors: those of catekv_decode_attn; INVALID_ARG for a bad block or decay;
 * UNSUPPORTED for an unknown format or a plan that would take a launch of 2^32
 * threads (512 for each of its shares; 512 for each query row, batch * hq, where it
 * splits a view, and with acc for each share besides); WORKSPACE for a wws too
 * small. */
int catekv_q8_decode_attn(int format, int dtype, int block, const catekv_decode_plan_t* plan, const void* q,
                          const catekv_q8_view* views, const int64_t* lens, int batch, int hq, int hkv, int d,
                          float scale, float* out, float* lse, float* const* acc, float decay, void* ws,
                          size_t ws_bytes, void* wws, size_t wws_bytes, void* stream);

/* catekv_decode_attn over the same views, with the weights added up as above
 * (acc must be given).  Errors: as above. */
int catekv_decode_attn_weights(int dtype, const catekv_decode_plan_t* plan, const void* q,
                               const catekv_kv_ptrs* kv, const int64_t* lens, int batch, int hq, int hkv, int d,
                               float scale, float* out, float* lse, float* const* acc, float decay, void* ws,
                               size_t ws_bytes, void* wws, size_t wws_bytes, void* stream);

/* Workspace bytes of the eviction calls; 0 for sizes they refuse.  Beside the
 * bounds below these are sizes that would take a launch of 2^32 threads: none with
 * max_rows up to 16384 or n_views * max_rows up to 2^32, all from 2^36 on. */
size_t catekv_evict_workspace(int n_views, int64_t max_rows, int cs);

/* Drops rows of every view by accumulated weight, in place.  Of the L = lens[bh]
 * rows, the first nc = max(L - recent, 0) / cs (rounded down) chunks of cs rows
 * compete; the rest is always kept.  A chunk's weight is the largest acc of its
 * rows (NaN counts as the largest value).  The k = min(budget[bh], nc) chunks of
 * largest weight stay, ties to the lower chunk:
 *   - kept chunks below k stay where they are; the kept chunks from k on, in
 *     ascending order, take the places of the dropped chunks below k, in
 *     ascending order (a softmax does not ask for an order, and so only as many
 *     rows move as have to);
 *   - the rows [nc cs, L) follow at k cs, in their order;
 *   - acc moves with its rows, lens[bh] = L - (nc - k) cs, acc is 0 from there
 *     to L, and the rows of K and V from there on are left as they were.
 * A view with budget[bh] < 0 or nc <= budget[bh], or with lens outside
 * [0, max_rows], is left alone.
 * Afterwards lens[bh] <= budget[bh] cs + recent + cs - 1 (where budget[bh] >= 0 and
 * lens was in range), a bound for the plan and max_rows of the steps that follow.
 * kv      [n_views] device, rows in dtype
 * lens    [n_views] int64, device, read and written
 * acc     [n_views] device pointers to fp32 arrays of at least lens values
 * budget  [n_views] int32, device: chunks kept among those that compete
 * max_rows  a bound on lens (sizes the launches and the workspace), at most 2^26
 * cs in [1, 2^20], recent >= 0, n_views at most 2^16
 * Errors: INVALID_ARG for null pointers or bad sizes; UNSUPPORTED for an unknown
 * dtype, d != 128 or sizes above these bounds or for which
 * catekv_evict_workspace() is 0; WORKSPACE for a ws too small. */
int catekv_evict_kv(int dtype, const catekv_kv_ptrs* kv, int64_t* lens, float* const* acc, const int32_t* budget,
                    int n_views, int64_t max_rows, int cs, int recent, int d, void* ws, size_t ws_bytes,
                    void* stream);

/* The same for 8-bit views; cs is a multiple of block, so that whole blocks move
 * with their scales, and the tails stay.  Errors: as above, and INVALID_ARG for
 * a bad block or another cs. */
int catekv_q8_evict(int block, const catekv_q8_view* views, int64_t* lens, float* const* acc,
                    const int32_t* budget, int n_views, int64_t max_rows, int cs, int recent, int d, void* ws,
                    size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CATEKV_CACHE_H */
