/*
 * catekv_paged.h -- caches held in pages of one pool, attention of several new
 * tokens per sequence over them, and what a serving program does with pages
 * (MI355X, gfx950).
 *
 *   catekv_paged_init      an empty cache: every page free
 *   catekv_paged_plan      work list of a batch's new tokens (host side, once per batch)
 *   catekv_paged_append    the new tokens' rows behind every view's, pages taken as needed
 *   catekv_paged_attn      attention of the new tokens: single tokens, chunks of prompts, or both
 *   catekv_paged_fork      slots that share another slot's pages until they write
 *   catekv_paged_drop      the last rows of every view of a slot off; all of them to free a slot
 *   catekv_paged_compact   critical chunks and the last rows of a view into pages of its own
 *   catekv_paged_gather    a slot's rows as dense views, for the calls of catekv.h that read those
 *
 * The conventions of catekv.h hold: caller-owned device pointers, checks before
 * any work is enqueued, caller-owned workspaces on 256-byte borders, asynchronous
 * work on `stream`, d == 128, hq / hkv in {1, 2, 4, 8}.  Calls on one cache that
 * change it, and those that read it, run one after the other (one stream, or
 * streams ordered by events).
 *
 * A cache has n_slots slots (sequences) of hkv views, view = slot * hkv + head.
 * Row t of a view lies in page table[view][t / page] at row t % page.  Entries
 * behind a view's last page are -1.  refs counts the views that hold a page; a
 * page is free if that is 0, and its bit in free_bits is then set (bit p % 64 of
 * word p / 64; bits behind n_pages are 0).  Calls that need pages take the free
 * pages of lowest number, in the order they state, so that a cache's tables
 * follow from its calls alone.  The state is device memory and may be read, saved
 * and restored as a whole; entries and lengths out of range are never followed
 * out of the arrays (such a view counts as empty, such an entry as page 0).
 */
#ifndef CATEKV_PAGED_H
#define CATEKV_PAGED_H

#include "catekv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Handle of a cache, filled by the caller.  k, v: 16-byte borders. */
typedef struct catekv_paged_cache {
  void* k;                /* [n_pages][page][d] (dtype) */
  void* v;
  int32_t* table;         /* [n_slots * hkv][max_pages] */
  int64_t* lens;          /* [n_slots * hkv] */
  int32_t* refs;          /* [n_pages] */
  uint64_t* free_bits;    /* [ceil(n_pages / 64)] */
  int32_t dtype;          /* CATEKV_F32 or CATEKV_BF16 */
  int32_t page;           /* rows of a page: 16, 32, 64, 128 or 256 */
  int32_t n_pages;
  int32_t n_slots, hkv;   /* at most 2^20 views */
  int32_t max_pages;      /* per view, at most 2^26 rows */
} catekv_paged_cache;

/* Host-side descriptor of a plan.  Treat as opaque. */
typedef struct catekv_paged_plan_t {
  uint64_t magic;
  int32_t n_seqs, n_tokens, hq, hkv, n_slots, page, dtype;
  int32_t n_tile, n_workers, n_joins, tile_joins, tile_parts, few_parts, reserved;
  uint64_t seqs_off, toks_off, tiles_off, tile_workers_off, segs_off, workers_off, joins_off, views_off, takes_off, slots_off, ws_bytes;
} catekv_paged_plan_t;

/* An empty cache: lens 0, table -1, refs 0, every page free.  k and v stay as
 * they are.
 * Errors of every call on a cache: INVALID_ARG for a null pointer in it, a page
 * size not listed, misaligned k or v, or sizes below 1; UNSUPPORTED for an unknown
 * dtype or sizes above the bounds stated. */
int catekv_paged_init(const catekv_paged_cache* cache, void* stream);

/* Workspace bytes of a plan with these arguments; 0 for arguments that
 * catekv_paged_plan refuses. */
size_t catekv_paged_workspace(const catekv_paged_cache* cache, const int32_t* slots_host, const int32_t* new_host,
                              const int64_t* max_rows_host, int n_seqs, int hq);

/* The work list of a batch: sequence i has new_host[i] >= 0 new tokens and lies in
 * slot slots_host[i] (all distinct).  Tokens are numbered through: sequence 0's
 * first.  max_rows_host [n_seqs][hkv]: upper bounds of the views' rows with the
 * new tokens in them; attention never looks past them, and its work is divided by
 * them.  Blocks until the upload has completed.  The plan and ws serve every later
 * append and attention of batches of this shape on caches of this geometry (other
 * layers, later steps); calls sharing a ws must not overlap in time.
 * Errors: INVALID_ARG for null pointers, n_seqs < 1, a slot out of range or listed
 * twice, new tokens below 0, max_rows below 0; UNSUPPORTED for unsupported heads,
 * more than 2^26 tokens, max_rows above 2^26 or work that would take a launch of
 * 2^32 threads; WORKSPACE if ws is too small; HIP on upload failure or when host
 * memory runs out. */
int catekv_paged_plan(const catekv_paged_cache* cache, const int32_t* slots_host, const int32_t* new_host,
                      const int64_t* max_rows_host, int n_seqs, int hq, catekv_paged_plan_t* plan, void* ws,
                      size_t ws_bytes, void* stream);

/* Appends the new tokens: view h of sequence i gets the rows k_new[token][h] of its
 * m = new_host[i] tokens behind its L = lens rows, lens becomes L + m.  A last page
 * that is partly filled and that other views hold too (refs > 1 before the call) is
 * copied first, its first L % page rows, and released.  Pages are taken lowest free
 * first, in the order of sequence, head, row (the copy before the new pages); pages
 * released by this call are free after it.
 * A sequence is appended whole or not at all.  One with a view that would exceed
 * max_pages, or whose lens is out of range, is left unchanged; so are the first
 * sequence, in order, that does not find its pages and all later ones that need
 * any.  Then *overflow = 1 when overflow is not NULL (never cleared here).
 * k_new, v_new  head h of token t at t * tok_stride + h * head_stride elements
 *               (multiples of 16 bytes; [token][hkv][d]: hkv d and d)
 * overflow      int32, device, or NULL
 * Errors: INVALID_ARG for null pointers, misaligned or negative strides, or a cache
 * that is not of the plan's geometry; WORKSPACE. */
int catekv_paged_append(const catekv_paged_cache* cache, const catekv_paged_plan_t* plan, const void* k_new,
                        const void* v_new, int64_t tok_stride, int64_t head_stride, int32_t* overflow, void* ws,
                        size_t ws_bytes, void* stream);

/* Attention of the new tokens, whose rows are the last of their views (after
 * catekv_paged_append).  For token j < m of sequence i and query head g of KV head
 * h, with L = min(lens, planned max_rows) of the view:
 *   see = L - m + j + 1;  s_t = scale q . K[t];  t < see
 *   out = sum_t softmax(s)_t V[t],  lse = log sum_t exp(s_t)
 * and out = 0, lse = -inf where see <= 0 or every score is -inf.  What lies in rows
 * that a token does not see (NaN and infinities among it) does not reach its result.
 * q     [n_tokens][hq][d] (dtype)
 * out   [n_tokens][hq][d] (dtype: fp32 sums, rounded once); q, which is read until the end, is not it
 * lse   [n_tokens][hq] fp32 or NULL
 * A token whose scores are all NaN has NaN results.  What a token sees of V reaches its result
 * as the formula says: an infinity is the result, however small its row's weight (the row's
 * score finite), both of them in a dim or one in a row of score -inf (0 times it) are NaN.
 * Such results take longer: 2 to 5 us for 8 of a view's rows, and 5 for each that holds an
 * infinity, in the kernel's longest piece.
 * bf16: for a sequence of up to 16 new rows (its new tokens times hq / hkv) the weights
 * exp(s - max) are kept to 16 bits for their product with V, for longer ones they are
 * rounded to bf16; their sum is of the unrounded ones.
 * Errors: INVALID_ARG for null pointers, q or out not on 16-byte borders, a scale that
 * is not positive and finite, or a cache that is not of the plan's geometry; WORKSPACE. */
int catekv_paged_attn(const catekv_paged_cache* cache, const catekv_paged_plan_t* plan, const void* q, float scale,
                      void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* Slot dst_host[i] becomes a copy of slot src_host[i] that shares its pages.  Every
 * view of dst must be empty: one that is not is left unchanged, and *refused = 1
 * when refused is not NULL (int32, device, never cleared here).
 * Any number of pairs (a launch for every 256).
 * Errors: INVALID_ARG for null pointers, n < 1, a slot out of range, a dst listed
 * twice or also as a src. */
int catekv_paged_fork(const catekv_paged_cache* cache, const int32_t* src_host, const int32_t* dst_host, int n,
                      int32_t* refused, void* stream);

/* Takes the last rows[slot] rows (int64 [n_slots], device) off every view of every
 * slot, all of a view's rows if it has no more; values <= 0 leave a slot alone.
 * Pages behind the rows left are released and their entries become -1. */
int catekv_paged_drop(const catekv_paged_cache* cache, const int64_t* rows, void* stream);

/* Workspace bytes of catekv_paged_compact; 0 for sizes it refuses. */
size_t catekv_paged_compact_workspace(const catekv_paged_cache* cache, int n_sel, int b, int cs, int tail);

/* Cache(K, V, i_k, L_obs) of Algorithm 1 on pages: view heads_host[s] of `slot` keeps
 * the rows of the chunks idx[s][*] (int32 [n_sel][b], device) in the order listed,
 * chunk c being the rows [c cs, min((c + 1) cs, L - tail)) (entries without rows
 * ignored), then its last `tail` rows.  They move to pages taken lowest free first,
 * in the order of s and row; the view's old pages are released, and free after the
 * call if no other view holds them.
 * A view of fewer than `tail` rows, one whose rows would exceed max_pages, and the
 * first that does not find its pages and all later ones, are left unchanged, and
 * *overflow = 1 when overflow is not NULL (int32, device, never cleared here).
 * Errors: INVALID_ARG for null pointers, a slot out of range, n_sel outside [1, 128],
 * a head out of range or listed twice, b < 1, cs < 1 or tail < 0; UNSUPPORTED for
 * n_sel * b above 2^24 or b * cs + tail above 2^26; WORKSPACE. */
int catekv_paged_compact(const catekv_paged_cache* cache, int slot, const int32_t* heads_host, int n_sel,
                         const int32_t* idx, int b, int cs, int tail, int32_t* overflow, void* ws, size_t ws_bytes,
                         void* stream);

/* Writes the first min(lens, max_rows) rows of every view of the listed slots to
 * kv_out [n][hkv] (catekv_kv_ptrs, device; rows of d elements; a null k or v is
 * left out).  Slots may be listed more than once.
 * Errors: INVALID_ARG for null pointers, n outside [1, 256], a slot out of range or
 * max_rows < 1; UNSUPPORTED for sizes that would take a launch of 2^32 threads. */
int catekv_paged_gather(const catekv_paged_cache* cache, const int32_t* slots_host, int n,
                        const catekv_kv_ptrs* kv_out, int64_t max_rows, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CATEKV_PAGED_H */
