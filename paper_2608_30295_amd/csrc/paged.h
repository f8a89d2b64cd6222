// Internal interface of the caches in pages: what paged_api.cpp passes to the
// kernels of paged_*.hip.
#pragma once

#include "cache.h"
#include "catekv_paged.h"

namespace catekv {

constexpr int64_t kPagedMaxRows = (int64_t)1 << 26;   // of a view
constexpr int kPagedMaxList = 256;                    // slots of a gather, pairs of one of a fork's launches
constexpr int kPagedMaxHeads = 128;                   // heads of a compaction
constexpr int kPagedMaxHkv = 1024;                    // views of a slot (threads of the taking workgroup)

// The cache as kernels see it.
struct PagedCache {
  char* k;
  char* v;
  int32_t* table;
  int64_t* lens;
  int32_t* refs;
  uint64_t* bits;
  int32_t n_pages, n_slots, hkv, max_pages;
  int32_t page_log;                 // page = 1 << page_log rows
  int32_t row_bytes;                // of a K or V row
};

// A sequence of a plan.
struct PagedSeq {
  int32_t slot, n_new, tok0, pad;
};

// What the append's first launch leaves for its second, per view of the batch.
struct PagedTake {
  int64_t len;                      // rows before the call; -1: nothing is appended
  int32_t start;                    // the view's first page among those taken
  int32_t from;                     // the shared last page that is copied, or -1
};

struct PagedAppend {
  PagedCache c;
  const PagedSeq* seqs;
  const int32_t* tok_seq;           // sequence of every token
  PagedTake* views;                 // [n_seqs * hkv]
  int32_t* takes;                   // pages taken
  const char* k_new;
  const char* v_new;
  int64_t tok_bytes, head_bytes;    // strides of k_new and v_new
  int32_t* overflow;
  int32_t n_seqs, n_tokens;
};
hipError_t launch_paged_init(const PagedCache& c, hipStream_t stream);
hipError_t launch_paged_append(const PagedAppend& a, hipStream_t stream);

struct PagedFork {
  PagedCache c;
  int32_t* refused;
  int32_t n;
  int32_t src[kPagedMaxList], dst[kPagedMaxList];
};
hipError_t launch_paged_fork(const PagedFork& a, hipStream_t stream);
hipError_t launch_paged_drop(const PagedCache& c, const int64_t* rows, hipStream_t stream);

struct PagedCompact {
  PagedCache c;
  const int32_t* idx;
  int32_t* offs;                    // [n_sel][b] first row of every listed chunk among the view's new rows
  PagedTake* views;                 // [n_sel]; from: the view's new rows
  int32_t* takes;
  int32_t* overflow;
  int32_t slot, n_sel, b, cs, tail;
  int32_t heads[kPagedMaxHeads];
};
hipError_t launch_paged_compact(const PagedCompact& a, hipStream_t stream);

struct PagedGather {
  PagedCache c;
  const catekv_kv_ptrs* out;
  int64_t max_rows;
  int32_t n;
  int32_t slots[kPagedMaxList];
};
constexpr int kGatherThreads = 256;
int64_t paged_gather_groups(int64_t max_rows, int row_bytes);   // workgroups per view
hipError_t launch_paged_gather(const PagedGather& a, hipStream_t stream);

// ---- attention -----------------------------------------------------------------
// New rows of a sequence in one view's group: row = token * G + head of the group.
// A piece of work: new rows [row0, row0 + R) over the cached rows [t0, t1) of a view.
struct PagedPiece {
  int32_t view;                     // slot * hkv + head
  int32_t tok0, n_new;              // of the sequence
  int32_t row0;
  int32_t t0, t1;
  int32_t max_rows;                 // planned rows of the view
  int32_t slot;                     // partial slot at that many 16-byte units, or -1: the rows' only piece
};
// New rows whose pieces are joined: n_parts slots of `rows` rows, one behind the other.
struct PagedJoin {
  int32_t view, tok0, n_new, row0;
  int32_t slot, n_parts, rows, pad;
};
// A partial slot of R rows: o [R][128], then m [R] and l [R]: o = sum exp2(c (s - m)) v and
// l = sum exp2(c (s - m)) of the scores s as the products give them, c = log2_scale; m = -inf:
// no row.
constexpr size_t paged_slot_floats(int R) { return (size_t)R * (kD + 2); }

constexpr int kStreamRows = 16;     // new rows of a stream piece at most (the 16 columns of an MFMA)
constexpr int kPagedUnit = 64;      // pieces begin at multiples of so many cached rows

struct PagedAttn {
  PagedCache c;
  const char* q;
  char* out;
  float* lse;
  const PagedPiece* pieces;         // tiles of many new rows by worker, and
  const int32_t* workers;           // the first of every worker
  const PagedPiece* segs;           // segments of few new rows, the same
  const int32_t* seg_workers;
  const PagedJoin* joins;
  float* slots;
  int32_t n, n_few;                 // workers of the tiles, of the segments
  int32_t hq;
  float scale;
  float log2_scale;                 // of the scores as the products give them, to units of log2
  float rise;                       // by how much a maximum grows before it is moved: 8 / log2_scale
};
constexpr int kTileThreads = 512;        // bf16; fp32: 256
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = kJoinThreads / 32;   // rows of a joining workgroup, where rows have few parts
// Joins of one kind (tiles, few new rows): how many, workgroups of each, and whether a row
// is shared by eight groups, which is so from more than 8 parts on.
struct JoinShape {
  int32_t n, blocks, deep;
};
inline JoinShape paged_join_shape(int n, int rows, int parts) { return {n, parts > 8 ? rows : (rows + kJoinRows - 1) / kJoinRows, parts > 8}; }
// New rows of a tile piece at most, and the launch, per type.
constexpr int kTileRows = 256, kTileRowsF32 = 128;
inline int paged_tile_rows(int dtype) { return dtype == CATEKV_BF16 ? kTileRows : kTileRowsF32; }
hipError_t launch_paged_tile(int G, const PagedAttn& a, hipStream_t stream);       // bf16
hipError_t launch_paged_mixed(int G, const PagedAttn& a, hipStream_t stream);      // bf16, tiles and segments
hipError_t launch_paged_tile_f32(int G, const PagedAttn& a, hipStream_t stream);
hipError_t launch_paged_stream(int dtype, int G, const PagedAttn& a, hipStream_t stream);
hipError_t launch_paged_join(int dtype, int G, const PagedAttn& a, const JoinShape& tile, const JoinShape& few, hipStream_t stream);

}  // namespace catekv
