// Pages of a cache: taking, sharing, releasing and copying them (gfx950).
//
// The state is the views' tables and lengths, a count per page and a bit per free
// page.  Pages are taken lowest number first, so that no list of free pages has to be
// kept in an order: releasing is an atomic decrement per page and, where it reaches
// 0, an atomic or of its bit, and the result does not depend on the order of either.
// Taking runs in one workgroup: a scan over the views' needs, then a scan over the
// bits' words (65536 pages a turn) until enough are found.  It is bound by loads that need each
// other (sequence, length, last page, its count: 2.5 us) and the scans: 6 to 10 us
// for 48 to 640 pages.  Rows and gathering are bound by HBM: gathering 8 views of
// 131072 bf16 rows 198 us, 5.4 TB/s read and written.
#include "common.h"
#include "paged.h"

namespace catekv {
namespace {

constexpr int kTakeThreads = 1024;
constexpr int kTakeWaves = kTakeThreads / 64;

// ---- state ---------------------------------------------------------------------

__device__ __forceinline__ int64_t cap_rows(const PagedCache& c) { return (int64_t)c.max_pages << c.page_log; }
__device__ __forceinline__ int pages_of(const PagedCache& c, int64_t rows) {
  return (int)((rows + (1 << c.page_log) - 1) >> c.page_log);
}
__device__ __forceinline__ int32_t* row_of(const PagedCache& c, int view) { return c.table + (size_t)view * c.max_pages; }
// A view's length; 0 for one out of range.
__device__ __forceinline__ int64_t rows_of(const PagedCache& c, int view) {
  const int64_t L = c.lens[view];
  return L < 0 || L > cap_rows(c) ? 0 : L;
}
__device__ __forceinline__ int page_in(const PagedCache& c, int id) { return (uint32_t)id < (uint32_t)c.n_pages ? id : 0; }

// One view fewer holds page id; the last one's leaving sets the page's bit.
__device__ __forceinline__ void release(const PagedCache& c, int id) {
  if ((uint32_t)id >= (uint32_t)c.n_pages) return;
  if (atomicSub(&c.refs[id], 1) == 1) atomicOr((unsigned long long*)&c.bits[id >> 6], 1ull << (id & 63));
}

// ---- scans within a workgroup of kTakeThreads -----------------------------------

// Sum of x over the threads before this one; total: over all.  Two barriers, which wait
// for LDS alone: stores to memory keep flowing.
__device__ __forceinline__ int scan_block(int x, int* s_wave, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  if (lane == 63) s_wave[wave] = v;
  barrier_lds_only();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kTakeWaves; ++w) {
    const int y = s_wave[w];
    if (w < wave) before += y;
    all += y;
  }
  barrier_lds_only();
  total = all;
  return before + v - x;
}

struct TakeLds {
  int wave[kTakeWaves];
  int before[kTakeThreads];
  uint64_t word[kTakeThreads];
};

// Word number `at` of the free pages' bits.
__device__ __forceinline__ uint64_t free_word(const PagedCache& c, int at) {
  uint64_t b = at < (c.n_pages + 63) >> 6 ? c.bits[at] : 0;
  const int last = c.n_pages - at * 64;                     // pages of the last word
  return last < 64 && last > 0 ? b & ((1ull << last) - 1) : b;
}

// Takes the lowest `need` free pages, or all that there are; returns how many.  A thread
// counts a word (the first turn's given: asked for before it was known what is needed);
// then the waves go over the words up to the last that is needed, every sixteenth each,
// a lane per bit.  A word has one writer, so that its bits go with a plain store.
__device__ int take_free(const PagedCache& c, uint64_t word, int need, int32_t* takes, TakeLds& s) {
  const int words = (c.n_pages + 63) >> 6, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int found = 0;
  for (int w0 = 0; w0 < words && found < need; w0 += kTakeThreads) {
    if (w0 > 0) word = free_word(c, w0 + tid);
    int total;
    const int before = found + scan_block(__popcll(word), s.wave, total);
    s.word[tid] = word;
    s.before[tid] = before;
    barrier_lds_only();
    for (int i = wave; i < kTakeThreads; i += kTakeWaves) {
      const int first = __builtin_amdgcn_readfirstlane(s.before[i]);
      if (first >= need) break;
      const uint64_t b = s.word[i];
      const int place = first + __popcll(b & ((1ull << lane) - 1));
      const bool mine = (b >> lane & 1) && place < need;
      const uint64_t gone = __builtin_amdgcn_ballot_w64(mine);
      if (mine) {
        const int p = (w0 + i) * 64 + lane;
        takes[place] = p;
        c.refs[p] = 1;
      }
      if (lane == 0 && gone) c.bits[w0 + i] = b & ~gone;
    }
    found += total;
    barrier_lds_only();
  }
  return found < need ? found : need;
}

// The pages [n, found) of those taken are free again.
__device__ void give_back(const PagedCache& c, const int32_t* takes, int n, int found) {
  __syncthreads();
  for (int j = n + (int)threadIdx.x; j < found; j += kTakeThreads) {
    const int p = takes[j];
    c.refs[p] = 0;
    atomicOr((unsigned long long*)&c.bits[p >> 6], 1ull << (p & 63));
  }
}

// ---- init ----------------------------------------------------------------------

__global__ __launch_bounds__(256) void paged_init_kernel(PagedCache c) {
  const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t views = (int64_t)c.n_slots * c.hkv;
  for (int64_t i = first; i < views * c.max_pages; i += step) c.table[i] = -1;
  for (int64_t i = first; i < views; i += step) c.lens[i] = 0;
  for (int64_t i = first; i < c.n_pages; i += step) c.refs[i] = 0;
  for (int64_t i = first; i < ((int64_t)c.n_pages + 63) / 64; i += step) {
    const int64_t left = c.n_pages - i * 64;
    c.bits[i] = left >= 64 ? ~0ull : (1ull << left) - 1;
  }
}

// ---- append --------------------------------------------------------------------

// First launch: what every view needs, the pages, lengths and released pages.
// Views are taken by whole sequences, as many as the workgroup has threads for; what a
// thread found out about its view stays in registers if that is all of them.
__global__ __launch_bounds__(kTakeThreads) void paged_take_kernel(PagedAppend a) {
  __shared__ TakeLds s;
  __shared__ int s_bad[kTakeThreads];
  __shared__ int s_end[kTakeThreads];
  __shared__ int s_used;
  const PagedCache& c = a.c;
  const int hkv = c.hkv, per = kTakeThreads / hkv, tid = threadIdx.x;
  const int si = tid / hkv, h = tid - si * hkv;
  const bool once = a.n_seqs <= per;
  PagedTake t{-1, 0, -1};
  PagedSeq q{};
  int need = 0;
  if (tid == 0) s_used = 0;
  const uint64_t word = free_word(c, tid);
  // needs, numbered through
  int total = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += per) {
    const bool mine = si < per && s0 + si < a.n_seqs;
    if (tid < per) s_bad[tid] = 0;
    barrier_lds_only();
    t = PagedTake{-1, 0, -1};
    need = 0;
    if (mine) {
      q = a.seqs[s0 + si];
      const int view = q.slot * hkv + h;
      const int64_t L = c.lens[view];
      if (q.n_new > 0) {
        if (L < 0 || L > cap_rows(c) - q.n_new) {     // (lengths of any size: L + n_new may not exist)
          s_bad[si] = 1;
          if (a.overflow) *a.overflow = 1;
        } else {
          t.len = L;
          const int had = pages_of(c, L);
          need = pages_of(c, L + q.n_new) - had;
          if (L & ((1 << c.page_log) - 1)) {
            const int last = page_in(c, row_of(c, view)[had - 1]);
            if (c.refs[last] > 1) {
              t.from = last;
              ++need;
            }
          }
        }
      }
    }
    barrier_lds_only();
    if (mine && s_bad[si]) {
      need = 0;
      t.len = -1;
    }
    int sum;
    t.start = total + scan_block(need, s.wave, sum);
    total += sum;
    if (mine && !once) a.views[(s0 + si) * hkv + h] = t;
  }
  const int found = total > 0 ? take_free(c, word, total, a.takes, s) : 0;
  bool copies = false;
  // a sequence whose last page was not found is left, and all after it that need any
  for (int s0 = 0; s0 < a.n_seqs; s0 += per) {
    const bool mine = si < per && s0 + si < a.n_seqs;
    const int v = (s0 + si) * hkv + h;
    if (!once) {
      need = 0;
      if (mine) {
        t = a.views[v];
        q = a.seqs[s0 + si];
        if (t.len >= 0) need = pages_of(c, t.len + q.n_new) - pages_of(c, t.len) + (t.from >= 0);
      }
    }
    if (found < total) {
      if (tid < per) s_end[tid] = 0;     // past the last page that the sequence needs
      barrier_lds_only();
      if (mine && need > 0) atomicMax(&s_end[si], t.start + need);
      barrier_lds_only();
      if (mine && t.len >= 0) {
        if (s_end[si] > found) {
          t.len = -1;
          if (a.overflow) *a.overflow = 1;
        } else if (need > 0) {
          atomicMax(&s_used, t.start + need);
        }
      }
      barrier_lds_only();
    }
    if (mine) {
      if (t.len >= 0) c.lens[q.slot * hkv + h] = t.len + q.n_new;
      copies |= t.len >= 0 && t.from >= 0;
      a.views[v] = t;
    }
  }
  if (found < total) give_back(c, a.takes, s_used, found);
  // what is left of shared pages, once the bits above are stored
  if (!__syncthreads_or(copies)) return;
  if (once) {
    if (t.len >= 0 && t.from >= 0) release(c, t.from);
    return;
  }
  for (int v = tid; v < a.n_seqs * hkv; v += kTakeThreads) {
    const PagedTake u = a.views[v];
    if (u.len >= 0 && u.from >= 0) release(c, u.from);
  }
}

// Second launch: rows, tables and copies.  LPR lanes move one row.
template <int LPR>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedAppend a, int row_groups) {
  const PagedCache& c = a.c;
  const int hkv = c.hkv;
  const int lane = threadIdx.x & (LPR - 1), group = threadIdx.x / LPR;
  constexpr int GROUPS = 256 / LPR;
  const int mask = (1 << c.page_log) - 1;
  if ((int)blockIdx.x >= row_groups) {               // a shared last page's rows, one view per workgroup
    const PagedTake t = a.views[blockIdx.x - row_groups];
    if (t.len < 0 || t.from < 0) return;
    const size_t to = (size_t)a.takes[t.start] << c.page_log, from = (size_t)t.from << c.page_log;
    const int n = (int)(t.len & mask);
    for (int r = group; r < n; r += GROUPS) {
      const size_t x = (from + r) * c.row_bytes + lane * 16, y = (to + r) * c.row_bytes + lane * 16;
      const uint4 kk = ldg16(c.k + x), vv = ldg16(c.v + x);
      *reinterpret_cast<uint4*>(c.k + y) = kk;
      *reinterpret_cast<uint4*>(c.v + y) = vv;
    }
    return;
  }
  const int64_t item = (int64_t)blockIdx.x * GROUPS + group;
  if (item >= (int64_t)a.n_tokens * hkv) return;
  const int tok = (int)(item / hkv), h = (int)(item - (int64_t)tok * hkv);
  const int si = a.tok_seq[tok];
  const PagedSeq q = a.seqs[si];
  const PagedTake t = a.views[si * hkv + h];
  if (t.len < 0) return;
  const int view = q.slot * hkv + h, j = tok - q.tok0;
  const int64_t row = t.len + j;
  const int p = (int)(row >> c.page_log), had = pages_of(c, t.len);
  int32_t* entry = row_of(c, view) + p;
  int id;
  if (p >= had) id = a.takes[t.start + (t.from >= 0) + p - had];
  else if (t.from >= 0) id = a.takes[t.start];
  else id = page_in(c, *entry);
  if (lane == 0 && ((row & mask) == 0 || (j == 0 && t.from >= 0))) *entry = id;
  const size_t src = (size_t)tok * a.tok_bytes + (size_t)h * a.head_bytes + lane * 16;
  const size_t dst = (((size_t)id << c.page_log) + (row & mask)) * c.row_bytes + lane * 16;
  const uint4 kk = ldg16(a.k_new + src), vv = ldg16(a.v_new + src);
  *reinterpret_cast<uint4*>(c.k + dst) = kk;
  *reinterpret_cast<uint4*>(c.v + dst) = vv;
}

// ---- fork and drop ---------------------------------------------------------------
// One workgroup per view: the view's length is read and written by it alone.  A thread
// has kAhead entries on their way at a time.
constexpr int kEntryThreads = 512;
constexpr int kAhead = 4;

// f(page, entry) of the entries [p0, p1) of a row
template <class F>
__device__ __forceinline__ void each_entry(const int32_t* row, int p0, int p1, F f) {
  for (int p = p0 + (int)threadIdx.x; p < p1; p += kEntryThreads * kAhead) {
    int id[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) id[i] = p + i * kEntryThreads < p1 ? row[p + i * kEntryThreads] : -1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (p + i * kEntryThreads < p1) f(p + i * kEntryThreads, id[i]);
  }
}

// The entries' pages released: all counts down before the first bit.
__device__ __forceinline__ void release_entries(const PagedCache& c, int32_t* row, int p0, int p1) {
  for (int p = p0 + (int)threadIdx.x; p < p1; p += kEntryThreads * kAhead) {
    int id[kAhead], was[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) id[i] = p + i * kEntryThreads < p1 ? row[p + i * kEntryThreads] : -1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) was[i] = (uint32_t)id[i] < (uint32_t)c.n_pages ? atomicSub(&c.refs[id[i]], 1) : 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (was[i] == 1) atomicOr((unsigned long long*)&c.bits[id[i] >> 6], 1ull << (id[i] & 63));
  }
}

__global__ __launch_bounds__(kEntryThreads) void paged_fork_kernel(PagedFork a) {
  const PagedCache& c = a.c;
  const int i = blockIdx.x / c.hkv, h = blockIdx.x - i * c.hkv;
  const int src = a.src[i] * c.hkv + h, dst = a.dst[i] * c.hkv + h;
  const int64_t L = rows_of(c, src);
  if (c.lens[dst] != 0) {
    if (threadIdx.x == 0 && a.refused) *a.refused = 1;
    return;
  }
  int32_t* to = row_of(c, dst);
  each_entry(row_of(c, src), 0, pages_of(c, L), [&](int p, int id) {
    id = page_in(c, id);
    to[p] = id;
    atomicAdd(&c.refs[id], 1);
  });
  __syncthreads();                                   // every thread has read the length
  if (threadIdx.x == 0) c.lens[dst] = L;
}

__global__ __launch_bounds__(kEntryThreads) void paged_drop_kernel(PagedCache c, const int64_t* rows) {
  const int view = blockIdx.x, slot = view / c.hkv;
  const int64_t off = rows[slot];
  const int64_t L = rows_of(c, view);
  if (off <= 0 || L == 0) return;
  const int64_t left = off < L ? L - off : 0;
  int32_t* row = row_of(c, view);
  const int p0 = pages_of(c, left), p1 = pages_of(c, L);
  release_entries(c, row, p0, p1);
  for (int p = p0 + (int)threadIdx.x; p < p1; p += kEntryThreads) row[p] = -1;   // a thread's own entries
  __syncthreads();
  if (threadIdx.x == 0) c.lens[view] = left;
}

// ---- compact ---------------------------------------------------------------------

// Rows of chunk `ch` of a view that has n rows before its tail (n < 0: none).
__device__ __forceinline__ int chunk_rows(const PagedCompact& a, int64_t n, int ch) {
  const int64_t len = ch >= 0 ? n - (int64_t)ch * a.cs : 0;
  return (int)(len < 0 ? 0 : len > a.cs ? a.cs : len);
}
// The view's entry for its rows before (L) and after (rows, the tail among them).
__device__ __forceinline__ PagedTake compact_take(const PagedCompact& a, int64_t L, int rows) {
  const bool fine = L >= a.tail && L <= cap_rows(a.c) && rows <= cap_rows(a.c);
  return PagedTake{fine ? L : -1, 0, rows};
}
__device__ __forceinline__ int64_t compact_len(const PagedCompact& a, int s) {
  return a.c.lens[a.slot * a.c.hkv + a.heads[s]];
}
// Rows before the tail of a view of L; -1: none of them can be listed.
__device__ __forceinline__ int64_t compact_body(const PagedCompact& a, int64_t L) {
  return L >= a.tail && L <= cap_rows(a.c) ? L - a.tail : -1;
}

// How many rows every view keeps, and where its chunks go.  Lists of up to kShortList
// chunks are gone over by a wave each of the taking workgroup; longer ones by a workgroup
// each, four chunks to a thread, in a launch of their own (5 lists of 512 chunks: 8.5 us with
// the taking, of 1024 11.8; as a launch 4.1 and 4.6 behind it, whichever; 3 of 29197: 20
// instead of 210).
constexpr int kShortList = 512;

__global__ __launch_bounds__(kTakeThreads) void paged_compact_list_kernel(PagedCompact a) {
  __shared__ int s_wave[kTakeWaves];
  const int s = blockIdx.x, tid = threadIdx.x;
  const int64_t L = compact_len(a, s), n = compact_body(a, L);
  const int32_t* list = a.idx + (size_t)s * a.b;
  int32_t* offs = a.offs + (size_t)s * a.b;
  int rows = 0, next[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) next[i] = 4 * tid + i < a.b ? list[4 * tid + i] : -1;
  for (int e0 = 0; e0 < a.b; e0 += 4 * kTakeThreads) {
    const int e = e0 + 4 * tid, f = e + 4 * kTakeThreads;
    int len[4], sum = 0, total;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += len[i] = chunk_rows(a, n, next[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = f + i < a.b ? list[f + i] : -1;
    int at = rows + scan_block(sum, s_wave, total);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (e + i < a.b) offs[e + i] = at;
      at += len[i];
    }
    rows += total;
  }
  if (tid == 0) a.views[s] = compact_take(a, L, rows + a.tail);
}

// The pages.
__global__ __launch_bounds__(kTakeThreads) void paged_compact_take_kernel(PagedCompact a) {
  __shared__ TakeLds s_find;
  __shared__ PagedTake s_take[kPagedMaxHeads];
  __shared__ int s_used, s_total;
  const PagedCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const uint64_t word = free_word(c, tid);
  if (a.b > kShortList) {
    if (tid < a.n_sel) s_take[tid] = a.views[tid];
  } else {
    for (int s = tid >> 6; s < a.n_sel; s += kTakeWaves) {
      const int64_t L = compact_len(a, s), n = compact_body(a, L);
      int rows = 0;
      const int32_t* list = a.idx + (size_t)s * a.b;
      int next = lane < a.b ? list[lane] : -1;
      for (int e0 = 0; e0 < a.b; e0 += 64) {
        const int e = e0 + lane, ch = next;
        next = e + 64 < a.b ? list[e + 64] : -1;
        const int len = chunk_rows(a, n, ch);
        int v = len;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(v, o);
          if (lane >= o) v += y;
        }
        if (e < a.b) a.offs[(size_t)s * a.b + e] = rows + v - len;
        rows += __shfl(v, 63);
      }
      if (lane == 0) s_take[s] = compact_take(a, L, rows + a.tail);
    }
  }
  __syncthreads();
  if (tid == 0) {
    int total = 0;
    for (int s = 0; s < a.n_sel; ++s) {
      s_take[s].start = total;
      if (s_take[s].len >= 0) total += pages_of(c, s_take[s].from);
      else if (a.overflow) *a.overflow = 1;
    }
    s_total = total;
  }
  __syncthreads();
  const int total = s_total;
  const int found = total > 0 ? take_free(c, word, total, a.takes, s_find) : 0;
  // the first view that does not find its pages and all after it that need any stay
  if (tid == 0) {
    int used = 0;
    for (int s = 0; s < a.n_sel; ++s) {
      const PagedTake t = s_take[s];
      if (t.len < 0 || t.from == 0) continue;
      const int end = t.start + pages_of(c, t.from);
      if (end <= found) {
        used = end;
      } else {
        s_take[s].len = -1;
        if (a.overflow) *a.overflow = 1;
      }
    }
    s_used = used;
  }
  __syncthreads();
  if (tid < a.n_sel) a.views[tid] = s_take[tid];
  if (s_used < found) give_back(c, a.takes, s_used, found);
}

template <int LPR>
__global__ __launch_bounds__(256) void paged_compact_rows_kernel(PagedCompact a, int groups) {
  const PagedCache& c = a.c;
  const int s = blockIdx.x / groups;
  const PagedTake t = a.views[s];
  if (t.len < 0) return;
  const int view = a.slot * c.hkv + a.heads[s];
  const int32_t* old = row_of(c, view);
  const int lane = threadIdx.x & (LPR - 1);
  const int mask = (1 << c.page_log) - 1;
  const int64_t n = t.len - a.tail;
  const int body = a.b * a.cs, step = groups * (256 / LPR);
  for (int i = ((int)blockIdx.x - s * groups) * (256 / LPR) + (int)threadIdx.x / LPR; i < body + a.tail; i += step) {
    int64_t from, to;
    if (i < body) {
      const int e = i / a.cs, r = i - e * a.cs;
      const int ch = a.idx[(size_t)s * a.b + e];
      from = (int64_t)ch * a.cs + r;
      if (ch < 0 || from >= n) continue;
      to = (int64_t)a.offs[(size_t)s * a.b + e] + r;
    } else {
      from = n + (i - body);
      to = t.from - a.tail + (i - body);
    }
    const size_t x = (((size_t)page_in(c, old[from >> c.page_log]) << c.page_log) + (from & mask)) * c.row_bytes + lane * 16;
    const size_t y = (((size_t)a.takes[t.start + (to >> c.page_log)] << c.page_log) + (to & mask)) * c.row_bytes + lane * 16;
    const uint4 kk = ldg16(c.k + x), vv = ldg16(c.v + x);
    *reinterpret_cast<uint4*>(c.k + y) = kk;
    *reinterpret_cast<uint4*>(c.v + y) = vv;
  }
}

__global__ __launch_bounds__(kEntryThreads) void paged_compact_swap_kernel(PagedCompact a) {
  const PagedCache& c = a.c;
  const int s = blockIdx.x;
  const PagedTake t = a.views[s];
  if (t.len < 0) return;
  const int view = a.slot * c.hkv + a.heads[s];
  int32_t* row = row_of(c, view);
  const int had = pages_of(c, t.len), have = pages_of(c, t.from);
  release_entries(c, row, 0, had);
  // a thread's own entries: the same ones that it released
  for (int p = threadIdx.x; p < (had > have ? had : have); p += kEntryThreads) row[p] = p < have ? a.takes[t.start + p] : -1;
  if (threadIdx.x == 0) c.lens[view] = t.from;
}

// ---- gather ----------------------------------------------------------------------

// GATHER_ROWS rows per group of LPR lanes, all loads before the first store.
constexpr int kGatherRows = 4;
template <int LPR>
__global__ __launch_bounds__(kGatherThreads) void paged_gather_kernel(PagedGather a, int groups) {
  const PagedCache& c = a.c;
  const int vi = blockIdx.x / groups, g = blockIdx.x - vi * groups;
  const int i = vi / c.hkv, h = vi - i * c.hkv;
  const int view = a.slots[i] * c.hkv + h;
  const int64_t L = min(rows_of(c, view), a.max_rows);
  const int lane = threadIdx.x & (LPR - 1);
  constexpr int GROUPS = kGatherThreads / LPR;
  const int mask = (1 << c.page_log) - 1;
  const int32_t* ids = row_of(c, view);
  const int64_t first = (int64_t)g * (GROUPS * kGatherRows) + threadIdx.x / LPR;
  if (first >= L) return;
  const catekv_kv_ptrs o = a.out[vi];
  uint4 kk[kGatherRows], vv[kGatherRows];
#pragma unroll
  for (int r = 0; r < kGatherRows; ++r) {
    const int64_t t = min(first + r * GROUPS, L - 1);
    const size_t x = (((size_t)page_in(c, ids[t >> c.page_log]) << c.page_log) + (t & mask)) * c.row_bytes + lane * 16;
    if (o.k) kk[r] = once16(c.k + x);
    if (o.v) vv[r] = once16(c.v + x);
  }
#pragma unroll
  for (int r = 0; r < kGatherRows; ++r) {
    const int64_t t = first + r * GROUPS;
    if (t >= L) break;
    char* kd = (char*)o.k + (size_t)t * c.row_bytes + lane * 16;
    char* vd = (char*)o.v + (size_t)t * c.row_bytes + lane * 16;
    if (o.k) *reinterpret_cast<uint4*>(kd) = kk[r];
    if (o.v) *reinterpret_cast<uint4*>(vd) = vv[r];
  }
}

}  // namespace

hipError_t launch_paged_init(const PagedCache& c, hipStream_t stream) {
  paged_init_kernel<<<1024, 256, 0, stream>>>(c);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t stream) {
  paged_take_kernel<<<1, kTakeThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_tokens == 0) return e;
  const int lpr = a.c.row_bytes / 16;
  const int groups = (int)(((int64_t)a.n_tokens * a.c.hkv * lpr + 255) / 256);
  const unsigned grid = (unsigned)(groups + a.n_seqs * a.c.hkv);
  if (lpr == 16) paged_rows_kernel<16><<<grid, 256, 0, stream>>>(a, groups);
  else paged_rows_kernel<32><<<grid, 256, 0, stream>>>(a, groups);
  return hipGetLastError();
}

hipError_t launch_paged_fork(const PagedFork& a, hipStream_t stream) {
  paged_fork_kernel<<<a.n * a.c.hkv, kEntryThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_drop(const PagedCache& c, const int64_t* rows, hipStream_t stream) {
  paged_drop_kernel<<<c.n_slots * c.hkv, kEntryThreads, 0, stream>>>(c, rows);
  return hipGetLastError();
}

hipError_t launch_paged_compact(const PagedCompact& a, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.b > kShortList) {
    paged_compact_list_kernel<<<a.n_sel, kTakeThreads, 0, stream>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  paged_compact_take_kernel<<<1, kTakeThreads, 0, stream>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int lpr = a.c.row_bytes / 16;
  const int64_t rows = (int64_t)a.b * a.cs + a.tail;
  int64_t groups = (rows * lpr + 255) / 256;
  const int64_t most = a.n_sel < 16 ? 4096 / a.n_sel : 256;   // workgroups of a view
  if (groups > most) groups = most;
  const unsigned grid = (unsigned)(groups * a.n_sel);
  if (lpr == 16) paged_compact_rows_kernel<16><<<grid, 256, 0, stream>>>(a, (int)groups);
  else paged_compact_rows_kernel<32><<<grid, 256, 0, stream>>>(a, (int)groups);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  paged_compact_swap_kernel<<<a.n_sel, kEntryThreads, 0, stream>>>(a);
  return hipGetLastError();
}

int64_t paged_gather_groups(int64_t max_rows, int row_bytes) {
  const int rows = kGatherThreads / (row_bytes / 16) * kGatherRows;
  return (max_rows + rows - 1) / rows;
}

hipError_t launch_paged_gather(const PagedGather& a, hipStream_t stream) {
  const int64_t groups = paged_gather_groups(a.max_rows, a.c.row_bytes);
  const unsigned grid = (unsigned)(groups * a.n * a.c.hkv);
  if (a.c.row_bytes == 256) paged_gather_kernel<16><<<grid, kGatherThreads, 0, stream>>>(a, (int)groups);
  else paged_gather_kernel<32><<<grid, kGatherThreads, 0, stream>>>(a, (int)groups);
  return hipGetLastError();
}

}  // namespace catekv
