// Pages of a cache: taking, sharing, releasing and copying them (gfx950).
//
// The state is the views' tables and lengths, a count per page and a bit per free
// page.  Pages are taken lowest number first, so that no list of free pages has to be
// kept in an order: releasing is an atomic decrement per page and, where it reaches
// 0, an atomic or of its bit, and the result does not depend on the order of either.
// Taking runs in one workgroup: a scan over the views' needs, then a scan over the
// bits' words (1024 threads x 4 words: 262144 pages a turn) until enough are found.
#include "common.h"
#include "paged.h"

namespace catekv {
namespace {

constexpr int kTakeThreads = 1024;
constexpr int kTakeWaves = kTakeThreads / 64;
constexpr int kTakeWords = 4;                    // words of bits per thread and turn

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

// Sum of x over the threads before this one; total: over all.  Two barriers.
__device__ __forceinline__ int scan_block(int x, int* s_wave, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(v, o);
    if (lane >= o) v += y;
  }
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kTakeWaves; ++w) {
    const int y = s_wave[w];
    if (w < wave) before += y;
    all += y;
  }
  __syncthreads();
  total = all;
  return before + v - x;
}

// The numbers of the lowest `need` free pages into takes; returns how many there
// are, at most need.  Nothing is marked yet.
__device__ int find_free(const PagedCache& c, int need, int32_t* takes, int* s_wave) {
  const int words = (c.n_pages + 63) >> 6;
  int found = 0;
  for (int w0 = 0; w0 < words && found < need; w0 += kTakeThreads * kTakeWords) {
    uint64_t bits[kTakeWords];
    int n = 0;
    const int at = w0 + threadIdx.x * kTakeWords;
#pragma unroll
    for (int i = 0; i < kTakeWords; ++i) {
      uint64_t b = at + i < words ? c.bits[at + i] : 0;
      const int last = c.n_pages - (at + i) * 64;           // pages of the last word
      if (last < 64 && last > 0) b &= (1ull << last) - 1;
      bits[i] = b;
      n += __popcll(b);
    }
    int total;
    int place = found + scan_block(n, s_wave, total);
#pragma unroll
    for (int i = 0; i < kTakeWords; ++i) {
      uint64_t b = bits[i];
      while (b && place < need) {
        takes[place++] = (at + i) * 64 + __ffsll((unsigned long long)b) - 1;
        b &= b - 1;
      }
    }
    found += total;
  }
  __syncthreads();
  return found < need ? found : need;
}

__device__ void mark_taken(const PagedCache& c, const int32_t* takes, int n) {
  for (int j = threadIdx.x; j < n; j += kTakeThreads) {
    const int p = takes[j];
    c.refs[p] = 1;
    atomicAnd((unsigned long long*)&c.bits[p >> 6], ~(1ull << (p & 63)));
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
// Views are taken by whole sequences, as many as the workgroup has threads for.
__global__ __launch_bounds__(kTakeThreads) void paged_take_kernel(PagedAppend a) {
  __shared__ int s_wave[kTakeWaves];
  __shared__ int s_bad[kTakeThreads];
  __shared__ int s_end[kTakeThreads];
  __shared__ int s_used;
  const PagedCache& c = a.c;
  const int hkv = c.hkv, per = kTakeThreads / hkv, tid = threadIdx.x;
  const int si = tid / hkv, h = tid - si * hkv;
  // needs, numbered through
  int total = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += per) {
    const bool mine = si < per && s0 + si < a.n_seqs;
    if (tid < per) s_bad[tid] = 0;
    __syncthreads();
    int need = 0, from = -1;
    int64_t L = -1;
    if (mine) {
      const PagedSeq q = a.seqs[s0 + si];
      const int view = q.slot * hkv + h;
      L = c.lens[view];
      if (L < 0 || L + q.n_new > cap_rows(c)) {
        s_bad[si] = 1;
        if (q.n_new > 0 && a.overflow) *a.overflow = 1;
      } else if (q.n_new > 0) {
        const int had = pages_of(c, L);
        need = pages_of(c, L + q.n_new) - had;
        if (L & ((1 << c.page_log) - 1)) {
          const int last = page_in(c, row_of(c, view)[had - 1]);
          if (c.refs[last] > 1) {
            from = last;
            ++need;
          }
        }
      }
      if (q.n_new == 0) L = -1;
    }
    __syncthreads();
    if (mine && s_bad[si]) {
      need = 0;
      L = -1;
    }
    int sum;
    const int start = total + scan_block(need, s_wave, sum);
    total += sum;
    if (mine) a.views[(s0 + si) * hkv + h] = PagedTake{L, start, from};
  }
  const int found = total > 0 ? find_free(c, total, a.takes, s_wave) : 0;
  if (tid == 0) s_used = 0;
  __syncthreads();
  // a sequence whose last page was not found is left, and all after it that need any
  for (int s0 = 0; s0 < a.n_seqs; s0 += per) {
    const bool mine = si < per && s0 + si < a.n_seqs;
    const int v = (s0 + si) * hkv + h;
    PagedTake t{-1, 0, -1};
    int need = 0, n_new = 0, slot = 0;
    if (mine) {
      t = a.views[v];
      n_new = a.seqs[s0 + si].n_new;
      slot = a.seqs[s0 + si].slot;
      if (t.len >= 0) need = pages_of(c, t.len + n_new) - pages_of(c, t.len) + (t.from >= 0);
    }
    if (tid < per) {
      s_bad[tid] = 0;      // pages that the sequence needs
      s_end[tid] = 0;
    }
    __syncthreads();
    if (mine && need > 0) {
      atomicAdd(&s_bad[si], need);
      atomicMax(&s_end[si], t.start + need);
    }
    __syncthreads();
    if (mine && t.len >= 0) {
      if (s_bad[si] > 0 && s_end[si] > found) {
        a.views[v].len = -1;
        if (a.overflow) *a.overflow = 1;
      } else {
        const int view = slot * hkv + h;
        c.lens[view] = t.len + n_new;
        if (need > 0) atomicMax(&s_used, t.start + need);
      }
    }
    __syncthreads();
  }
  __syncthreads();
  const int used = s_used;
  mark_taken(c, a.takes, used);
  __syncthreads();
  for (int v = tid; v < a.n_seqs * hkv; v += kTakeThreads) {
    const PagedTake t = a.views[v];
    if (t.len >= 0 && t.from >= 0) release(c, t.from);
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
// One workgroup per view: the view's length is read and written by it alone.

__global__ __launch_bounds__(256) void paged_fork_kernel(PagedFork a) {
  const PagedCache& c = a.c;
  const int i = blockIdx.x / c.hkv, h = blockIdx.x - i * c.hkv;
  const int src = a.src[i] * c.hkv + h, dst = a.dst[i] * c.hkv + h;
  const int64_t L = rows_of(c, src);
  if (c.lens[dst] != 0) {
    if (threadIdx.x == 0 && a.refused) *a.refused = 1;
    return;
  }
  const int n = pages_of(c, L);
  const int32_t* from = row_of(c, src);
  int32_t* to = row_of(c, dst);
  for (int p = threadIdx.x; p < n; p += 256) {
    const int id = page_in(c, from[p]);
    to[p] = id;
    atomicAdd(&c.refs[id], 1);
  }
  __syncthreads();                                   // every thread has read the length
  if (threadIdx.x == 0) c.lens[dst] = L;
}

__global__ __launch_bounds__(256) void paged_drop_kernel(PagedCache c, const int64_t* rows) {
  const int view = blockIdx.x, slot = view / c.hkv;
  const int64_t off = rows[slot];
  const int64_t L = rows_of(c, view);
  if (off <= 0 || L == 0) return;
  const int64_t left = off < L ? L - off : 0;
  int32_t* row = row_of(c, view);
  const int n = pages_of(c, L);
  for (int p = pages_of(c, left) + (int)threadIdx.x; p < n; p += 256) {
    release(c, row[p]);
    row[p] = -1;
  }
  __syncthreads();
  if (threadIdx.x == 0) c.lens[view] = left;
}

// ---- compact ---------------------------------------------------------------------

__global__ __launch_bounds__(kTakeThreads) void paged_compact_take_kernel(PagedCompact a) {
  __shared__ int s_wave[kTakeWaves];
  __shared__ int64_t s_len[kPagedMaxHeads];
  __shared__ PagedTake s_take[kPagedMaxHeads];
  __shared__ int s_used;
  const PagedCache& c = a.c;
  const int tid = threadIdx.x;
  if (tid < a.n_sel) s_len[tid] = c.lens[a.slot * c.hkv + a.heads[tid]];
  __syncthreads();
  int total = 0;
  for (int s = 0; s < a.n_sel; ++s) {
    const int64_t L = s_len[s];
    const int64_t n = L - a.tail;
    const bool fine = n >= 0 && L <= cap_rows(c);
    int64_t rows = 0;
    for (int e0 = 0; e0 < a.b; e0 += kTakeThreads) {
      const int e = e0 + tid;
      int64_t len = 0;
      if (fine && e < a.b) {
        const int ch = a.idx[(size_t)s * a.b + e];
        if (ch >= 0) {
          len = n - (int64_t)ch * a.cs;
          len = len < 0 ? 0 : len > a.cs ? a.cs : len;
        }
      }
      int sum;
      const int before = scan_block((int)len, s_wave, sum);
      if (e < a.b) a.offs[(size_t)s * a.b + e] = (int)rows + before;
      rows += sum;
    }
    rows += a.tail;
    const bool fits = fine && rows <= cap_rows(c);
    const int need = fits ? pages_of(c, rows) : 0;
    if (tid == 0) {
      s_take[s] = PagedTake{fits ? L : -1, total, (int)rows};
      if (!fits && a.overflow) *a.overflow = 1;
    }
    total += need;
  }
  const int found = total > 0 ? find_free(c, total, a.takes, s_wave) : 0;
  __syncthreads();
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
  mark_taken(c, a.takes, s_used);
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

__global__ __launch_bounds__(256) void paged_compact_swap_kernel(PagedCompact a) {
  const PagedCache& c = a.c;
  const int s = blockIdx.x;
  const PagedTake t = a.views[s];
  if (t.len < 0) return;
  const int view = a.slot * c.hkv + a.heads[s];
  int32_t* row = row_of(c, view);
  const int had = pages_of(c, t.len), have = pages_of(c, t.from);
  for (int p = threadIdx.x; p < (had > have ? had : have); p += 256) {
    if (p < had) release(c, row[p]);
    row[p] = p < have ? a.takes[t.start + p] : -1;
  }
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
  paged_fork_kernel<<<a.n * a.c.hkv, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_drop(const PagedCache& c, const int64_t* rows, hipStream_t stream) {
  paged_drop_kernel<<<c.n_slots * c.hkv, 256, 0, stream>>>(c, rows);
  return hipGetLastError();
}

hipError_t launch_paged_compact(const PagedCompact& a, hipStream_t stream) {
  paged_compact_take_kernel<<<1, kTakeThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int lpr = a.c.row_bytes / 16;
  const int64_t rows = (int64_t)a.b * a.cs + a.tail;
  int64_t groups = (rows * lpr + 255) / 256;
  if (groups > 256) groups = 256;
  const unsigned grid = (unsigned)(groups * a.n_sel);
  if (lpr == 16) paged_compact_rows_kernel<16><<<grid, 256, 0, stream>>>(a, (int)groups);
  else paged_compact_rows_kernel<32><<<grid, 256, 0, stream>>>(a, (int)groups);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  paged_compact_swap_kernel<<<a.n_sel, 256, 0, stream>>>(a);
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
