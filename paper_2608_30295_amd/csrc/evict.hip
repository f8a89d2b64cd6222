// Eviction by accumulated weight: which chunks of a view stay, and the moves.
//
// The chunks' largest weights become ordered 32-bit keys, in the selecting
// workgroup itself or, for long views, in a launch of their own.  Up to kOneChunks
// chunks one workgroup per view selects: few chunks by counting, for each, the
// better ones; more by a radix selection of the k-th largest key in up to three
// digits, the keys in registers.  It lists the pairs (place that becomes free below
// k, kept chunk from k on) in ascending order.  More chunks are counted by many
// workgroups, a launch per digit, one for the counts that place their pairs and one
// that lists them (73000 chunks of 8 views: 144 us per eviction with one workgroup
// per view, of which 29 must move).
//
// One launch moves.  The pairs' sources lie from k on, their places below, so all
// of them move at once, whole chunks at a time.  The rows behind the chunks
// shift down over places that may still be sources: those pairs (the first of
// the list, as sources ascend) belong to the workgroups that shift, one per strip
// of the rows of K and of V, which read a turn's rows before they write any of
// them.  No order between workgroups is needed.
//
// Bound by latency where little moves (16 x 8 views of 2304 rows: 9 us select, of
// it 5 in dependent loads and barriers, 9 move) and by HBM where much does (8 views
// of 131072 rows to 16384: 117 MB moved in 26 us, 4.5 TB/s in 2 KB chunks, 61 MB read
// and 60 written by the counters; loads past the caches 24 us there, but 9.7 -> 11.8
// for the short views).  Many rows behind the chunks are what it is slow at: their few
// workgroups take them turn by turn (8 views of 131072 bf16 rows to 8192 and the rows
// behind: move 17 us with recent = 1024, 62 with 8192; in e4m3 42 with 8192).
#include "cache.h"
#include "common.h"

namespace catekv {

constexpr int kEvictThreads = 1024;
constexpr int kEvictWaves = kEvictThreads / 64;
constexpr int kBins = 2048;             // 11-bit digits: 11 + 11 + 10
constexpr int kMoveThreads = 256;
constexpr int64_t kMaxEvictRows = 1 << 26;   // 32 pieces a row, a workgroup per kKeyRows rows:
constexpr int kMaxEvictChunk = 1 << 20;      // element, piece and workgroup numbers stay below 2^31
constexpr int kMaxEvictViews = 1 << 16;
// Up to so many chunks their ranks are counted, else the k-th largest key is selected
// by radix.  us of the selecting launch, counted / radix, 128 views of 64 chunks: 6.2 /
// 8.8, 128: 6.2 / 9.3, 256: 7.4 / 9.4, 384: 9.4 / 10.0, 512: 10.6 / 9.3, 768: 18.6 / 10.5.
constexpr int kRankChunks = 384;
constexpr int kOneChunks = 16 * kEvictThreads;   // most chunks of a selecting workgroup (their keys' registers)
constexpr int kGroupChunks = 4 * kEvictThreads;  // chunks of one of many
// Views up to here: keys and zeros by the selecting and the shifting workgroup, two
// launches less.  us of all kernels, own / launches of their own, chunks of 8 rows, 64
// views of 8256 rows: 26.4 / 27.7, 16384: 40 / 42, 20480: 56 / 55, 32768: 89 / 78; us
// of a pass over 8 views of 8256 rows 22.5 / 22.8, 12288: 26.0 / 22.5, 16384: 30.4 /
// 22.4 (64 of 16384: 45.8 / 44.9), so that 8192 would suit few views better.
constexpr int kOwnKeyRows = 16384;
// Else by a workgroup per so many rows.  us of the keys at 2048 / 4096 / 8192 rows: 32
// views of 32768 rows 5.5 / 4.4 / 5.5, 8 of 131072 5.7 / 4.4 / 5.6, 32 of 131072 15.0 /
// 9.6 / 7.5, 8 of 524288 17.4 / 10.4 / 8.6.
constexpr int kKeyRows = 4096;

struct EvictInfo {
  int32_t moves;                        // pairs; the view is left alone if shift is 0
  int32_t nc, k, len;
  int32_t shift;                        // rows dropped
  int32_t rest;                         // rows of K and V behind the chunks (8 bits: those in codes)
  int32_t lead;                         // pairs whose source the shifted rows will cover
  uint32_t limit;                       // keys above it stay, and the first `ties` equal ones
  int32_t ties;
};

// What a group of kGroupChunks chunks holds: keys above the limit and equal to it,
// below chunk k and from there on.
struct GroupCount {
  int32_t above_lo, equal_lo, above_hi, equal_hi;
};

// Workspace: infos, the pairs of every view, then (long views) their keys, and
// (many chunks) the digits' histograms and the groups' counts.
static size_t info_bytes(int n_views) { return ((size_t)n_views * sizeof(EvictInfo) + 255) & ~(size_t)255; }
static int64_t max_chunks_of(int64_t max_rows, int cs) { return max_rows / cs; }
// at most half of the chunks can change places: min(k, nc - k)
static int64_t max_moves_of(int64_t chunks) { return chunks / 2 + 1; }
static size_t pairs_bytes(int n_views, int64_t chunks) {
  return ((size_t)n_views * (size_t)max_moves_of(chunks) * 2 * sizeof(int32_t) + 255) & ~(size_t)255;
}
static size_t key_bytes(int n_views, int64_t chunks) { return ((size_t)n_views * (size_t)chunks * sizeof(uint32_t) + 255) & ~(size_t)255; }
static int64_t groups_of(int64_t chunks) { return (chunks + kGroupChunks - 1) / kGroupChunks; }
static size_t hist_bytes(int n_views) { return (size_t)n_views * 3 * kBins * sizeof(uint32_t); }
size_t evict_workspace_bytes(int n_views, int64_t max_rows, int cs) {
  const int64_t chunks = max_chunks_of(max_rows, cs);
  size_t bytes = info_bytes(n_views) + pairs_bytes(n_views, chunks);
  if (max_rows > kOwnKeyRows) bytes += key_bytes(n_views, chunks);
  if (chunks > kOneChunks) bytes += hist_bytes(n_views) + (size_t)n_views * groups_of(chunks) * sizeof(GroupCount);
  return bytes;
}

// Chunks of a workgroup of evict_keys_kernel, and the workgroups per view of the
// launches whose grid grows with the rows.
static int key_chunks(int cs) { return kKeyRows / cs > 0 ? kKeyRows / cs : 1; }
static int64_t key_groups(int64_t chunks, int cs) { return (chunks + key_chunks(cs) - 1) / key_chunks(cs); }
static int64_t zero_groups(int64_t max_rows) { return (max_rows + kKeyRows - 1) / kKeyRows; }

bool evict_fits(int n_views, int64_t max_rows, int cs) {
  if (max_rows > kMaxEvictRows || cs > kMaxEvictChunk || n_views > kMaxEvictViews) return false;
  if (max_rows <= kOwnKeyRows) return true;             // a workgroup or a few per view
  const int64_t chunks = max_chunks_of(max_rows, cs);
  return launch_fits(key_groups(chunks, cs) * n_views, kEvictThreads) && launch_fits(groups_of(chunks) * n_views, kEvictThreads) &&
         launch_fits(zero_groups(max_rows) * n_views, kMoveThreads);
}

// Pointers that come out of tables are global ones: without the cast their accesses
// are flat, which wait for LDS as well.
template <typename E>
using Global = __attribute__((address_space(1))) E*;
template <typename E>
__device__ __forceinline__ Global<E> global(E* p) { return (Global<E>)p; }

// Larger key = larger weight; NaN above all, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float x) {
  uint32_t b = __float_as_uint(x);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (b == 0x80000000u) b = 0;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Maximum over each aligned group of g lanes, g a power of two.
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t group_max(uint32_t x, int g) {
  if (g >= 2) x = max_dpp<kDppXor1>(x);
  if (g >= 4) x = max_dpp<kDppXor2>(x);
  if (g >= 8) x = max_dpp<kDppHalfMirror>(x);
  if (g >= 16) x = max_dpp<kDppMirror>(x);
  if (g >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(r[0], r[1]);
  }
  if (g >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = max(r[0], r[1]);
  }
  return x;
}

// Keys of the chunks [c_lo, c_hi), by all threads of a workgroup: as many lanes to a
// chunk as it has rows (a power of two, at most 64), so that a wave reads
// consecutive weights; four groups of chunks per lane in flight.
template <typename Put>
__device__ __forceinline__ void chunk_keys(const float* acc, int cs, int c_lo, int c_hi, int threads, Put put) {
  const int g = 1 << (31 - __builtin_clz(min(cs, 64))), log_g = 31 - __builtin_clz(g);
  const int lane = threadIdx.x & (g - 1), per = threads >> log_g;
  for (int c0 = c_lo + (int)(threadIdx.x >> log_g); c0 - (int)(threadIdx.x >> log_g) < c_hi; c0 += 4 * per) {
    uint32_t x[4] = {0, 0, 0, 0};
    for (int i = lane; i < cs; i += g) {
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = min(c0 + u * per, c_hi - 1);
        w[u] = global(acc)[(size_t)c * cs + i];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = max(x[u], weight_key(w[u]));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t m = group_max(x[u], g);
      const int c = c0 + u * per;
      if (lane == 0 && c < c_hi) put(c, m);
    }
  }
}

// What a view has to drop: nc competing chunks of which k stay; false: nothing.
__device__ __forceinline__ bool evict_view(const EvictArgs& a, int bh, int64_t& len, int& nc, int& k) {
  len = a.lens[bh];
  k = a.budget[bh];
  const int64_t eligible = len > a.recent ? len - a.recent : 0;
  nc = (int)(eligible / a.cs);
  return len >= 0 && len <= a.max_rows && k >= 0 && nc > k;
}

struct SelectShared {
  uint32_t hist[kBins];
  int part[kEvictWaves];
  int part2[kEvictWaves];
  int lead;
  uint32_t digit;
  int above, inside;                    // keys above the chosen digit's bin, and in it
};

// The digit that holds the `want`-th largest of the histogram; s.above and
// s.inside: how many lie above its bin and in it.  Every thread calls it.
__device__ __forceinline__ void find_digit(SelectShared& s, int want) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  // thread t owns bins 2047 - 2 t and 2046 - 2 t: sums from the top
  const int h0 = (int)s.hist[kBins - 1 - 2 * t], h1 = (int)s.hist[kBins - 2 - 2 * t];
  int incl = h0 + h1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __builtin_amdgcn_ds_bpermute((lane - o) << 2, incl);
    if (lane >= o) incl += y;
  }
  if (lane == 63) s.part[wave] = incl;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < wave; ++w) base += s.part[w];
  const int before = base + incl - h0 - h1;
  if (before < want && want <= before + h0) {
    s.digit = (uint32_t)(kBins - 1 - 2 * t);
    s.above = before;
    s.inside = h0;
  } else if (before + h0 < want && want <= before + h0 + h1) {
    s.digit = (uint32_t)(kBins - 2 - 2 * t);
    s.above = before + h0;
    s.inside = h1;
  }
  __syncthreads();
}

// Where the wave's chunks lie: rows of 64 consecutive ones, [lo, hi).
struct Run {
  int lo, hi;
};

// The pairs of a view's chunks.  rows(f): f(row number, first chunk) for every row
// of this wave; stays(row, c): whether c, a chunk of the wave, stays, asked in order
// after each reset().  h, m: places and sources before this workgroup's chunks.
// Returns the number of its places; s.lead gets that of its sources below `covered`.
template <typename Rows, typename Reset, typename Stays>
__device__ __forceinline__ int list_pairs(SelectShared& s, Run run, int k, int covered, int32_t* pairs, Rows rows, Reset reset,
                                          Stays stays, int h = 0, int m = 0) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0;
  int holes = 0, movers = 0;
  reset();
  // a row below k holds places only, one from k on sources only
  rows([&](int i, int c0) {
    const int c = c0 + lane;
    const bool st = stays(i, c);
    if (c0 < k) holes += __popcll(__builtin_amdgcn_ballot_w64(!st && c < min(k, run.hi)));
    if (c0 + 63 >= k) movers += __popcll(__builtin_amdgcn_ballot_w64(st && c >= k));
  });
  __syncthreads();
  if (lane == 0) {
    s.part[wave] = holes;
    s.part2[wave] = movers;
  }
  if (threadIdx.x == 0) s.lead = 0;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    h += w < wave ? s.part[w] : 0;
    m += w < wave ? s.part2[w] : 0;
    total += s.part[w];
  }
  reset();
  rows([&](int i, int c0) {
    const int c = c0 + lane;
    const bool st = stays(i, c);
    if (c0 < k) {
      const bool hole = !st && c < min(k, run.hi);
      const uint64_t hm = __builtin_amdgcn_ballot_w64(hole);
      if (hole) pairs[2 * (h + __popcll(hm & below))] = c;
      h += __popcll(hm);
    }
    if (c0 + 63 >= k) {
      const bool mover = st && c >= k;
      const uint64_t mm = __builtin_amdgcn_ballot_w64(mover);
      if (mover) pairs[2 * (m + __popcll(mm & below)) + 1] = c;
      m += __popcll(mm);
      if (c0 < covered) {
        const int lead = __popcll(__builtin_amdgcn_ballot_w64(mover && c < covered));
        if (lane == 0 && lead) atomicAdd(&s.lead, lead);
      }
    }
  });
  __syncthreads();
  return total;
}

// Up to kRankChunks keys in LDS (padded to a multiple of four with zeros, which are
// no chunk's key): chunk c stays if fewer than k are better (ties: the lower
// chunk).  The better ones are counted by as many waves per chunk as there are;
// against the chunks of another wave a tie always or never counts, so that two
// instructions do.  s.hist holds the counts, zero on entry.
__device__ __forceinline__ int rank_pairs(SelectShared& s, const uint32_t* keys, int nc, int k, int covered, int32_t* pairs) {
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int per = (nc + 63) / 64, parts = kEvictWaves / per;       // waves per part: one chunk per lane
  const int part = wave / per, own = (wave - part * per) * 64, c = own + lane;
  if (part < parts) {
    const uint32_t x = keys[min(c, nc - 1)];
    const int step = ((nc + 3) / 4 + parts - 1) / parts * 4, j0 = part * step, j1 = min(nc, j0 + step);
    int rank = 0;
    auto count = [&](int lo, int hi, uint32_t limit) {               // keys above limit
#pragma unroll 4
      for (int j = lo; j < hi; j += 4) {
        const uint4 w = *reinterpret_cast<const uint4*>(keys + j);
        rank += w.x > limit;
        rank += w.y > limit;
        rank += w.z > limit;
        rank += w.w > limit;
      }
    };
    count(j0, min(j1, own), x - 1);
#pragma unroll 4
    for (int j = max(j0, own); j < min(j1, own + 64); j += 4) {
      const uint4 w = *reinterpret_cast<const uint4*>(keys + j);
      rank += w.x > (j < c ? x - 1 : x);
      rank += w.y > (j + 1 < c ? x - 1 : x);
      rank += w.z > (j + 2 < c ? x - 1 : x);
      rank += w.w > (j + 3 < c ? x - 1 : x);
    }
    count(max(j0, own + 64), j1, x);
    if (c < nc) atomicAdd(&s.hist[c], (uint32_t)rank);
  }
  __syncthreads();
  const bool st = t < nc && (int)s.hist[min(t, nc - 1)] < k;
  return list_pairs(s, Run{wave * 64, min(nc, wave * 64 + 64)}, k, covered, pairs,
                    [&](auto f) { if (wave * 64 < nc) f(0, wave * 64); }, [] {}, [&](int, int) { return st; });
}

// Which of any number of keys stay, k < nc of them: those above `limit` and the
// first `ties` equal ones.  key(row, c): the key of chunk c of this wave's row.
template <typename Rows, typename Keys>
__device__ __forceinline__ void radix_limit(SelectShared& s, Run run, Rows rows, Keys key, int k, uint32_t& limit, int& ties) {
  const int t = threadIdx.x, lane = t & 63;
  limit = 0xffffffffu;
  ties = 0;
  if (k == 0) return;
  uint32_t prefix = 0;
  ties = k;
#pragma unroll 1
  for (int p = 0; p < 3; ++p) {
    const int sh = p == 0 ? 21 : p == 1 ? 10 : 0, bits = p == 2 ? 10 : 11;
    const uint32_t mask = p == 0 ? 0u : 0xffffffffu << (sh + bits);
    __syncthreads();
    s.hist[t] = 0;
    s.hist[t + kEvictThreads] = 0;
    __syncthreads();
    rows([&](int i, int c0) {
      const int c = c0 + lane;
      const uint32_t x = key(i, c);
      if (c < run.hi && (x & mask) == prefix) atomicAdd(&s.hist[(x >> sh) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    find_digit(s, ties);
    prefix |= s.digit << sh;
    ties -= s.above;
    limit = prefix;
    if (ties == s.inside && prefix != 0) {       // all of this bin stays: no ties to tell apart
      limit = prefix - 1;
      ties = 0;
      return;
    }
  }
}

// Keys equal to limit in the waves before this one.
template <typename Rows, typename Keys>
__device__ __forceinline__ int ties_before(SelectShared& s, Run run, Rows rows, Keys key, uint32_t limit) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int n = 0;
  rows([&](int i, int c0) {
    const int c = c0 + lane;
    n += __popcll(__builtin_amdgcn_ballot_w64(c < run.hi && key(i, c) == limit));
  });
  __syncthreads();
  if (lane == 0) s.part[wave] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) n += w < wave ? s.part[w] : 0;
  return n;
}

// Whether chunk c stays; `tie`: equal keys before its row.
__device__ __forceinline__ bool stays_at(uint32_t x, bool valid, uint32_t limit, int ties, int& tie) {
  bool st = valid && x > limit;
  if (ties > 0) {
    const int lane = threadIdx.x & 63;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(valid && x == limit);
    st = st || (valid && x == limit && tie + __popcll(eq & (lane ? ~0ull >> (64 - lane) : 0)) < ties);
    tie += __popcll(eq);
  }
  return st;
}

// A lane's R keys in registers: nc <= 1024 R.  R = 2 where they fit, else 16: us of the
// selecting launch with 2 / 16, 512 chunks 8.9 / 15.0, 1024: 11.1 / 17.5, 2048: 12.9 /
// 19.2.
template <int R, typename Load>
__device__ __forceinline__ int register_pairs(SelectShared& s, Load load, int nc, int k, int covered, int32_t* pairs) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Run run{min(nc, wave * 64 * R), min(nc, (wave + 1) * 64 * R)};
  uint32_t x[R];
#pragma unroll
  for (int i = 0; i < R; ++i) x[i] = load(min(run.lo + i * 64 + lane, nc - 1));
  auto rows = [&](auto f) {
#pragma unroll
    for (int i = 0; i < R; ++i) f(i, run.lo + i * 64);
  };
  auto key = [&](int i, int) { return x[i]; };
  uint32_t limit;
  int ties;
  radix_limit(s, run, rows, key, k, limit, ties);
  int tie = ties > 0 ? ties_before(s, run, rows, key, limit) : 0;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) bits |= (uint32_t)stays_at(x[i], run.lo + i * 64 + lane < run.hi, limit, ties, tie) << i;
  return list_pairs(s, run, k, covered, pairs, rows, [] {}, [&](int i, int) { return (bits >> i & 1) != 0; });
}

// Rows behind the competing chunks: all of them (whose chunks' worth of places after
// k the shift covers), and those of K and V that move (8 bits: the ones in codes).
__device__ __forceinline__ EvictInfo evict_info(const EvictArgs& a, int64_t len, int nc, int k) {
  const int64_t from = (int64_t)nc * a.cs;
  EvictInfo f{};
  f.nc = nc;
  f.k = k;
  f.len = (int32_t)len;
  f.shift = (nc - k) * a.cs;
  f.rest = (int)((a.q8 ? len / a.block * a.block : len) - from);
  return f;
}
__device__ __forceinline__ int covered_below(const EvictInfo& f, int cs) {
  return f.k + (int)(((int64_t)f.len - (int64_t)f.nc * cs + cs - 1) / cs);
}

// ---- many chunks: a workgroup per group, a launch per step ----------------------
__global__ __launch_bounds__(kEvictThreads) void evict_clear_kernel(uint32_t* hist, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kEvictThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kEvictThreads) hist[i] = 0;
}

// A workgroup's histogram in LDS added to the view's.
__device__ __forceinline__ void add_hist(const SelectShared& s, uint32_t* hist) {
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kEvictThreads)
    if (s.hist[i]) atomicAdd(&hist[i], s.hist[i]);
}

// The digits decided by the first n of the view's histograms: limit so far (its lower
// bits 0) and how many of its keys stay; false: all of a bin stays, nothing is open.
__device__ __forceinline__ bool decide(SelectShared& s, const uint32_t* hist, int n, int k, uint32_t& limit, int& ties) {
  const int t = threadIdx.x;
  limit = 0xffffffffu;
  ties = 0;
  if (k == 0) return false;
  uint32_t prefix = 0;
  ties = k;
#pragma unroll 1
  for (int p = 0; p < n; ++p) {
    __syncthreads();
    s.hist[t] = hist[p * kBins + t];
    s.hist[t + kEvictThreads] = hist[p * kBins + t + kEvictThreads];
    __syncthreads();
    find_digit(s, ties);
    prefix |= s.digit << (p == 0 ? 21 : p == 1 ? 10 : 0);
    ties -= s.above;
    limit = prefix;
    if (ties == s.inside && prefix != 0) {
      limit = prefix - 1;
      ties = 0;
      return false;
    }
  }
  return true;
}

// Digit P (1 or 2) of the keys that share the digits before it.
template <int P>
__global__ __launch_bounds__(kEvictThreads) void evict_digit_kernel(EvictArgs a, const uint32_t* keys, uint32_t* hist,
                                                                    int64_t max_chunks) {
  __shared__ SelectShared s;
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views, t = threadIdx.x;
  int64_t len;
  int nc, k;
  if (!evict_view(a, bh, len, nc, k) || (int64_t)group * kGroupChunks >= nc) return;
  uint32_t x[4];
  const uint32_t* mine = keys + (size_t)bh * max_chunks;
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = mine[min(group * kGroupChunks + u * kEvictThreads + t, nc - 1)];
  uint32_t* h = hist + (size_t)bh * 3 * kBins;
  uint32_t limit;
  int ties;
  if (!decide(s, h, P, k, limit, ties)) return;
  __syncthreads();
  s.hist[t] = 0;
  s.hist[t + kEvictThreads] = 0;
  __syncthreads();
  constexpr int sh = P == 1 ? 10 : 0, bits = P == 1 ? 11 : 10;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (group * kGroupChunks + u * kEvictThreads + t < nc && (x[u] >> (sh + bits)) == (limit >> (sh + bits)))
      atomicAdd(&s.hist[(x[u] >> sh) & ((1u << bits) - 1)], 1u);
  add_hist(s, h + P * kBins);
}

// The limit, and every group's counts.
__global__ __launch_bounds__(kEvictThreads) void evict_count_kernel(EvictArgs a, EvictInfo* infos, const uint32_t* keys,
                                                                    const uint32_t* hist, GroupCount* counts,
                                                                    int64_t max_chunks, int groups) {
  __shared__ SelectShared s;
  __shared__ GroupCount total;
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views, t = threadIdx.x, lane = t & 63;
  int64_t len;
  int nc, k;
  if (!evict_view(a, bh, len, nc, k)) {
    if (group == 0 && t == 0) infos[bh] = EvictInfo{};
    return;
  }
  if ((int64_t)group * kGroupChunks >= nc) return;
  uint32_t x[4];
  const uint32_t* mine = keys + (size_t)bh * max_chunks;
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = mine[min(group * kGroupChunks + u * kEvictThreads + t, nc - 1)];
  if (t == 0) total = GroupCount{};
  uint32_t limit;
  int ties;
  decide(s, hist + (size_t)bh * 3 * kBins, 3, k, limit, ties);
  __syncthreads();
  GroupCount n{};
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int c = group * kGroupChunks + u * kEvictThreads + t;
    const bool above = c < nc && x[u] > limit, equal = c < nc && x[u] == limit;
    n.above_lo += __popcll(__builtin_amdgcn_ballot_w64(above && c < k));
    n.equal_lo += __popcll(__builtin_amdgcn_ballot_w64(equal && c < k));
    n.above_hi += __popcll(__builtin_amdgcn_ballot_w64(above && c >= k));
    n.equal_hi += __popcll(__builtin_amdgcn_ballot_w64(equal && c >= k));
  }
  if (lane == 0) {
    atomicAdd(&total.above_lo, n.above_lo);
    atomicAdd(&total.equal_lo, n.equal_lo);
    atomicAdd(&total.above_hi, n.above_hi);
    atomicAdd(&total.equal_hi, n.equal_hi);
  }
  __syncthreads();
  if (t == 0) {
    counts[(size_t)bh * groups + group] = total;
    if (group == 0) {
      EvictInfo f = evict_info(a, len, nc, k);
      f.limit = limit;
      f.ties = ties;
      infos[bh] = f;
    }
  }
}

// Every group's pairs; the first group also writes their number and the new length
// (no workgroup of this launch reads lens).
__global__ __launch_bounds__(kEvictThreads) void evict_list_kernel(EvictArgs a, EvictInfo* infos, int32_t* pairs,
                                                                   const uint32_t* keys, const GroupCount* counts,
                                                                   int64_t max_chunks, int64_t max_moves, int groups) {
  __shared__ SelectShared s;
  __shared__ GroupCount before, total;
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views, t = threadIdx.x;
  const int lane = t & 63, wave = t >> 6;
  const EvictInfo f = infos[bh];
  const int nc = f.nc, k = f.k, first = group * kGroupChunks;
  if (f.shift == 0 || first >= nc) return;
  const int n_groups = (nc + kGroupChunks - 1) / kGroupChunks;
  const Run run{min(nc, first + wave * 256), min(nc, first + (wave + 1) * 256)};
  const uint32_t* mine = keys + (size_t)bh * max_chunks;
  uint32_t x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = mine[min(run.lo + i * 64 + lane, nc - 1)];
  if (t == 0) before = total = GroupCount{};
  __syncthreads();
  for (int g = t; g < n_groups; g += kEvictThreads) {
    const GroupCount c = counts[(size_t)bh * groups + g];
    if (g < group) {
      atomicAdd(&before.above_lo, c.above_lo);
      atomicAdd(&before.equal_lo, c.equal_lo);
      atomicAdd(&before.above_hi, c.above_hi);
      atomicAdd(&before.equal_hi, c.equal_hi);
    }
    atomicAdd(&total.above_lo, c.above_lo);
    atomicAdd(&total.equal_lo, c.equal_lo);
  }
  __syncthreads();
  // equal keys stay in order: those below k first
  const int holes = min(k, first) - before.above_lo - min(f.ties, before.equal_lo);
  const int movers = before.above_hi + min(f.ties, total.equal_lo + before.equal_hi) - min(f.ties, total.equal_lo);
  auto rows = [&](auto g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) g(i, run.lo + i * 64);
  };
  auto key = [&](int i, int) { return x[i]; };
  int tie = before.equal_lo + before.equal_hi;
  if (f.ties > 0) tie += ties_before(s, run, rows, key, f.limit);
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) bits |= (uint32_t)stays_at(x[i], run.lo + i * 64 + lane < run.hi, f.limit, f.ties, tie) << i;
  list_pairs(s, run, k, covered_below(f, a.cs), pairs + (size_t)bh * max_moves * 2, rows, [] {},
             [&](int i, int) { return (bits >> i & 1) != 0; }, holes, movers);
  if (t == 0) {
    if (s.lead) atomicAdd(&infos[bh].lead, s.lead);
    if (group == 0) {
      infos[bh].moves = k - total.above_lo - min(f.ties, total.equal_lo);
      a.lens[bh] = (int64_t)f.len - f.shift;
    }
  }
}

// Keys of long views: workgroups over kKeyRows rows each; hist: the first digit's
// histogram of every view (many chunks), or null.
__global__ __launch_bounds__(kEvictThreads) void evict_keys_kernel(EvictArgs a, uint32_t* keys, uint32_t* hist,
                                                                   int64_t max_chunks, int per_wg) {
  __shared__ SelectShared s;
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views;
  int64_t len;
  int nc, k;
  if (!evict_view(a, bh, len, nc, k)) return;
  const int64_t c_lo = (int64_t)group * per_wg;
  if (c_lo >= nc) return;
  uint32_t* mine = keys + (size_t)bh * max_chunks;
  s.hist[threadIdx.x] = 0;
  s.hist[threadIdx.x + kEvictThreads] = 0;
  __syncthreads();
  chunk_keys(a.acc[bh], a.cs, (int)c_lo, (int)min((int64_t)nc, c_lo + per_wg), kEvictThreads, [&](int c, uint32_t x) {
    mine[c] = x;
    if (hist) atomicAdd(&s.hist[x >> 21], 1u);
  });
  if (hist) add_hist(s, hist + (size_t)bh * 3 * kBins);
}

// keys: null where this workgroup makes its own.
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a, EvictInfo* infos, int32_t* pairs,
                                                                     const uint32_t* keys, int64_t max_chunks,
                                                                     int64_t max_moves) {
  extern __shared__ uint4 s_dyn[];
  uint32_t* s_keys = reinterpret_cast<uint32_t*>(s_dyn);
  __shared__ SelectShared s;
  const int bh = blockIdx.x, t = threadIdx.x;
  int64_t len;
  int nc, k;
  const bool drops = evict_view(a, bh, len, nc, k);
  __syncthreads();                       // the length is read before it is replaced
  if (!drops) {
    if (t == 0) infos[bh] = EvictInfo{};
    return;
  }
  const uint32_t* mine = keys ? keys + (size_t)bh * max_chunks : s_keys;
  if (!keys) {
    chunk_keys(a.acc[bh], a.cs, 0, nc, kEvictThreads, [&](int c, uint32_t x) { s_keys[c] = x; });
  } else if (nc <= kRankChunks) {
    if (t < nc) s_keys[t] = mine[t];
  }
  if (nc <= kRankChunks) {
    if (t < 4) s_keys[nc + t] = 0;       // rank_pairs reads four at a time
    if (t < kRankChunks) s.hist[t] = 0;
  }
  __syncthreads();
  int32_t* out = pairs + (size_t)bh * max_moves * 2;
  EvictInfo f = evict_info(a, len, nc, k);
  const int covered = covered_below(f, a.cs);
  auto load = [&](int c) { return mine[c]; };
  f.moves = nc <= kRankChunks          ? rank_pairs(s, s_keys, nc, k, covered, out)
            : nc <= 2 * kEvictThreads ? register_pairs<2>(s, load, nc, k, covered, out)
                                      : register_pairs<16>(s, load, nc, k, covered, out);
  if (t == 0) {
    f.lead = s.lead;
    infos[bh] = f;
    a.lens[bh] = len - f.shift;
  }
}

constexpr int kMoveBatch = 8;           // loads of a thread in flight

// Three runs of elements of p in one sequence: n_fill from p[src(i)] to p[dst(i)],
// n_shift from p[from + i] to p[to + i] (to < from), then n_zero zeros from p[end]
// on.  A turn's elements are all read before one is written.  What a turn writes
// no later turn reads: fills lie below all sources, shifted elements below the
// sources of the shifts still to come, and zeros come last.
template <typename E, typename Src, typename Dst, typename From, typename To>
__device__ __forceinline__ void move_elements(E* generic, int n_fill, Src src, Dst dst, int n_shift, From from, To to, int n_zero,
                                              size_t end) {
  const Global<E> p = global(generic);
  const int n = n_fill + n_shift + n_zero;
  for (int i0 = 0; i0 < n; i0 += kMoveThreads * kMoveBatch) {
    E w[kMoveBatch];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int i = i0 + u * kMoveThreads + (int)threadIdx.x;
      w[u] = E{};
      if (i < n_fill) w[u] = p[src(i)];
      else if (i < n_fill + n_shift) w[u] = p[from(i - n_fill)];
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int i = i0 + u * kMoveThreads + (int)threadIdx.x;
      if (i < n_fill) p[dst(i)] = w[u];
      else if (i < n_fill + n_shift) p[to(i - n_fill)] = w[u];
      else if (i < n) p[end + (size_t)(i - n_fill - n_shift)] = w[u];
    }
  }
}

// blockIdx.x: view.  blockIdx.y: first the workgroups that shift: one for the weights
// (and, for codes, one for the scales of K and one for those of V, which they move
// whole), one per strip of K and of V (16 << strip_log bytes); then `fills` that fill
// places in K, as many for V, and `acc_fills` for the weights (none where their
// shifting workgroup writes the zeros behind them too).
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, const EvictInfo* infos,
                                                                  const int32_t* pairs, int64_t max_moves, int fills,
                                                                  int acc_fills, int strip_log, bool zeros) {
  const int bh = blockIdx.x, cs = a.cs;
  const EvictInfo f = infos[bh];
  if (f.shift == 0) return;
  const int2* pr = reinterpret_cast<const int2*>(pairs) + (size_t)bh * max_moves;
  const int pieces = a.row_bytes / 16, strips = pieces >> strip_log, floats = a.q8 ? 3 : 1;
  int y = blockIdx.y;
  if (y < floats) {
    // elements of a chunk: its rows' weights, or its blocks' scales
    const int per = y == 0 ? cs : cs / a.block;
    float* p = y == 0 ? a.acc[bh] : y == 1 ? a.q8[bh].k_scale : a.q8[bh].v_scale;
    // with the zeros all of them: they may cover any source of a pair
    const int fill = y == 0 && !zeros ? f.lead : f.moves;
    const int behind = y == 0 ? (int)((int64_t)f.len - (int64_t)f.nc * cs) : f.rest / a.block;
    move_elements(p, fill * per,
                  [&](int i) { const int q = i / per; return (size_t)pr[q].y * per + (i - q * per); },
                  [&](int i) { const int q = i / per; return (size_t)pr[q].x * per + (i - q * per); },
                  behind, [&](int i) { return (size_t)f.nc * per + i; }, [&](int i) { return (size_t)f.k * per + i; },
                  y == 0 && zeros ? f.shift : 0, (size_t)(f.len - f.shift));
    return;
  }
  y -= floats;
  const bool shifting = y < 2 * strips;
  if (!shifting) y -= 2 * strips;
  if (!shifting && y >= 2 * fills) {
    y -= 2 * fills;
    const Global<float> p = global(a.acc[bh]);
    const int n = (f.moves - f.lead) * cs, step = kMoveThreads * kMoveBatch;
    for (int i0 = y * step; i0 < n; i0 += acc_fills * step) {
      int2 c[kMoveBatch];
      int off[kMoveBatch];
      float w[kMoveBatch];
#pragma unroll
      for (int u = 0; u < kMoveBatch; ++u) {
        const int i = min(i0 + u * kMoveThreads + (int)threadIdx.x, n - 1), q = i / cs;
        off[u] = i - q * cs;
        c[u] = pr[f.lead + q];
      }
#pragma unroll
      for (int u = 0; u < kMoveBatch; ++u) w[u] = p[(size_t)c[u].y * cs + off[u]];
#pragma unroll
      for (int u = 0; u < kMoveBatch; ++u) p[(size_t)c[u].x * cs + off[u]] = w[u];   // beyond n: the last one again
    }
    return;
  }
  const int of_k = shifting ? strips : fills;
  const bool is_v = y >= of_k;
  if (is_v) y -= of_k;
  char* base = a.q8 ? reinterpret_cast<char*>(is_v ? a.q8[bh].v : a.q8[bh].k)
                    : reinterpret_cast<char*>(const_cast<void*>(is_v ? a.kv[bh].v : a.kv[bh].k));
  if (shifting) {
    // element i: piece i % 2^strip_log of the strip's row i / 2^strip_log
    const int64_t at = (int64_t)f.k * cs, from = (int64_t)f.nc * cs;
    u32x4_t* p = reinterpret_cast<u32x4_t*>(base) + (y << strip_log);
    const int in = (1 << strip_log) - 1;
    move_elements(p, (f.lead * cs) << strip_log,
                  [&](int i) { const int r = i >> strip_log, q = r / cs; return ((size_t)pr[q].y * cs + (r - q * cs)) * pieces + (i & in); },
                  [&](int i) { const int r = i >> strip_log, q = r / cs; return ((size_t)pr[q].x * cs + (r - q * cs)) * pieces + (i & in); },
                  f.rest << strip_log, [&](int i) { return (size_t)(from + (i >> strip_log)) * pieces + (i & in); },
                  [&](int i) { return (size_t)(at + (i >> strip_log)) * pieces + (i & in); }, 0, 0);
    return;
  }
  const int piece = cs * pieces;                     // 16-byte pieces of a chunk
  const int64_t n = (int64_t)(f.moves - f.lead) * piece;
  const size_t chunk_bytes = (size_t)cs * a.row_bytes;
  for (int64_t i0 = (int64_t)y * (kMoveThreads * kMoveBatch); i0 < n; i0 += (int64_t)fills * (kMoveThreads * kMoveBatch)) {
    // chunk and piece of the turn's first element, then 32-bit steps from there
    const int64_t q0 = i0 / piece, first = f.lead + q0;
    const uint32_t off0 = (uint32_t)(i0 - q0 * piece);
    int2 c[kMoveBatch];
    uint32_t off[kMoveBatch];
    uint4 w[kMoveBatch];
    bool mine[kMoveBatch];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const uint32_t j = off0 + u * kMoveThreads + threadIdx.x, q = j / (uint32_t)piece;
      const int64_t pi = first + q;
      off[u] = (j - q * piece) * 16;
      c[u] = pr[min(pi, (int64_t)f.moves - 1)];
      mine[u] = pi < f.moves;
    }
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) w[u] = ldg16(base + (size_t)c[u].y * chunk_bytes + off[u]);
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u)
      if (mine[u]) *global(reinterpret_cast<u32x4_t*>(base + (size_t)c[u].x * chunk_bytes + off[u])) = u32x4_t{w[u].x, w[u].y, w[u].z, w[u].w};
  }
}

// Zeros behind the new lengths of long views (16 KB of weights per workgroup).
__global__ __launch_bounds__(kMoveThreads) void evict_zero_kernel(EvictArgs a, const EvictInfo* infos) {
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views;
  const EvictInfo f = infos[bh];
  if (f.shift == 0) return;
  const Global<float> acc = global(a.acc[bh]);
  const int64_t lo = (int64_t)(f.len - f.shift) + (int64_t)group * kKeyRows, hi = min((int64_t)f.len, lo + kKeyRows);
#pragma unroll 4
  for (int64_t i = lo + threadIdx.x; i < hi; i += kMoveThreads) acc[i] = 0.f;
}

// Every launch is followed by a look at its status: none may run on what a refused one
// before it has not written.
hipError_t launch_evict(const EvictArgs& a, hipStream_t stream) {
  hipError_t e;
  const int64_t chunks = max_chunks_of(a.max_rows, a.cs), moves = max_moves_of(chunks);
  char* w = reinterpret_cast<char*>(a.ws);
  EvictInfo* infos = reinterpret_cast<EvictInfo*>(w);
  int32_t* pairs = reinterpret_cast<int32_t*>(w + info_bytes(a.n_views));
  uint32_t* keys = nullptr;
  const bool many = chunks > kOneChunks;
  if (a.max_rows > kOwnKeyRows && chunks > 0) {
    char* behind = w + info_bytes(a.n_views) + pairs_bytes(a.n_views, chunks);
    keys = reinterpret_cast<uint32_t*>(behind);
    uint32_t* hist = many ? reinterpret_cast<uint32_t*>(behind + key_bytes(a.n_views, chunks)) : nullptr;
    if (many) {
      const int64_t n = (int64_t)a.n_views * 3 * kBins;
      hipLaunchKernelGGL(evict_clear_kernel, dim3((unsigned)(n / kEvictThreads < 1024 ? n / kEvictThreads : 1024)),
                         dim3(kEvictThreads), 0, stream, hist, n);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(evict_keys_kernel, dim3((unsigned)(key_groups(chunks, a.cs) * a.n_views)), dim3(kEvictThreads), 0, stream,
                       a, keys, hist, chunks, key_chunks(a.cs));
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (many) {
      GroupCount* counts = reinterpret_cast<GroupCount*>(behind + key_bytes(a.n_views, chunks) + hist_bytes(a.n_views));
      const int groups = (int)groups_of(chunks);
      const dim3 grid((unsigned)((int64_t)groups * a.n_views)), block(kEvictThreads);
      hipLaunchKernelGGL(evict_digit_kernel<1>, grid, block, 0, stream, a, keys, hist, chunks);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(evict_digit_kernel<2>, grid, block, 0, stream, a, keys, hist, chunks);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(evict_count_kernel, grid, block, 0, stream, a, infos, keys, hist, counts, chunks, groups);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(evict_list_kernel, grid, block, 0, stream, a, infos, pairs, keys, counts, chunks, moves, groups);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (!many) {
    const int64_t in_lds = keys ? kRankChunks : chunks;
    hipLaunchKernelGGL(evict_select_kernel, dim3(a.n_views), dim3(kEvictThreads), (size_t)(in_lds + 4) * sizeof(uint32_t),
                       stream, a, infos, pairs, keys, chunks, moves);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  // A fill workgroup moves kTurn bytes per turn: as many as the most chunks that may
  // move keep busy, but about four rounds of the device at most (512 each for K and V,
  // at least 4 per view.  us of the move with 128 / 512 / 2048: 128 views of 2304 rows,
  // 40 chunks to drop, 8.4 / 8.5 / 10.0; 8 views of 131072 rows to 16384 31.1 / 23.6 /
  // 22.9; 128 of 16384 to 8192 119.4 / 119.6 / 114.7).  A strip is as wide
  // as its workgroup moves in one turn, the rows behind the chunks being fewer than
  // recent + cs and those filled first hardly more.
  constexpr int64_t kTurn = kMoveThreads * kMoveBatch * 16;
  const int64_t turns = (moves * a.cs * a.row_bytes + kTurn - 1) / kTurn;
  const int64_t room = 512 / a.n_views > 4 ? 512 / a.n_views : 4;
  const int fills = (int)(turns < room ? turns : room);
  int strip_log = 2;
  while ((16 << strip_log) < a.row_bytes && 2 * ((int64_t)a.recent + a.cs) * (32 << strip_log) <= kTurn) ++strip_log;
  const int64_t acc_turns = (moves * a.cs + kMoveThreads * kMoveBatch - 1) / (kMoveThreads * kMoveBatch);
  const int acc_fills = !keys ? 0 : (int)(acc_turns < room / 4 + 1 ? acc_turns : room / 4 + 1);
  const int shifts = (a.q8 ? 3 : 1) + 2 * ((a.row_bytes / 16) >> strip_log);
  hipLaunchKernelGGL(evict_move_kernel, dim3(a.n_views, shifts + 2 * fills + acc_fills), dim3(kMoveThreads), 0, stream, a,
                     infos, pairs, moves, fills, acc_fills, strip_log, keys == nullptr);
  if ((e = hipGetLastError()) != hipSuccess || !keys) return e;
  hipLaunchKernelGGL(evict_zero_kernel, dim3((unsigned)(zero_groups(a.max_rows) * a.n_views)), dim3(kMoveThreads), 0, stream, a,
                     infos);
  return hipGetLastError();
}

}  // namespace catekv
