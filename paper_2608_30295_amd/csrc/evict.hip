// Eviction by accumulated weight: which chunks of a view stay, and the moves.
//
// One launch selects (a workgroup per view): the chunks' largest weights as
// ordered 32-bit keys, kept in LDS (or, for more than kLdsChunks, in the
// workspace), a radix selection of the k-th largest key in three digits, and the
// pairs (place that becomes free below k, kept chunk from k on) in ascending
// order.  One launch moves: a workgroup per view and 64-byte strip of the rows of
// K and of V (and one for the weights and scales) first fills the free places,
// whose sources and destinations do not meet, then shifts the rows behind the
// chunks down, a tile of rows read before any of it is written.  A strip belongs
// to one workgroup, so in-place moves need no order between workgroups.
#include "cache.h"
#include "common.h"

namespace catekv {

constexpr int kEvictThreads = 1024;
constexpr int kEvictWaves = kEvictThreads / 64;
constexpr int kLdsChunks = 32768;       // 128 KB of keys
constexpr int kBins = 2048;             // 11-bit digits: 11 + 11 + 10
constexpr int kMoveThreads = 512;

struct EvictInfo {
  int32_t moves;                        // pairs; the view is left alone if shift is 0
  int32_t nc, k, len;
  int32_t shift;                        // rows dropped
};

// Workspace: infos, then the pairs of every view, then (long views) its keys.
static size_t info_bytes(int n_views) { return ((size_t)n_views * sizeof(EvictInfo) + 255) & ~(size_t)255; }
static int64_t max_chunks_of(int64_t max_rows, int cs) { return max_rows / cs; }
// at most half of the chunks can change places: min(k, nc - k)
static int64_t max_moves_of(int64_t chunks) { return chunks / 2 + 1; }
static size_t pairs_bytes(int n_views, int64_t chunks) {
  return ((size_t)n_views * (size_t)max_moves_of(chunks) * 2 * sizeof(int32_t) + 255) & ~(size_t)255;
}
size_t evict_workspace_bytes(int n_views, int64_t max_rows, int cs) {
  const int64_t chunks = max_chunks_of(max_rows, cs);
  const size_t keys = chunks > kLdsChunks ? (size_t)n_views * (size_t)chunks * sizeof(uint32_t) : 0;
  return info_bytes(n_views) + pairs_bytes(n_views, chunks) + ((keys + 255) & ~(size_t)255);
}

// Larger key = larger weight; NaN above all, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float x) {
  uint32_t b = __float_as_uint(x);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (b == 0x80000000u) b = 0;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __builtin_amdgcn_ds_bpermute(((int)__lane_id() ^ o) << 2, x);
  return x;
}

struct SelectShared {
  uint32_t hist[kBins];
  int part[kEvictWaves];
  int part2[kEvictWaves];
  uint32_t digit;
  int above;                            // keys above the chosen digit's bin
};

// The digit that holds the `want`-th largest of the histogram, and how many lie
// above it.  Every thread calls it.
__device__ __forceinline__ void find_digit(SelectShared& s, int want, uint32_t& digit, int& above) {
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
  } else if (before + h0 < want && want <= before + h0 + h1) {
    s.digit = (uint32_t)(kBins - 2 - 2 * t);
    s.above = before + h0;
  }
  __syncthreads();
  digit = s.digit;
  above = s.above;
}

// Selection over nc keys of which k < nc stay; writes the pairs, returns their number.
template <typename Keys>
__device__ __forceinline__ int select_pairs(SelectShared& s, Keys key, int nc, int k, int32_t* pairs) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t prefix = 0;
  int want = k;
  if (k > 0) {
    const int shifts[3] = {21, 10, 0};
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      const int sh = shifts[p], bits = p == 2 ? 10 : 11;
      __syncthreads();
      s.hist[t] = 0;
      s.hist[t + kEvictThreads] = 0;
      __syncthreads();
      for (int c = t; c < nc; c += kEvictThreads) {
        const uint32_t x = key(c);
        if (p == 0 || (x >> (sh + bits)) == (prefix >> (sh + bits)))
          atomicAdd(&s.hist[(x >> sh) & ((1u << bits) - 1)], 1u);
      }
      __syncthreads();
      uint32_t digit;
      int above;
      find_digit(s, want, digit, above);
      prefix |= digit << sh;
      want -= above;
    }
  } else {
    prefix = 0xffffffffu;
    want = 0;                            // nothing stays: no key above, no tie taken
  }
  // keys above prefix stay, and the first `want` equal ones.  Wave w owns a run of
  // chunks, 64 at a time in order.
  const int run = (nc + kEvictThreads - 1) / kEvictThreads * 64;
  const int lo = wave * run, hi = min(nc, lo + run);
  int ties = 0;
  for (int c0 = lo; c0 < hi; c0 += 64) {
    const int c = c0 + lane;
    ties += __popcll(__builtin_amdgcn_ballot_w64(c < hi && key(c) == prefix));
  }
  __syncthreads();
  if (lane == 0) s.part[wave] = ties;
  __syncthreads();
  int tie0 = 0;
  for (int w = 0; w < wave; ++w) tie0 += s.part[w];
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0;
  auto classify = [&](int c, int& tie, bool& stays) {
    const uint32_t x = c < hi ? key(c) : 0;
    const uint64_t eq = __builtin_amdgcn_ballot_w64(c < hi && x == prefix);
    stays = c < hi && (x > prefix || (x == prefix && tie + __popcll(eq & below) < want));
    tie += __popcll(eq);
  };
  int holes = 0, movers = 0, tie = tie0;
  for (int c0 = lo; c0 < hi; c0 += 64) {
    const int c = c0 + lane;
    bool stays;
    classify(c, tie, stays);
    holes += __popcll(__builtin_amdgcn_ballot_w64(c < hi && !stays && c < k));
    movers += __popcll(__builtin_amdgcn_ballot_w64(stays && c >= k));
  }
  __syncthreads();
  if (lane == 0) {
    s.part[wave] = holes;
    s.part2[wave] = movers;
  }
  __syncthreads();
  int total = 0, h = 0, m = 0;
  for (int w = 0; w < kEvictWaves; ++w) {
    if (w == wave) {
      h = total;
    }
    total += s.part[w];
  }
  for (int w = 0; w < wave; ++w) m += s.part2[w];
  tie = tie0;
  for (int c0 = lo; c0 < hi; c0 += 64) {
    const int c = c0 + lane;
    bool stays;
    classify(c, tie, stays);
    const bool hole = c < hi && !stays && c < k, mover = stays && c >= k;
    const uint64_t hm = __builtin_amdgcn_ballot_w64(hole), mm = __builtin_amdgcn_ballot_w64(mover);
    if (hole) pairs[2 * (h + __popcll(hm & below))] = c;
    if (mover) pairs[2 * (m + __popcll(mm & below)) + 1] = c;
    h += __popcll(hm);
    m += __popcll(mm);
  }
  return total;
}

__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(EvictArgs a, EvictInfo* infos, int32_t* pairs,
                                                                     uint32_t* keys, int64_t max_chunks,
                                                                     int64_t max_moves) {
  extern __shared__ uint32_t s_keys[];
  __shared__ SelectShared s;
  const int bh = blockIdx.x, t = threadIdx.x;
  const int64_t len = a.lens[bh];
  const int budget = a.budget[bh];
  const int64_t eligible = len - a.recent > 0 ? len - a.recent : 0;
  const int nc = (int)(eligible / a.cs);
  const bool alone = len < 0 || len > a.max_rows || budget < 0 || nc <= budget;
  __syncthreads();                       // the length is read before it is replaced
  if (alone) {
    if (t == 0) infos[bh] = EvictInfo{0, 0, 0, 0, 0};
    return;
  }
  const int k = budget, cs = a.cs;
  const float* acc = a.acc[bh];
  const bool in_lds = nc <= kLdsChunks;
  uint32_t* mine = in_lds ? nullptr : keys + (size_t)bh * max_chunks;
  for (int c = t; c < nc; c += kEvictThreads) {
    const float* p = acc + (size_t)c * cs;
    uint32_t x = 0;
    for (int i = 0; i < cs; ++i) x = max(x, weight_key(p[i]));
    if (in_lds) s_keys[c] = x;
    else mine[c] = x;
  }
  __syncthreads();
  int32_t* out = pairs + (size_t)bh * max_moves * 2;
  const int moves = in_lds ? select_pairs(s, [&](int c) { return s_keys[c]; }, nc, k, out)
                           : select_pairs(s, [&](int c) { return mine[c]; }, nc, k, out);
  if (t == 0) {
    const int shift = (nc - k) * cs;
    infos[bh] = EvictInfo{moves, nc, k, (int32_t)len, shift};
    a.lens[bh] = len - shift;
  }
}

// Rows [0, n) of a strip: row i from src(i) to dst(i), each row `pieces` 16-byte
// pieces wide at a stride of `pitch` bytes.  All rows of a tile are read before
// one is written; a tile's destinations lie below the sources of the next.
constexpr int kMoveBatch = 8;

template <typename Src, typename Dst>
__device__ __forceinline__ void move_rows(char* base, size_t pitch, int pieces_log, int64_t n, bool apart, Src src, Dst dst) {
  const int piece = threadIdx.x & ((1 << pieces_log) - 1);
  const int64_t row = threadIdx.x >> pieces_log, step = kMoveThreads >> pieces_log;
  for (int64_t i0 = 0; i0 < n; i0 += step * kMoveBatch) {
    uint4 w[kMoveBatch];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int64_t i = i0 + u * step + row;
      if (i < n) w[u] = ldg16(base + (size_t)src(i) * pitch + piece * 16);
    }
    if (!apart) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int64_t i = i0 + u * step + row;
      if (i < n) *reinterpret_cast<uint4*>(base + (size_t)dst(i) * pitch + piece * 16) = w[u];
    }
  }
}

template <typename Src, typename Dst>
__device__ __forceinline__ void move_floats(float* p, int64_t n, bool apart, Src src, Dst dst) {
  for (int64_t i0 = 0; i0 < n; i0 += (int64_t)kMoveThreads * kMoveBatch) {
    float w[kMoveBatch];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int64_t i = i0 + u * kMoveThreads + threadIdx.x;
      w[u] = i < n ? p[src(i)] : 0.f;
    }
    if (!apart) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int64_t i = i0 + u * kMoveThreads + threadIdx.x;
      if (i < n) p[dst(i)] = w[u];
    }
  }
}

// blockIdx.x: view; blockIdx.y: strips of K, strips of V, then the weights (and scales).
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, const EvictInfo* infos,
                                                                  const int32_t* pairs, int64_t max_moves) {
  const int bh = blockIdx.x, cs = a.cs;
  const EvictInfo f = infos[bh];
  if (f.shift == 0) return;
  const int32_t* pr = pairs + (size_t)bh * max_moves * 2;
  const int64_t filled = (int64_t)f.moves * cs, at = (int64_t)f.k * cs, from = (int64_t)f.nc * cs;
  const int strips = a.row_bytes / 64;
  // row i of the fill: pair i / cs, row i % cs of its chunk
  auto fill_src = [&](int64_t i) { const int p = (int)(i / cs); return (int64_t)pr[2 * p + 1] * cs + (i - (int64_t)p * cs); };
  auto fill_dst = [&](int64_t i) { const int p = (int)(i / cs); return (int64_t)pr[2 * p] * cs + (i - (int64_t)p * cs); };
  auto rest_src = [&](int64_t i) { return from + i; };
  auto rest_dst = [&](int64_t i) { return at + i; };
  if ((int)blockIdx.y < 2 * strips) {
    const bool is_v = (int)blockIdx.y >= strips;
    const int strip = is_v ? blockIdx.y - strips : blockIdx.y;
    char* base;
    int64_t rest;
    if (a.q8) {
      base = reinterpret_cast<char*>(is_v ? a.q8[bh].v : a.q8[bh].k);
      rest = (int64_t)(f.len / a.block) * a.block - from;     // the codes behind the chunks
    } else {
      base = reinterpret_cast<char*>(const_cast<void*>(is_v ? a.kv[bh].v : a.kv[bh].k));
      rest = f.len - from;
    }
    base += strip * 64;
    move_rows(base, a.row_bytes, 2, filled, true, fill_src, fill_dst);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    move_rows(base, a.row_bytes, 2, rest, false, rest_src, rest_dst);
    return;
  }
  float* acc = a.acc[bh];
  const int64_t rest = f.len - from;
  move_floats(acc, filled, true, fill_src, fill_dst);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  move_floats(acc, rest, false, rest_src, rest_dst);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  for (int64_t i = f.len - f.shift + threadIdx.x; i < f.len; i += kMoveThreads) acc[i] = 0.f;
  if (a.q8) {
    const int per = cs / a.block;        // blocks of a chunk
    auto src = [&](int64_t i) { const int p = (int)(i / per); return (int64_t)pr[2 * p + 1] * per + (i - (int64_t)p * per); };
    auto dst = [&](int64_t i) { const int p = (int)(i / per); return (int64_t)pr[2 * p] * per + (i - (int64_t)p * per); };
    const int64_t n = (int64_t)f.moves * per, left = f.len / a.block - (int64_t)f.nc * per;
#pragma unroll 1
    for (int v = 0; v < 2; ++v) {
      float* p = v ? a.q8[bh].v_scale : a.q8[bh].k_scale;
      move_floats(p, n, true, src, dst);
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      move_floats(p, left, false, [&](int64_t i) { return (int64_t)f.nc * per + i; },
                  [&](int64_t i) { return (int64_t)f.k * per + i; });
    }
  }
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t stream) {
  const int64_t chunks = max_chunks_of(a.max_rows, a.cs), moves = max_moves_of(chunks);
  char* w = reinterpret_cast<char*>(a.ws);
  EvictInfo* infos = reinterpret_cast<EvictInfo*>(w);
  int32_t* pairs = reinterpret_cast<int32_t*>(w + info_bytes(a.n_views));
  uint32_t* keys = reinterpret_cast<uint32_t*>(w + info_bytes(a.n_views) + pairs_bytes(a.n_views, chunks));
  const size_t lds = (size_t)(chunks < kLdsChunks ? chunks : kLdsChunks) * sizeof(uint32_t);
  hipLaunchKernelGGL(evict_select_kernel, dim3(a.n_views), dim3(kEvictThreads), lds, stream, a, infos, pairs, keys,
                     chunks, moves);
  hipLaunchKernelGGL(evict_move_kernel, dim3(a.n_views, 2 * (a.row_bytes / 64) + 1), dim3(kMoveThreads), 0, stream, a,
                     infos, pairs, moves);
  return hipGetLastError();
}

}  // namespace catekv
