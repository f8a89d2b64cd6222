// Attention of few new tokens (up to 16 rows: tokens x heads of a group) over caches
// in pages (gfx950): bound by reading K and V once.
//
// All views are laid end to end and cut into equal shares, one per workgroup of 8
// waves, one workgroup per compute unit (fewer beside chunks, in their launch).  A wave
// streams tiles of 16 cached rows (a page holds whole ones) through two stages of registers,
// also from one segment into the next; the page number of the tile after the next is on its
// way meanwhile.
// Scores are S^T = K Q^T: lane l holds row l % 16 of the new ones and cached rows
// 4 (l / 16) + i, which is how O^T = V^T P^T takes P; what belongs to a new row
// (maximum, sum, factor) is a lane's own.  V^T's rows are the 8 dims that a lane
// loaded of each cached row, one product per dim.
//
// bf16, 3 views of 131072 rows and 5 of 2112, 4 heads a group: 207 MB in 37 us, 5.6 TB/s with
// the start; 64 sequences: 553 MB in 95 us, 5.8 TB/s.  fp32, 8 views of 65536 rows: 537 MB in 102 us,
// 5.3 TB/s; 64 sequences 1108 MB in 210, the same: with 256 registers in use, 15 to 27 spilled, most in
// the last tiles of a segment, and a quarter of the cycles in its fp32 products.  A
// compute unit takes 22 GB/s with all of them at work and 23 to 28 with a third: all are given a share, but for those
// that a batch's chunks keep.
#pragma once

#include <type_traits>

#include "paged_math.h"

namespace catekv {
namespace {

constexpr int kStreamWaves = 8;
constexpr int kStreamThreads = kStreamWaves * 64;
constexpr int R = kStreamRows;
constexpr int kStreamTile = 16;
constexpr int kPad = kD + 4;

template <typename T> struct Ops;

template <> struct Ops<uint16_t> {
  static constexpr int kK = 4, kV = 4;    // 16-byte registers of a tile, K and V each
  static __device__ __forceinline__ int v_chunk(int, int n16) { return n16; }
  static constexpr int kVPer = 1;         // registers per cached row of V
  static __device__ __forceinline__ pg_f32x4 score(const uint4 (&k)[kK], const uint4 (&q)[kK]) {
    pg_f32x4 s = {};
#pragma unroll
    for (int i = 0; i < kK; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pg_bf16x8, k[i]), __builtin_bit_cast(pg_bf16x8, q[i]), s, 0, 0, 0);
    return s;
  }
  // element e of the four rows
  static __device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
  static __device__ __forceinline__ uint2 column(const uint4 (&v)[kV], int e) {
    const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
    return make_uint2(__builtin_amdgcn_perm(word(v[1], e / 2), word(v[0], e / 2), sel),
                      __builtin_amdgcn_perm(word(v[3], e / 2), word(v[2], e / 2), sel));
  }
  static __device__ __forceinline__ pg_f32x4 mul(uint2 v, uint2 p, pg_f32x4 o) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(pg_s16x4, v), __builtin_bit_cast(pg_s16x4, p), o, 0, 0, 0);
  }
  // the weights in two parts, 16 bits of them in all: p = hi + lo
  static __device__ __forceinline__ void split(const pg_f32x4& p, uint2& hi, uint2& lo) {
    hi = make_uint2(pg_pack2(p[0], p[1]), pg_pack2(p[2], p[3]));
    lo = make_uint2(pg_pack2(p[0] - bf16_lo(hi.x), p[1] - bf16_hi(hi.x)), pg_pack2(p[2] - bf16_lo(hi.y), p[3] - bf16_hi(hi.y)));
  }
  static __device__ __forceinline__ void pv(const uint4 (&v)[kV], const pg_f32x4& p, pg_f32x4 (&o)[8]) {
    uint2 hi, lo;
    split(p, hi, lo);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint2 c = column(v, e);
      o[e] = mul(c, lo, mul(c, hi, o[e]));
    }
  }
  static __device__ __forceinline__ bool any_bad(const uint4 (&v)[kV]) {
    pg_u16x2 top = {0, 0};                // the largest magnitude, as bits
#pragma unroll
    for (int r = 0; r < kV; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(pg_u16x2, word(v[r], i) & 0x7fff7fffu));
    return top[0] >= 0x7f80 || top[1] >= 0x7f80;
  }
  static __device__ __forceinline__ uint4 clean(const uint4& v) {
    return make_uint4(pg_both(v.x, pg_clean16), pg_both(v.y, pg_clean16), pg_both(v.z, pg_clean16), pg_both(v.w, pg_clean16));
  }
  // dims [d, d + 4) of a row
  static __device__ __forceinline__ float4 four(const char* row, int d) {
    const uint2 x = *reinterpret_cast<const uint2*>(row + d * 2);
    return make_float4(bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y));
  }
  // dims of o[4 x .. 4 x + 3][i]
  static __device__ __forceinline__ int dim(int x, int k4, int i) { return 8 * (4 * k4 + i) + 4 * x; }
};

template <> struct Ops<float> {
  static constexpr int kK = 8, kV = 8;
  static constexpr int kVPer = 2;
  static __device__ __forceinline__ int v_chunk(int x, int n16) { return n16 + 16 * x; }
  static __device__ __forceinline__ float el(const uint4& v, int i) {
    return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
  }
  static __device__ __forceinline__ pg_f32x4 score(const uint4 (&k)[kK], const uint4 (&q)[kK]) {
    pg_f32x4 s = {};
#pragma unroll
    for (int i = 0; i < kK; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(el(k[i], e), el(q[i], e), s, 0, 0, 0);
    return s;
  }
  static __device__ __forceinline__ void pv(const uint4 (&v)[kV], const pg_f32x4& p, pg_f32x4 (&o)[8]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(el(v[2 * r + e / 4], e & 3), p[r], o[e], 0, 0, 0);
  }
  static __device__ __forceinline__ bool any_bad(const uint4 (&v)[kV]) {
    bool b = false;
#pragma unroll
    for (int r = 0; r < kV; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) b = b || pg_bad32(el(v[r], i));
    return b;
  }
  static __device__ __forceinline__ uint4 clean(const uint4& v) {
    return make_uint4(pg_bad32(el(v, 0)) ? 0u : v.x, pg_bad32(el(v, 1)) ? 0u : v.y, pg_bad32(el(v, 2)) ? 0u : v.z,
                      pg_bad32(el(v, 3)) ? 0u : v.w);
  }
  static __device__ __forceinline__ float4 four(const char* row, int d) { return *reinterpret_cast<const float4*>(row + d * 4); }
  static __device__ __forceinline__ int dim(int x, int k4, int i) { return 4 * (4 * k4 + i) + 64 * x; }
};

// A segment as the waves read it.
struct Seg {
  int32_t view, t0, t_end, n_units;
  int32_t see0;                           // cached rows that the first new token sees
  int32_t rows;                           // new rows
  int32_t q0;                             // their first (token, head) row: tok0 * hq + head * G
  int32_t slot;
};

// What a workgroup needs of LDS: kBatch segments, described at a time, and the waves' sums.
template <typename T, int kBatch>
struct StreamLds {
  Seg (*seg)[kBatch];
  uint4 (*q)[kBatch][R][kD * sizeof(T) / 16];
  float (*o)[kStreamWaves][R][kPad];
  float (*m)[kStreamWaves][R], (*l)[kStreamWaves][R];
};

constexpr int kOwnRows = R / kStreamWaves;    // of a segment's results, that a wave writes
// pg_restore() as a function by itself: inlined here, one fp32 token over 65536 rows took 115 to
// 125 us for 105, with registers that the kernel then has to spill.
template <typename T, int G>
__device__ __attribute__((noinline)) void stream_restore(char* k, char* v, int32_t* ids, int n_pages, int page_log, const char* q, float scale,
                                                         char* out, int t0, int t1, int see0, int row0, int n_rows, int skip, int hq, int q0,
                                                         float* slot) {
  PagedCache c{};
  c.k = k;
  c.v = v;
  c.table = ids;
  c.n_pages = n_pages;
  c.page_log = page_log;
  c.max_pages = INT32_MAX;                    // the rows are the view's
  pg_restore<T, G>(c, 0, q, scale, out, {t0, t1, see0, row0, kOwnRows, n_rows, skip, hq, (size_t)q0, slot});
}

// A workgroup's share: segments [first, last).
template <typename T, int G, int kBatch>
__device__ __forceinline__ void stream_share(const PagedAttn& a, const PagedPiece* pieces, int first, int last,
                                             const StreamLds<T, kBatch>& lds) {
  using X = Ops<T>;
  constexpr int RB = kD * (int)sizeof(T);
  auto& s_seg = *lds.seg;
  auto& s_q = *lds.q;
  auto& s_o = *lds.o;
  auto& s_m = *lds.m;
  auto& s_l = *lds.l;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, k4 = lane >> 4;
  const float cs = a.log2_scale, thr = a.rise;
  const int mask = (1 << c.page_log) - 1;

  for (int s0 = first; s0 < last; s0 += kBatch) {
    const int nseg = min(last - s0, kBatch);
    __syncthreads();                                  // the batch before is done
    if ((int)threadIdx.x < nseg) {
      const PagedPiece p = pieces[s0 + threadIdx.x];
      const int L = pg_rows(c, c.lens[p.view], p.max_rows);
      Seg s;
      s.view = p.view;
      s.t0 = p.t0;
      s.t_end = min(p.t1, L);
      s.n_units = s.t_end > p.t0 ? (s.t_end - p.t0 + kStreamTile - 1) / kStreamTile : 0;
      s.see0 = L - p.n_new + 1;
      s.rows = p.n_new * G;
      s.q0 = p.tok0 * a.hq + (p.view % c.hkv) * G;
      s.slot = p.slot;
      s_seg[threadIdx.x] = s;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < nseg * R * (RB / 16); i += kStreamThreads) {
      const int sg = i / (R * (RB / 16)), x = i - sg * (R * (RB / 16)), r = x / (RB / 16), ch = x - r * (RB / 16);
      const int tok = r / G;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < s_seg[sg].rows) v = ldg16(a.q + ((size_t)s_seg[sg].q0 + (size_t)tok * a.hq + (r - tok * G)) * RB + ch * 16);
      v = pg_scale_q((const T*)nullptr, v, a.scale);
      s_q[sg][r][ch] = v;
    }
    __syncthreads();

    // ---- this wave's tiles: those of number wave, wave + 8, ... of every segment ----
    int is = 0, iu = wave;                            // next tile to load
    auto skip = [&]() __attribute__((always_inline)) {
      while (is < nseg && iu >= s_seg[is].n_units) {
        ++is;
        iu = wave;
      }
    };
    skip();
    int next_id = 0;
    auto fetch_id = [&]() __attribute__((always_inline)) {                           // the page number of that tile
      if (is < nseg) {
        const int t = s_seg[is].t0 + iu * kStreamTile;
        next_id = pg_entry(c.table + (size_t)s_seg[is].view * c.max_pages, t >> c.page_log);
      }
    };
    fetch_id();
    uint4 kb[2][X::kK], vb[2][X::kV];
    int seg_of[2] = {0, 0}, tile_of[2] = {0, 0};
    auto issue = [&](auto tag) __attribute__((always_inline)) {                      // the next tile; there is one
      constexpr int B = decltype(tag)::value;
      const int tile = s_seg[is].t0 + iu * kStreamTile, rows = s_seg[is].t_end - tile;   // at least one row
      const size_t base = (pg_page(c, next_id) + (tile & mask)) * RB;
      const char* kr = c.k + base + (size_t)min(n16, rows - 1) * RB + k4 * 16;
#pragma unroll
      for (int i = 0; i < X::kK; ++i) kb[B][i] = once16(kr + i * 64);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* vr = c.v + base + (size_t)min(4 * k4 + r, rows - 1) * RB;
#pragma unroll
        for (int x = 0; x < X::kVPer; ++x) vb[B][r * X::kVPer + x] = once16(vr + X::v_chunk(x, n16) * 16);
      }
      seg_of[B] = is;
      tile_of[B] = tile;
      iu += kStreamWaves;
      skip();
      fetch_id();
    };

    uint4 q[X::kK];
    pg_f32x4 o[8];
    float m, l;
    float cw;                                         // of the weights: pg_factor()
    bool purged;                                      // a tile of the segment, in the wave
    int odd = 0, kept = 0;                            // bits of segments: results to be taken from V, and rows that are not
    int cur = 0;
    auto begin = [&]() __attribute__((always_inline)) {
      m = -INFINITY;
      l = 0.f;
      cw = cs;
      purged = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = pg_f32x4{};
      if (sizeof(T) == 2)
#pragma unroll
        for (int i = 0; i < X::kK; ++i) q[i] = s_q[cur][n16][i * 4 + k4];
    };
    auto consume = [&](auto tag) __attribute__((always_inline)) {
      constexpr int B = decltype(tag)::value;
      const Seg& sg = s_seg[cur];
      const int tile = tile_of[B];
      if (sizeof(T) == 4)                               // registers are few: the new rows come from LDS each time
#pragma unroll
        for (int i = 0; i < X::kK; ++i) q[i] = s_q[cur][n16][i * 4 + k4];
      pg_f32x4 s = X::score(kb[B], q);
      const bool masked = tile + kStreamTile > sg.see0;       // the first token does not see all of it
      const int see = min(sg.see0 + n16 / G, sg.t_end);
      if (masked) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = tile + 4 * k4 + r;
          s[r] = t < see ? s[r] : -INFINITY;
          if (t >= sg.t_end)
#pragma unroll
            for (int x = 0; x < X::kVPer; ++x) vb[B][r * X::kVPer + x] = make_uint4(0, 0, 0, 0);
        }
      }
      // 0 * NaN is NaN: V that is not finite, and that some of the tokens do not see, is left
      // out here and added to the sums of those that do at the segment's end.  In bf16 it is
      // wherever it stands: an infinity times the two parts of a weight is NaN, too.
      if ((sizeof(T) == 2 || (masked && sg.rows > G)) && __builtin_amdgcn_ballot_w64(X::any_bad(vb[B]))) {
        purged = true;
#pragma unroll
        for (int i = 0; i < X::kV; ++i) vb[B][i] = X::clean(vb[B][i]);
      }
      float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      mx = max_xor32(max_xor16(mx));
      if (__builtin_amdgcn_ballot_w64(mx > m && !(mx <= m + thr))) {
        const float corr = mx > m ? fast_exp2((m - mx) * cs) : 1.f;
        m = fmaxf(m, mx);
        cw = pg_factor(m, cs);
        l *= corr;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[e][i] *= corr;
      }
      const float mc = m == -INFINITY ? 0.f : m * cw;
      pg_f32x4 p;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = fast_exp2(__builtin_fmaf(s[r], cw, -mc));
        l += p[r];
      }
      X::pv(vb[B], p, o);
    };
    // The waves' parts of segment cur joined; its result or partial slot written.
    auto finish = [&]() __attribute__((always_inline)) {
      if (purged) {
        const Seg& sg = s_seg[cur];
        const int see = min(sg.see0 + n16 / G, sg.t_end);
#pragma unroll 1
        for (int u = wave; u < sg.n_units; u += kStreamWaves) {
          const int tile = sg.t0 + u * kStreamTile;
          if (sizeof(T) == 4 && tile + kStreamTile <= sg.see0) continue;   // all tokens see it: taken as it was
          const size_t base = (pg_page(c, pg_entry(c.table + (size_t)sg.view * c.max_pages, tile >> c.page_log)) + (tile & mask)) * RB;
#pragma unroll 1
          for (int r = 0; r < min(kStreamTile, sg.t_end - tile); ++r)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float4 z = X::four(c.v + base + (size_t)r * RB, X::dim(x, k4, i));
                const float f[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) o[4 * x + e][i] += tile + r < see && pg_bad32(f[e]) ? f[e] : 0.f;
              }
        }
      }
      l = add_xor32(add_xor16(l));
      barrier_lds_only();                             // the join before has been read
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(&s_o[wave][n16][X::dim(x, k4, i)]) =
              make_float4(o[4 * x][i], o[4 * x + 1][i], o[4 * x + 2][i], o[4 * x + 3][i]);
      if (k4 == 0) {
        s_m[wave][n16] = pg_top(m, l);
        s_l[wave][n16] = l;
      }
      barrier_lds_only();
      const Seg sg = s_seg[cur];
      bool bad = false, keep = false;
      for (int t = threadIdx.x; t < sg.rows * (kD / 4); t += kStreamThreads) {   // one turn at most
        const int r = t / (kD / 4), d = (t - r * (kD / 4)) * 4;
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kStreamWaves; ++w) M = fmaxf(M, s_m[w][r]);
        const float fM = pg_factor(M, cs);
        float sum = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kStreamWaves; ++w) {
          const float mw = s_m[w][r];
          const float f = pg_share(mw, M, fM);
          const float4 v = *reinterpret_cast<const float4*>(&s_o[w][r][d]);
          sum += f * s_l[w][r];
          x[0] += f * v.x;
          x[1] += f * v.y;
          x[2] += f * v.z;
          x[3] += f * v.w;
        }
        const bool none = M == -INFINITY;
        bad = sum == sum && pg_unusual(x);
        keep = none || sum != sum;
        if (sg.slot >= 0) {
          float* slot = a.slots + (size_t)sg.slot * 4;
          *reinterpret_cast<float4*>(slot + r * kD + d) = make_float4(x[0], x[1], x[2], x[3]);
          if (d == 0) {
            slot[R * kD + r] = M;
            slot[R * (kD + 1) + r] = sum;
          }
        } else {
          const float inv = none ? 0.f : 1.f / sum;
          const int tok = r / G;
          const size_t row = (size_t)sg.q0 + (size_t)tok * a.hq + (r - tok * G);
          pg_put4((T*)nullptr, a.out + (row * kD + d) * sizeof(T), none ? 0.f : x[0] * inv, none ? 0.f : x[1] * inv,
                  none ? 0.f : x[2] * inv, none ? 0.f : x[3] * inv);
          if (a.lse && d == 0) a.lse[row] = pg_lse(M, sum, cs);
        }
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(bad) != 0, 0)) {         // half a wave has a row
        const uint64_t k = __builtin_amdgcn_ballot_w64(keep);
        odd |= 1 << cur;
        kept |= (int)((k & 1) | (k >> 31 & 2)) << kOwnRows * cur;
      }
    };
    auto use = [&](auto tag) __attribute__((always_inline)) {
      while (cur < seg_of[decltype(tag)::value]) {
        finish();
        ++cur;
        begin();
      }
      consume(tag);
    };
    using B0 = std::integral_constant<int, 0>;
    using B1 = std::integral_constant<int, 1>;
    int n = 0;
    for (int i = 0; i < nseg; ++i) n += max(0, (s_seg[i].n_units - wave + kStreamWaves - 1) / kStreamWaves);
    n = __builtin_amdgcn_readfirstlane(n);
    begin();
    // Two tiles are on their way at the loop's head, and every turn asks for as many as
    // it uses: a wait for one tile is then never one for the other, too.
    if (n > 0) issue(B0{});
    if (n > 1) issue(B1{});
    for (; n >= 4; n -= 2) {
      use(B0{});
      issue(B0{});
      use(B1{});
      issue(B1{});
    }
    for (; n > 0; --n) {
      use(B0{});
      if (n == 1) break;
#pragma unroll
      for (int i = 0; i < X::kK; ++i) kb[0][i] = kb[1][i];
#pragma unroll
      for (int i = 0; i < X::kV; ++i) vb[0][i] = vb[1][i];
      seg_of[0] = seg_of[1];
      tile_of[0] = tile_of[1];
      if (n == 3) issue(B1{});
    }
    for (;;) {
      finish();
      if (++cur == nseg) break;
      begin();
    }

    for (int i = 0; odd >> i; ++i)                    // results that are not finite
      if (odd >> i & 1) {
        const Seg sg = s_seg[i];
        stream_restore<T, G>(c.k, c.v, c.table + (size_t)sg.view * c.max_pages, c.n_pages, c.page_log, a.q, a.scale, a.out,
                             sg.t0, sg.t_end, sg.see0, wave * kOwnRows, sg.rows, kept >> kOwnRows * i & 3, a.hq, sg.q0,
                             sg.slot >= 0 ? a.slots + (size_t)sg.slot * 4 + wave * kOwnRows * kD : nullptr);
      }
  }
}

}  // namespace
}  // namespace catekv
