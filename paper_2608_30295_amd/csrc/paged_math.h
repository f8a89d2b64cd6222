// What the attention kernels over pages share (gfx950).
#pragma once

#include "common.h"
#include "paged.h"

namespace catekv {

typedef float pg_f32x2 __attribute__((ext_vector_type(2)));
typedef float pg_f32x4 __attribute__((ext_vector_type(4)));
typedef float pg_f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 pg_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 pg_bf16x8 __attribute__((ext_vector_type(8)));
typedef short pg_s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short pg_u16x2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.6931471805599453f;

// A row's weights are exp2(s c - m c), m c rounded once: off by a factor 2^(|m c| 2^-24)
// that all of them share and that their sum takes out again.  From |m c| = 2^29 on that
// could overflow, but there scores that differ do so by 32 and more (a step of fp32), and
// any factor c' from c / 2 on gives weights of 1 and next to 0: with a power of two m c'
// and s c' are exact, and equal scores of any size weigh the same.
__device__ __forceinline__ float pg_factor(float m, float c) {
  return fabsf(m) * c < 536870912.f || m == -INFINITY ? c : __uint_as_float(__float_as_uint(c) & 0x7f800000u);
}

// A row's maximum as results and partial slots take it.  -inf stands for a row without
// scores above -inf, whose sum is 0; where all scores are NaN the maximum stays at -inf, too,
// but the sum is NaN and has to come through.
__device__ __forceinline__ float pg_top(float m, float l) { return m > -INFINITY ? m : l != l ? 0.f : -INFINITY; }

// What a part of maximum m counts for beside the largest maximum M, f = pg_factor(M, c).  The
// products are rounded each, as those that the parts' weights refer to are; scores that differ
// must not meet in them, so that maxima stay unscaled until here.
__device__ __forceinline__ float pg_share(float m, float M, float f) {
#pragma clang fp contract(off)
  return m == -INFINITY ? 0.f : fast_exp2(m * f - M * f);
}

// The log-sum-exp of a row of maximum M and sum l.
__device__ __forceinline__ float pg_lse(float M, float l, float c) {
#pragma clang fp contract(off)
  return M == -INFINITY ? -INFINITY : (M * c + __builtin_amdgcn_logf(l)) * kLn2;
}

// bf16 pair (to nearest, ties to even) of two fp32 values, x in the low half.
__device__ __forceinline__ uint32_t pg_pack2(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((pg_f32x2{x, y}), pg_bf16x2));
}
__device__ __forceinline__ void pg_put4(uint16_t*, char* p, float a, float b, float c, float d) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pg_pack2(a, b), pg_pack2(c, d));
}
__device__ __forceinline__ void pg_put4(float*, char* p, float a, float b, float c, float d) {
  *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}

// fp32 queries are scaled on their way in (one rounding of 2^-24 more; a product q k
// that only fits fp32 with the scale in it does); bf16 ones enter their products as they
// are, and the scores are scaled.
__device__ __forceinline__ uint4 pg_scale_q(const float*, uint4 q, float scale) {
  return make_uint4(__float_as_uint(__uint_as_float(q.x) * scale), __float_as_uint(__uint_as_float(q.y) * scale),
                    __float_as_uint(__uint_as_float(q.z) * scale), __float_as_uint(__uint_as_float(q.w) * scale));
}
__device__ __forceinline__ uint4 pg_scale_q(const uint16_t*, uint4 q, float) { return q; }

// Rows of a view as attention takes them: none if its length is out of range, and
// no more than were planned for.
__device__ __forceinline__ int pg_rows(const PagedCache& c, int64_t len, int max_rows) {
  const int64_t cap = (int64_t)c.max_pages << c.page_log;
  return len < 0 || len > cap ? 0 : (int)min(len, (int64_t)max_rows);
}
__device__ __forceinline__ size_t pg_page(const PagedCache& c, int id) {
  return (size_t)((uint32_t)id < (uint32_t)c.n_pages ? id : 0) << c.page_log;
}

// A value that is the same for all lanes, and that no one writes meanwhile, through the scalar
// cache: its wait is its own, and not one for every vector load and store issued before it.
template <typename T>
__device__ __forceinline__ T pg_scalar(const T* p) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
  struct Words { int32_t w[sizeof(T) / 4]; } x;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i)
    x.w[i] = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>((uint64_t)hi << 32 | lo)[i];
  return __builtin_bit_cast(T, x);
}
__device__ __forceinline__ int pg_entry(const int32_t* ids, int p) { return pg_scalar(ids + p); }

// ---- V that is not finite: the exponent's bits all ones ----------------------------
__device__ __forceinline__ bool pg_bad16(uint32_t x) { return (x & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ uint32_t pg_clean16(uint32_t x) { return pg_bad16(x) ? 0u : x; }
// f of both halves of a word
template <class F>
__device__ __forceinline__ uint32_t pg_both(uint32_t w, F f) { return f(w & 0xffffu) | (uint32_t)f(w >> 16) << 16; }
__device__ __forceinline__ bool pg_bad32(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ void pg_pair(const uint16_t* p, float& x, float& y) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  x = bf16_lo(w);
  y = bf16_hi(w);
}
__device__ __forceinline__ void pg_pair(const float* p, float& x, float& y) {
  const float2 w = *reinterpret_cast<const float2*>(p);
  x = w.x;
  y = w.y;
}
__device__ __forceinline__ void pg_store(uint16_t* p, float x) { *p = (uint16_t)pg_pack2(x, 0.f); }
__device__ __forceinline__ void pg_store(float* p, float x) { *p = x; }

// An infinite V in a row of finite score is infinite in the result, whatever the row's weight:
// next to a score 150 powers of two higher its fp32 weight is 0, and 0 inf NaN.  Sums that
// turned out not to be finite are therefore taken from V itself, once a piece's results are
// stored, and where parts are joined such a value is not scaled.

// Whether any of n sums (n even) is not finite (or any two have a product that is not).
template <int N>
__device__ __forceinline__ bool pg_unusual(const float (&o)[N]) {
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < N; i += 2) t = __builtin_fmaf(o[i], o[i + 1], t);
  return pg_bad32(t);
}

// Whether the score of a new row (a lane's own) and a cached one (the same for all lanes) is -inf.
// fp32 queries are scaled first, as they are for the products.
__device__ __forceinline__ float pg_dot(const uint16_t*, float s, uint32_t q, uint32_t k, float) {
  return __builtin_fmaf(bf16_hi(q), bf16_hi(k), __builtin_fmaf(bf16_lo(q), bf16_lo(k), s));
}
__device__ __forceinline__ float pg_dot(const float*, float s, uint32_t q, uint32_t k, float scale) {
  return __builtin_fmaf(__uint_as_float(q) * scale, __uint_as_float(k), s);
}
template <typename T>
__device__ __forceinline__ bool pg_struck(const T* q, const T* k, float scale) {
  float s = 0.f;
#pragma unroll 4
  for (int i = 0; i < kD * (int)sizeof(T) / 16; ++i) {
    const uint4 x = ld16(q + i * 16 / sizeof(T)), y = ld16(k + i * 16 / sizeof(T));
    s = pg_dot((const T*)nullptr, s, x.x, y.x, scale);
    s = pg_dot((const T*)nullptr, s, x.y, y.y, scale);
    s = pg_dot((const T*)nullptr, s, x.z, y.z, scale);
    s = pg_dot((const T*)nullptr, s, x.w, y.w, scale);
  }
  return s == -INFINITY;
}

// What V holds of a dim that is not finite, as bits of new rows.
struct OddDim {
  uint32_t up = 0, down = 0, nan = 0;                  // inf, -inf, NaN
  __device__ __forceinline__ void add(float x, uint32_t sees, uint32_t struck) {
    const uint32_t n = x != x ? sees : x == INFINITY || x == -INFINITY ? sees & struck : 0;
    nan |= n;
    up |= x == INFINITY ? sees & ~struck : 0;
    down |= x == -INFINITY ? sees & ~struck : 0;
  }
  template <typename E>
  __device__ __forceinline__ void put(E* p, int r) const {
    const bool u = up >> r & 1, d = down >> r & 1, n = nan >> r & 1;
    if (u || d || n) pg_store(p, n || (u && d) ? __builtin_nanf("") : u ? INFINITY : -INFINITY);
  }
};

// The results of up to 32 new rows of a wave, where V of the cached rows [t0, t1) that they see
// is not finite: the infinity that there is alone, or NaN.  A row without weight, of a score of
// -inf, makes NaN of an infinity.  New row row0 + r, r < n, of a sequence's n_rows in a view sees
// see0 + (row0 + r) / G rows; its query is row q_row(row0 + r) of q, its result lies at slot + r *
// 128 or, without slots, at that row of out, where it stays if bit r of `skip` is set.
// Once the results are stored, in their place: the kernels' registers are all in use before.
struct RestoreAt {
  int32_t t0, t1, see0, row0, n, n_rows, skip, hq;
  size_t q0;                                           // of the sequence's first token and the group's first head
  float* slot;
};
template <typename T, int G>
__device__ __forceinline__ void pg_restore(const PagedCache& c, int view, const char* q, float scale, char* out, const RestoreAt& at) {
  constexpr int AHEAD = 8;                             // cached rows at a time (a page holds whole sixteens); 16: the same
  const int32_t* ids = c.table + (size_t)view * c.max_pages;
  const int lane = __lane_id(), mask = (1 << c.page_log) - 1;
  const int own = min(at.row0 + min(lane & 31, at.n - 1), at.n_rows - 1), see = at.see0 + own / G;
  auto q_row = [&](int r) { return at.q0 + (size_t)(r / G) * at.hq + r % G; };
  const T* mine = reinterpret_cast<const T*>(q) + q_row(own) * kD;
  OddDim a, b;                                         // dims 2 lane and 2 lane + 1
#pragma unroll 1
  for (int t = at.t0; t < at.t1; t += AHEAD) {
    const size_t row = pg_page(c, pg_entry(ids, min(t >> c.page_log, c.max_pages - 1))) + (t & mask);
    const T* from = reinterpret_cast<const T*>(c.v) + row * kD + 2 * lane;
    float x[AHEAD], y[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) pg_pair(from + i * kD, x[i], y[i]);
    bool odd = false;                                  // where NaN is known for all rows, nothing changes
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) odd = odd || (pg_bad32(x[i]) && ~a.nan) || (pg_bad32(y[i]) && ~b.nan);
    if (!__builtin_amdgcn_ballot_w64(odd)) continue;
#pragma unroll 1
    for (int i = 0; i < min(AHEAD, at.t1 - t); ++i) {
      float u, v;
      pg_pair(from + i * kD, u, v);
      const uint32_t sees = (uint32_t)__builtin_amdgcn_ballot_w64(t + i < see);
      uint32_t struck = 0;
      if (__builtin_amdgcn_ballot_w64(u == INFINITY || u == -INFINITY || v == INFINITY || v == -INFINITY))
        struck = (uint32_t)__builtin_amdgcn_ballot_w64(pg_struck(mine, reinterpret_cast<const T*>(c.k) + (row + i) * kD, scale));
      a.add(u, sees, struck);
      b.add(v, sees, struck);
    }
  }
  __builtin_amdgcn_s_waitcnt(0);                       // the results lie where they belong
#pragma unroll 1
  for (int r = 0; r < at.n && at.row0 + r < at.n_rows; ++r) {
    if (at.slot) {
      a.put(at.slot + r * kD + 2 * lane, r);
      b.put(at.slot + r * kD + 2 * lane + 1, r);
    } else if (!(at.skip >> r & 1)) {
      T* to = reinterpret_cast<T*>(out) + q_row(at.row0 + r) * kD + 2 * lane;
      a.put(to, r);
      b.put(to + 1, r);
    }
  }
}

}  // namespace catekv
