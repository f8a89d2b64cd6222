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
__device__ __forceinline__ bool pg_any_bad(const uint16_t*, const uint4& x) {
  return pg_bad16(x.x) || pg_bad16(x.x >> 16) || pg_bad16(x.y) || pg_bad16(x.y >> 16) || pg_bad16(x.z) || pg_bad16(x.z >> 16) ||
         pg_bad16(x.w) || pg_bad16(x.w >> 16);
}
__device__ __forceinline__ bool pg_any_bad(const float*, const uint4& x) {
  return pg_bad32(__uint_as_float(x.x)) || pg_bad32(__uint_as_float(x.y)) || pg_bad32(__uint_as_float(x.z)) || pg_bad32(__uint_as_float(x.w));
}

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
// x and y into the elements p[0] and p[1], if they are not 0
__device__ __forceinline__ void pg_over(uint16_t* p, float x, float y) {
  const uint32_t w = pg_pack2(x, y);
  if (x != 0.f) p[0] = (uint16_t)w;
  if (y != 0.f) p[1] = (uint16_t)(w >> 16);
}
__device__ __forceinline__ void pg_over(float* p, float x, float y) {
  if (x != 0.f) p[0] = x;
  if (y != 0.f) p[1] = y;
}

// An infinite V in a row of finite score is infinite in the result, whatever the row's weight:
// next to a score 150 powers of two higher its fp32 weight is 0, and 0 inf NaN.  Sums that
// turned out not to be finite are therefore taken from V itself, once a piece's results are
// stored, and where parts are joined such a value is not scaled.  (In the results' place, when
// the sums' registers are free: this is to take none from what runs always.)

// Whether any of n sums (n even) is not finite (or any two have a product that is not).
template <int N>
__device__ __forceinline__ bool pg_unusual(const float (&o)[N]) {
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < N; i += 2) t = __builtin_fmaf(o[i], o[i + 1], t);
  return pg_bad32(t);
}
// sum + w x, where parts are joined
__device__ __forceinline__ float pg_add(float sum, float w, float x) { return pg_bad32(x) ? sum + x : __builtin_fmaf(w, x, sum); }

// The first cached row of [t, t1) whose V is not finite, or t1.  For all lanes of a wave together.
template <typename T>
__device__ __forceinline__ int pg_next_bad(const PagedCache& c, const int32_t* ids, int t, int t1) {
  constexpr int RB = kD * (int)sizeof(T), LPR = RB / 16, PER = 64 / LPR;   // lanes of a row, rows of a load
  const int lane = threadIdx.x & 63, mask = (1 << c.page_log) - 1;
#pragma unroll 1
  for (; t < t1; t = (t | 15) + 1) {                   // a page holds whole sixteens
    const char* from = c.v + (pg_page(c, pg_entry(ids, min(t >> c.page_log, c.max_pages - 1))) + (t & mask & ~15)) * RB;
    uint32_t rows = 0;
#pragma unroll 2
    for (int i = 0; i < 16 / PER; ++i) {
      const uint64_t b = __builtin_amdgcn_ballot_w64(pg_any_bad((const T*)nullptr, ldg16(from + (i * 64 + lane) * 16)));
#pragma unroll
      for (int y = 0; y < PER; ++y) rows |= (uint32_t)((b >> y * LPR & ((1ull << LPR) - 1)) != 0) << (i * PER + y);
    }
    rows >>= t & 15;
    if (rows) return min(t + __builtin_ctz(rows), t1);
  }
  return t1;
}
// The elements of the new rows [row0, row0 + ROWS) whose sums of V hold what is not finite, of
// the cached rows [t0, t1): put(row, x, y) gives dims 2 lane and 2 lane + 1 to where the row's
// result lies (0: finite).  `see`: cached rows that row number lane sees.
template <typename T, int ROWS, class F>
__device__ __forceinline__ void pg_restore(const PagedCache& c, const int32_t* ids, int t0, int t1, int see, int row0, F put) {
  const int lane = threadIdx.x & 63, mask = (1 << c.page_log) - 1;
  float z[ROWS][2] = {};
#pragma unroll 1
  for (int t = t0; (t = pg_next_bad<T>(c, ids, t, t1)) < t1; ++t) {
    const size_t row = pg_page(c, pg_entry(ids, min(t >> c.page_log, c.max_pages - 1))) + (t & mask);
    float x, y;
    pg_pair(reinterpret_cast<const T*>(c.v) + row * kD + 2 * lane, x, y);
    x = pg_bad32(x) ? x : 0.f;
    y = pg_bad32(y) ? y : 0.f;
    const uint64_t sees = __builtin_amdgcn_ballot_w64(t < see) >> row0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (sees >> r & 1) {
        z[r][0] += x;
        z[r][1] += y;
      }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
    if (__builtin_amdgcn_ballot_w64(z[r][0] != 0.f || z[r][1] != 0.f)) put(row0 + r, z[r][0], z[r][1]);
}

}  // namespace catekv
