// Decode attention of single tokens over caches of several kinds, with the
// weights added up per row on request: the stream kernel (one template for
// 8-bit, bf16 and fp32 views) and the kernel that joins its partials.
//
// Mathematics, per view and query head, everything in log2 units:
//   x_t = c q . K_t,  c = scale log2(e);  m the running maximum of x, raised only
//   when it would grow by more than kSlack;  P_t = 2^(x_t - m + kShift);
//   l = sum P,  O = sum P V;  out = O / l,  lse = ln 2 (m + log2 l - kShift).
// kShift lifts P so that two fp16 numbers hold it to 2^-22 of itself or 2^-36 of the
// largest P, whichever is more, and 2^(kShift + kSlack) still fits an fp16.
//
// Bound by HBM: 4 FLOP per byte of bf16, 8 per byte of codes.  128K rows (3 full
// views, 5 of 2112 rows) in e4m3: 103 MB in 24 us, 6 TB/s from the first tile's
// request (2.6 us: three dependent loads, the query rows) to the end of the average
// share, 3 us more to that of the slowest XCD (by time stamps in a copy); the same in
// bf16 with weights: 206 MB in 37 us; 1M rows (2 views) in int8: 544 MB in 95 us (5.7
// TB/s).  What is read from memory is what there is (104 MB, 207 MB and 546 MB by the
// counters, the tables and queries with it).  The join takes 4 to 5 us more, with
// weights 7, in fp32 9.
//
// Work: the plan's shares (equal numbers of rows), one workgroup of 8 waves
// each, tile u of a segment to wave u % 8, two tiles per wave in flight across
// segment borders.  A tile's scores come from the matrix cores as S^T = K Q^T
// with the group's heads as columns; lane n16 + 16 k4 then holds head n16's
// scores of the rows 4 k4 + r, which is the A operand of P V as it stands.  O:
// head 4 k4 + r, dim 8 n16 + e in register r of tile e.
#pragma once

#include "cache.h"
#include "common.h"

namespace catekv {

constexpr int kAtThreads = kAttendThreads;
constexpr int kAtWaves = kAtThreads / 64;
constexpr int kAtMaxSeg = kDecodeV2MaxSeg;   // segments described in LDS at a time
constexpr float kShift = 11.f;
constexpr float kSlack = 4.f;
// Maximum of no row, the lowest finite number: 2^(floor - m) is 0 for any score above
// it, 2^(-inf - floor) is 0, and inf - inf does not come up.
constexpr float kAtFloor = -3.402823466e38f;
constexpr float kLn2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// Rows of K and V, read once per step: their loads pass the caches by (once16, and
// the same for 8 bytes).  us per step, cached / past the caches: int8 1M 100.4 / 95.4,
// e4m3 16 x 16K-64K with the append 125.4 / 119.6, bf16 128K with weights 48.4 / 44.3;
// over the caches of 24 layers in turn e4m3 128K 28.6 / 27.8, int8 16 x 2304 with
// append and weights 39.4 / 37.6.  Where the Infinity Cache would have kept rows from
// one step to the next it is the other way round: the same two over 3 layers 26.2 /
// 27.1 and 36.0 / 36.7.
__device__ __forceinline__ uint2 once8(const void* p) {
  const u32x2 v = __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x2*)(p));
  return make_uint2(v.x, v.y);
}
__device__ __forceinline__ float ldg4f(const float* p) {
  return *(const __attribute__((address_space(1))) float*)(p);
}
// A pointer (or an int) that is the same on every lane, kept in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <typename P>
__device__ __forceinline__ P* uniform(P* p) {
  const uint64_t x = (uint64_t)p;
  const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint64_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (P*)(hi << 32 | lo);
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// A segment as the waves read it from LDS.
struct AtSeg {
  const char* k;
  const char* v;
  const float* ks;
  const float* vs;
  const char* kt;
  const char* vt;
  int32_t t0, t_end;        // rows of the main part (codes, or the rows themselves)
  int32_t n_units;          // tiles of the main part
  int32_t tail0, tail_n;    // rows of the tail buffer: first and how many
  int32_t row0;             // first query head
  int32_t slot;             // partial slot, or -1: the segment covers its view
  int32_t ml_slot;          // slot that keeps (m, l) for the weights
  int32_t soff, srows;      // the worker's scores: first row, rows per head
};

// ---- 4 rows x 4 bytes -> 4 words of one byte of each row ---------------------
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&o)[4]) {
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
  o[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

// Four codes as four fp16, exactly: int8 through 0x6400 | (code + 128) = 1152 +
// code, e4m3 by the conversion instruction (every e4m3 value is an fp16).
template <int FMT>
__device__ __forceinline__ uint2 codes_to_f16(uint32_t w) {
  if constexpr (FMT == CATEKV_I8) {
    w ^= 0x80808080u;
    const f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
    const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  } else {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  }
}
template <int FMT>
__device__ __forceinline__ f16x8 codes8_to_f16(uint32_t a, uint32_t b) {
  const uint2 x = codes_to_f16<FMT>(a), y = codes_to_f16<FMT>(b);
  return __builtin_bit_cast(f16x8, make_uint4(x.x, x.y, y.x, y.y));
}

__device__ __forceinline__ uint32_t pack_f16(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), f16x2));
}
__device__ __forceinline__ f32x2 unpack_f16(uint32_t w) {
  return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
}
__device__ __forceinline__ uint32_t pack_bf16x2(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}

// Elements of a stored row, T = uint16_t (bf16) or float: element i of 16 bytes.
template <typename T>
__device__ __forceinline__ float elem(const uint4& w, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(word(w, i));
  const uint32_t x = word(w, i >> 1);
  return i & 1 ? bf16_hi(x) : bf16_lo(x);
}

// 16 rows on the fp32 matrix instruction: S^T (16 rows x 16 heads) += K Q^T, with
// lane (n16, k4) holding the 16-byte pieces 4 i + k4 of row n16 and of head n16 (a
// load covers 64 bytes of a row; the loads of a line find it in cache, so none passes
// it by: 113 against 72 us for fp32 100K rows); and O += P V with the four rows
// 4 k4 + r of V.  Serves fp32 views and the tails
// of 8-bit views (exact products, fp32 sums).
template <typename T>
struct Rows16 {
  static constexpr int NK = 32 * (int)sizeof(T) / 16, NV = 8 * (int)sizeof(T) / 16, PER = 16 / (int)sizeof(T);
  uint4 k[NK];
  uint4 v[4][NV];
  // rows kp, vp .. + last (uniform), a row behind them is the last one again
  __device__ __forceinline__ void load(const char* kp, const char* vp, int last, int n16, int k4) {
    const uint32_t ko = (uint32_t)(min(n16, last) * kD) * sizeof(T) + k4 * 16;
#pragma unroll
    for (int i = 0; i < NK; ++i) k[i] = ldg16(kp + ko + 64 * i);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t vo = (uint32_t)(min(4 * k4 + r, last) * kD + n16 * 8) * sizeof(T);
#pragma unroll
      for (int i = 0; i < NV; ++i) v[r][i] = ldg16(vp + vo + 16 * i);
    }
  }
  // q(i): the 16 bytes 4 i + k4 of the head's query, in the storage type
  template <typename F>
  __device__ __forceinline__ f32x4 scores(F q) const {
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const uint4 w = q(i);
#pragma unroll
      for (int e = 0; e < PER; e += 2) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(elem<T>(k[i], e), elem<T>(w, e), s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(elem<T>(k[i], e + 1), elem<T>(w, e + 1), s1, 0, 0, 0);
      }
    }
    return s0 + s1;
  }
  __device__ __forceinline__ void pv(const float* p, f32x4 (&O)[8]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        O[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[r], elem<T>(v[r][e / PER], e % PER), O[e], 0, 0, 0);
  }
};

// ---- the kinds of views -------------------------------------------------------
// A Kind has TOK rows per tile, its queries in the layout of its products, and a
// tile: load(), scores() (raw; x = S * factor()), pv().

// 8-bit codes: both products on fp16 MFMAs.  A query row is scaled by a power of
// two to a maximum in [2^14, 2^15), so that a bf16 element is an fp16 exactly
// down to 2^-31 of the largest (below, off by at most 2^-39 of it); an fp32 row is
// split into two fp16 rows (22 bits).  The block's K scale multiplies the scores
// in fp32, its V scale the tile's P V sums.  Converting costs 1.25 (int8) or 0.5
// instructions per code of K and about twice that with the transpose of V: by the
// counters 31% of the issue slots in e4m3 (128K rows: 4.5M wave instructions in 24 us),
// 44% in int8 (1M: 25.6M in 95 us), the matrix cores busy 6 and 11%.  Tiles of 16 rows: 27.2
// against 26.8 us at 128K, 135.5 against 132.0 at 16 x 16K-64K (e4m3).
template <int FMT, typename QT>
struct Kind8 {
  static constexpr int TOK = 32;
  static constexpr bool kTail = true;
  typedef catekv_q8_view View;
  typedef QT T;
  static constexpr int NQ = sizeof(QT) == 4 ? 2 : 1;
  struct Q {
    f16x8 w[NQ][4];
    float unscale;
  };
  struct Tile {
    uint4 k[2][2];
    uint2 v[8];
    float ks, vs;
  };
  __device__ static __forceinline__ void load_q(Q& q, const uint4* row, bool head, int k4) {
    // product (j, half) of a tile's row: dims 16 (4 j + k4) + 8 half, eight of them
    float f[4][8];
    float big = 0.f;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int d0 = 16 * (4 * (p >> 1) + k4) + 8 * (p & 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 w = row[(d0 + i) * (int)sizeof(QT) / 16];
        f[p][i] = head ? elem<QT>(w, (d0 + i) % (16 / (int)sizeof(QT))) : 0.f;
        big = fmaxf(big, fabsf(f[p][i]));
      }
    }
    big = max_xor32(max_xor16(big));
    const int e = min(14 - ((int)(__float_as_uint(big) >> 23) - 127), 126);
    const float up = __uint_as_float((uint32_t)(e + 127) << 23);
    q.unscale = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = f[p][2 * i] * up, b = f[p][2 * i + 1] * up;
        hi[i] = pack_f16(a, b);
        const f32x2 h = unpack_f16(hi[i]);
        lo[i] = pack_f16(a - h.x, b - h.y);
      }
      q.w[0][p] = __builtin_bit_cast(f16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
      if constexpr (NQ == 2) q.w[1][p] = __builtin_bit_cast(f16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
    }
  }
  // A block is whole and holds the tile: no row is behind its end.
  __device__ static __forceinline__ void load(Tile& b, const AtSeg& sg, int t, int block, int n16, int k4) {
    const char* kp = uniform(sg.k) + (size_t)t * kD;
    const char* vp = uniform(sg.v) + (size_t)t * kD;
    const uint32_t ko = n16 * kD + k4 * 16, vo = 4 * k4 * kD + n16 * 8;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) b.k[h][j] = once16(kp + ko + h * 16 * kD + j * 64);
#pragma unroll
    for (int r = 0; r < 8; ++r) b.v[r] = once8(vp + vo + ((r >> 2) * 16 + (r & 3)) * kD);
    b.ks = ldg4f(uniform(sg.ks) + t / block);
    b.vs = ldg4f(uniform(sg.vs) + t / block);
  }
  __device__ static __forceinline__ float factor(const Tile& b, const Q& q, float c) { return b.ks * (c * q.unscale); }
  __device__ static __forceinline__ void scores(const Tile& b, const Q& q, f32x4 (&S)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint4& w = b.k[h][p >> 1];
        const f16x8 a = p & 1 ? codes8_to_f16<FMT>(w.z, w.w) : codes8_to_f16<FMT>(w.x, w.y);
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q.w[0][p], s, 0, 0, 0);
        if constexpr (NQ == 2) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q.w[1][p], s, 0, 0, 0);
      }
      S[h] = s;
    }
  }
  // P = hi + lo in fp16, 22 bits.  Lane (n16, k4) holds P of the rows 4 k4 + r of both
  // halves, eight of the 32 that a product sums over, and the codes of the same
  // rows: dims 8 n16 .. + 8, one product each.
  __device__ static __forceinline__ void pv(const Tile& b, const float (&P)[8], f32x4 (&O)[8]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = pack_f16(P[2 * i], P[2 * i + 1]);
      const f32x2 h = unpack_f16(hi[i]);
      lo[i] = pack_f16(P[2 * i] - h.x, P[2 * i + 1] - h.y);
    }
    const f16x8 A_hi = __builtin_bit_cast(f16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    const f16x8 A_lo = __builtin_bit_cast(f16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
    for (int half = 0; half < 2; ++half) {      // dims 8 n16 + 4 half + e
      uint32_t w[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint2* v = b.v + 4 * h;
        if (half) transpose4(v[0].y, v[1].y, v[2].y, v[3].y, w[h]);
        else transpose4(v[0].x, v[1].x, v[2].x, v[3].x, w[h]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f16x8 B = codes8_to_f16<FMT>(w[0][e], w[1][e]);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(A_hi, B, o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(A_lo, B, o, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) O[4 * half + e][r] = __builtin_fmaf(b.vs, o[r], O[4 * half + e][r]);
      }
    }
  }
};

// bf16 rows: K Q^T on bf16 MFMAs; P as three bf16 parts (24 bits).
struct KindBf16 {
  static constexpr int TOK = 16;
  static constexpr bool kTail = false;
  typedef catekv_kv_ptrs View;
  typedef uint16_t T;
  struct Q {
    uint4 w[4];
  };
  struct Tile {
    uint4 k[4], v[4];
  };
  __device__ static __forceinline__ void load_q(Q& q, const uint4* row, bool head, int k4) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const uint4 w = row[4 * ks + k4];
      q.w[ks] = head ? w : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ static __forceinline__ void load(Tile& b, const AtSeg& sg, int t, int, int n16, int k4) {
    const int last = uniform(sg.t_end) - 1 - t;   // a row behind the end is the last one again
    const char* kp = uniform(sg.k) + (size_t)t * (kD * 2);
    const char* vp = uniform(sg.v) + (size_t)t * (kD * 2);
    const uint32_t ko = min(n16, last) * (kD * 2) + k4 * 16;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) b.k[ks] = once16(kp + ko + ks * 64);
#pragma unroll
    for (int r = 0; r < 4; ++r) b.v[r] = once16(vp + (uint32_t)(min(4 * k4 + r, last) * (kD * 2) + n16 * 16));
  }
  __device__ static __forceinline__ float factor(const Tile&, const Q&, float c) { return c; }
  __device__ static __forceinline__ void scores(const Tile& b, const Q& q, f32x4 (&S)[1]) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b.k[ks]), __builtin_bit_cast(bf16x8, q.w[ks]),
                                                  s, 0, 0, 0);
    S[0] = s;
  }
  __device__ static __forceinline__ void pv(const Tile& b, const float (&P)[4], f32x4 (&O)[8]) {
    s16x4 A[3];
    float rest[4] = {P[0], P[1], P[2], P[3]};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const uint32_t a = pack_bf16x2(rest[0], rest[1]), c = pack_bf16x2(rest[2], rest[3]);
      A[i] = __builtin_bit_cast(s16x4, make_uint2(a, c));
      rest[0] -= bf16_lo(a);
      rest[1] -= bf16_hi(a);
      rest[2] -= bf16_lo(c);
      rest[3] -= bf16_hi(c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {               // dims 8 n16 + 2 i and + 1
      const uint32_t w[4] = {word(b.v[0], i), word(b.v[1], i), word(b.v[2], i), word(b.v[3], i)};
      const s16x4 even = __builtin_bit_cast(s16x4, make_uint2(__builtin_amdgcn_perm(w[1], w[0], 0x05040100u),
                                                              __builtin_amdgcn_perm(w[3], w[2], 0x05040100u)));
      const s16x4 odd = __builtin_bit_cast(s16x4, make_uint2(__builtin_amdgcn_perm(w[1], w[0], 0x07060302u),
                                                             __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)));
#pragma unroll
      for (int a = 0; a < 3; ++a) {
        O[2 * i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(A[a], even, O[2 * i], 0, 0, 0);
        O[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(A[a], odd, O[2 * i + 1], 0, 0, 0);
      }
    }
  }
};

// fp32 rows: fp32 MFMAs.  The queries stay in LDS (their 32 registers beside two
// tiles' 128 would spill).
struct KindF32 {
  static constexpr int TOK = 16;
  static constexpr bool kTail = false;
  typedef catekv_kv_ptrs View;
  typedef float T;
  struct Q {
    const uint4* row;
    bool head;
  };
  typedef Rows16<float> Tile;
  __device__ static __forceinline__ void load_q(Q& q, const uint4* row, bool head, int k4) {
    q.row = row + k4;
    q.head = head;
  }
  __device__ static __forceinline__ void load(Tile& b, const AtSeg& sg, int t, int, int n16, int k4) {
    const size_t at = (size_t)t * (kD * 4);
    b.load(uniform(sg.k) + at, uniform(sg.v) + at, uniform(sg.t_end) - 1 - t, n16, k4);
  }
  __device__ static __forceinline__ float factor(const Tile&, const Q&, float c) { return c; }
  __device__ static __forceinline__ void scores(const Tile& b, const Q& q, f32x4 (&S)[1]) {
    S[0] = b.scores([&](int i) { return q.head ? q.row[4 * i] : make_uint4(0, 0, 0, 0); });
  }
  __device__ static __forceinline__ void pv(const Tile& b, const float (&P)[4], f32x4 (&O)[8]) { b.pv(P, O); }
};

// ---- the stream kernel ----------------------------------------------------------
template <class K, int G, bool ACC>
__global__ __launch_bounds__(kAtThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attend_stream_kernel(AttendArgs a) {
  typedef typename K::T T;
  constexpr int WAVES = kAtWaves, NT = kAtThreads, TOK = K::TOK, NS = TOK / 16;
  constexpr int SF = (int)decode_slot_floats(G);
  constexpr int QW = kD * (int)sizeof(T) / 16;   // 16-byte words of a query row
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  const int n16 = lane & 15, k4 = lane >> 4;
  const int hkv = a.hkv, hq = hkv * G;
  const float c = a.scale * kLog2e;
  const bool head_lane = n16 < G;

  __shared__ AtSeg s_seg[kAtMaxSeg];
  __shared__ uint4 s_q[kAtMaxSeg][G][QW];
  __shared__ float s_o[2][WAVES][G][kD];
  __shared__ float s_ml[2][WAVES][2][G];
  extern __shared__ float4 s_scores[];           // the worker's scores, where they fit (a.staged)

  // A one-workgroup-per-CU plan lists a worker's segments in one place, each with
  // their count; any other has them behind an index, sixteen of them taken at a time.
  typedef typename K::View View;
  const View* views = reinterpret_cast<const View*>(a.views);
  const bool v2 = a.variant == kDecodeStreamV2;
  V2Item mine{};
  if (v2) mine = a.v2items[(size_t)blockIdx.x * kAtMaxSeg + min((int)threadIdx.x, kAtMaxSeg - 1)];
  const int seg_lo = v2 ? 0 : a.worker_seg[blockIdx.x];
  const int seg_hi = v2 ? (int)((uint32_t)uniform(mine.bh_n) >> 24) : a.worker_seg[blockIdx.x + 1];
  int sbase = 0;                                 // the worker's score rows given out so far

  for (int s0 = seg_lo; s0 < seg_hi; s0 += kAtMaxSeg) {
    const int nseg = min(seg_hi - s0, kAtMaxSeg);
    if ((int)threadIdx.x < nseg) {
      int bh, t0, t1, slot;
      if (v2) {
        bh = mine.bh_n & 0xFFFFFF;
        t0 = mine.t0;
        t1 = mine.t1;
        slot = mine.slot;
      } else {
        const DecodeItem it = a.items[s0 + threadIdx.x];
        const ViewInfo vi = a.infos[it.bh];
        bh = it.bh;
        t0 = it.t0;
        t1 = it.t1;
        slot = vi.n_parts > 1 ? vi.first_slot + it.part : -1;
      }
      int64_t len = a.lens[bh];
      len = len < 0 ? 0 : len;
      const View view = views[bh];
      const int b = bh / hkv, h = bh - b * hkv;
      AtSeg sg{};
      sg.t0 = t0;
      const int end = (int)(len < (int64_t)t1 ? len : (int64_t)t1);     // rows [t0, end) of this segment
      sg.k = reinterpret_cast<const char*>(view.k);
      sg.v = reinterpret_cast<const char*>(view.v);
      sg.t_end = end;
      if constexpr (K::kTail) {
        sg.ks = view.k_scale;
        sg.vs = view.v_scale;
        sg.kt = reinterpret_cast<const char*>(view.k_tail);
        sg.vt = reinterpret_cast<const char*>(view.v_tail);
        const int64_t coded = len / a.block * a.block;                  // rows in whole blocks
        sg.t_end = (int)(coded < (int64_t)end ? coded : (int64_t)end);
        const int64_t first = coded > (int64_t)t0 ? coded : (int64_t)t0;
        sg.tail0 = first < (int64_t)end ? (int)(first - coded) : 0;
        sg.tail_n = first < (int64_t)end ? (int)(end - first) : 0;
      }
      sg.n_units = sg.t_end > t0 ? (sg.t_end - t0 + TOK - 1) / TOK : 0;
      sg.row0 = b * hq + h * G;
      sg.slot = slot;
      sg.ml_slot = slot;
      if (ACC && slot < 0) sg.ml_slot = a.infos[bh].first_slot;
      sg.srows = (t1 - t0 + 63) & ~63;
      s_seg[threadIdx.x] = sg;
    }
    __syncthreads();
    if constexpr (ACC) {
      if ((int)threadIdx.x < nseg) {
        int off = sbase;
        for (int s = 0; s < (int)threadIdx.x; ++s) off += s_seg[s].srows;
        s_seg[threadIdx.x].soff = off;
      }
      for (int s = 0; s < nseg; ++s) sbase += s_seg[s].srows;
    }

    // The query rows of every segment, waited for before any tile is requested: behind
    // the first tiles of all workgroups they would take 2 us longer.
    const int nq = nseg * G * QW;
    auto q_row = [&](int t) {
      const int s = t / (G * QW), r = t - s * (G * QW);
      return ldg16(reinterpret_cast<const char*>(a.q) + ((size_t)s_seg[s].row0 + r / QW) * (kD * sizeof(T)) + (r % QW) * 16);
    };
    const int tq = min((int)threadIdx.x, nq - 1);
    const uint4 qv = q_row(tq);

    // ---- this wave's tiles ------------------------------------------------------
    int is = 0, iu = wave;                        // next tile: segment, tile of the segment
    auto skip = [&]() {
      while (is < nseg && iu >= s_seg[is].n_units) {
        ++is;
        iu = wave;
      }
    };
    skip();
    int n_my = 0;                                 // tiles left to use
    for (int s = 0; s < nseg; ++s) {
      const int u = s_seg[s].n_units;
      n_my += u > wave ? (u - wave + WAVES - 1) / WAVES : 0;
    }
    n_my = uniform(n_my);
    {
      const int s = tq / (G * QW), r = tq - s * (G * QW);
      s_q[s][r / QW][r % QW] = qv;
    }
    for (int t = threadIdx.x + NT; t < nq; t += NT) {
      const int s = t / (G * QW), r = t - s * (G * QW);
      s_q[s][r / QW][r % QW] = q_row(t);
    }
    __syncthreads();
    typename K::Tile tb[2];
    auto issue = [&](int buf) {                   // called only while the wave has tiles left
      const AtSeg& sg = s_seg[is];
      K::load(tb[buf], sg, uniform(sg.t0 + iu * TOK), a.block, n16, k4);
      iu += WAVES;
      skip();
    };

    f32x4 O[8];
    float m, l;
    typename K::Q q;
    auto reset_state = [&]() {
#pragma unroll
      for (int e = 0; e < 8; ++e) O[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      m = head_lane ? kAtFloor : INFINITY;        // +inf: P = 0 in the columns behind the heads
      l = 0.f;
    };

    // scores S (x = S kf) of NG groups of 16 rows: raises the maximum, turns them
    // into P and adds them to l; rows from `rows` on are masked
    auto softmax = [&](auto ng, const f32x4* S, float kf, int rows, float* P) {
      constexpr int NG = decltype(ng)::value;
      float sv[4 * NG];
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4 * NG; ++i) {
        sv[i] = 16 * (i >> 2) + 4 * k4 + (i & 3) < rows ? S[i >> 2][i & 3] * kf : -INFINITY;
        mx = fmaxf(mx, sv[i]);
      }
      mx = max_xor32(max_xor16(mx));
      if (__builtin_amdgcn_ballot_w64(head_lane && mx > m + kSlack)) {
        float corr = 1.f;
        if (head_lane && mx > m) {
          corr = fast_exp2(m - mx);               // 0 while m is the floor
          m = mx;
        }
        l *= corr;
#pragma unroll
        for (int r = 0; r < 4; ++r) {             // register r of O belongs to head 4 k4 + r
          const float cr = __int_as_float(__builtin_amdgcn_ds_bpermute((4 * k4 + r) << 2, __float_as_int(corr)));
#pragma unroll
          for (int e = 0; e < 8; ++e) O[e][r] *= cr;
        }
      }
#pragma unroll
      for (int i = 0; i < 4 * NG; ++i) {
        P[i] = fast_exp2(sv[i] - m + kShift);
        l += P[i];
      }
    };
    // x of 16 rows into the worker's scores, four rows of a head per lane
    auto keep_scores = [&](const AtSeg& sg, int t, f32x4 S, float kf) {
      if (head_lane) {
        const size_t at = (size_t)sg.soff * G + (size_t)n16 * sg.srows + (t - sg.t0) + 4 * k4;
        const float4 x = make_float4(S[0] * kf, S[1] * kf, S[2] * kf, S[3] * kf);
        if (a.staged) s_scores[at >> 2] = x;
        else *reinterpret_cast<float4*>(a.scores + (size_t)blockIdx.x * a.score_rows * G + at) = x;
      }
    };

    // The tail of segment s: tiles of 16 rows, to the waves behind the last tile's.
    auto tail = [&](int s) {
      if constexpr (K::kTail) {
        const AtSeg& sg = s_seg[s];
        const int n_tiles = (sg.tail_n + 15) / 16;
        for (int i = (wave + WAVES - sg.n_units % WAVES) % WAVES; i < n_tiles; i += WAVES) {
          Rows16<T> rows;
          const size_t at = (size_t)uniform(sg.tail0 + 16 * i) * (kD * sizeof(T));
          rows.load(uniform(sg.kt) + at, uniform(sg.vt) + at, uniform(sg.tail_n) - 16 * i - 1, n16, k4);
          const f32x4 S[1] = {rows.scores([&](int j) {
            const uint4 w = s_q[s][head_lane ? n16 : 0][4 * j + k4];
            return head_lane ? w : make_uint4(0, 0, 0, 0);
          })};
          float P[4];
          softmax(std::integral_constant<int, 1>{}, S, c, sg.tail_n - 16 * i, P);
          // rows of the tail stand behind the codes' in the segment's order
          if constexpr (ACC) keep_scores(sg, max(sg.t_end, sg.t0) + 16 * i, S[0], c);
          rows.pv(P, O);
        }
      }
    };

    // end of segment s: the eight waves' states joined through LDS, the output or
    // the partial written
    auto merge = [&](int s) {
      const int buf = s & 1;
      const float lt = add_xor32(add_xor16(l));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int head = 4 * k4 + r;
        if (head < G) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s_o[buf][wave][head][8 * n16 + e] = O[e][r];
        }
      }
      if (lane < G) {
        s_ml[buf][wave][0][lane] = m;
        s_ml[buf][wave][1][lane] = lt;
      }
      barrier_lds_only();
      const AtSeg& sg = s_seg[s];
      for (int t = threadIdx.x; t < G * kD; t += NT) {
        const int g = t / kD, e = t - g * kD;
        float M = kAtFloor;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) M = fmaxf(M, s_ml[buf][w][0][g]);
        float L = 0.f, Ov = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const float cw = fast_exp2(s_ml[buf][w][0][g] - M);
          L += s_ml[buf][w][1][g] * cw;
          Ov += s_o[buf][w][g][e] * cw;
        }
        if (sg.slot < 0) {
          a.out[((size_t)sg.row0 + g) * kD + e] = L == 0.f ? 0.f : Ov / L;
          if (a.lse && e == 0) a.lse[sg.row0 + g] = L == 0.f ? -INFINITY : kLn2 * M + logf(L * fast_exp2(-kShift));
        } else {
          a.slots[(size_t)sg.slot * SF + g * kD + e] = Ov;
        }
        if ((ACC || sg.slot >= 0) && e == 0) {
          float* ml = a.slots + (size_t)sg.ml_slot * SF + G * kD + g;
          ml[0] = M;
          ml[G] = L;
        }
      }
    };

    auto consume = [&](int buf, int s, int t) {
      const AtSeg& sg = s_seg[s];
      f32x4 S[NS];
      K::scores(tb[buf], q, S);
      const float kf = K::factor(tb[buf], q, c);
      float P[4 * NS];
      softmax(std::integral_constant<int, NS>{}, S, kf, sg.t_end - t, P);
      if constexpr (ACC) {
#pragma unroll
        for (int h = 0; h < NS; ++h) keep_scores(sg, t + 16 * h, S[h], kf);
      }
      K::pv(tb[buf], P, O);
    };

    // One tile is in flight while another is used, across segments too, and every
    // issue loads a real tile: the wave's very last tile is used without one.
    // `odd`: the tile to be used next is in buffer 1.
    if (n_my > 0) issue(0);
    bool odd = false;
    for (int s = 0; s < nseg; ++s) {
      const int u = s_seg[s].n_units;
      const int n_s = u > wave ? (u - wave + WAVES - 1) / WAVES : 0;
      reset_state();
      if (n_s > 0) {
        K::load_q(q, s_q[s][head_lane ? n16 : 0], head_lane, k4);
        n_my -= n_s;
        int n = n_my > 0 ? n_s : n_s - 1;         // tiles used with another one in flight
        int t = s_seg[s].t0 + wave * TOK;
        constexpr int STEP = WAVES * TOK;
        if (odd && n > 0) {
          issue(0);
          consume(1, s, t);
          t += STEP;
          --n;
          odd = false;
        }
        while (n >= 2) {
          issue(1);
          consume(0, s, t);
          issue(0);
          consume(1, s, t + STEP);
          t += 2 * STEP;
          n -= 2;
        }
        if (n == 1) {
          issue(1);
          consume(0, s, t);
          t += STEP;
          odd = true;
        }
        if (n_my == 0) {                          // the wave's last tile
          if (odd) consume(1, s, t);
          else consume(0, s, t);
        }
      }
      tail(s);
      merge(s);
    }
    __syncthreads();                              // the tables and the merge area are free
    if (ACC && a.staged) {                        // (a plan of one batch of segments)
      float4* to = reinterpret_cast<float4*>(a.scores + (size_t)blockIdx.x * a.score_rows * G);
      for (int i = threadIdx.x; i < sbase * G / 4; i += NT) to[i] = s_scores[i];
    }
  }
}

// Views of up to so many parts are joined by one workgroup instead of one per head.  us
// of the join with 1 / 8 / 32: with weights, 128 views of 2 or 3 parts, 4 heads 6.4 /
// 5.1 / 8.0, 64 views of 4 parts 4.1 / 4.2 / 4.3; without, 16 views of 16 parts, 8
// heads 3.9 / 3.9 / 7.0; elsewhere the same.
constexpr int kFewParts = 8;

// ---- joining the partials, and the weights ----------------------------------------
// With acc, workgroup w < n_workers first: the weights of worker w's rows, from the
// scores it kept (they come from behind the L2: 9.1 MB read at 128K rows, of them 6.5
// scores) and from all of the view's (m, l); they take longer than the rest.  Behind them, for every view and head: its partials,
// when it has more than one.
template <int G, bool ACC>
__global__ __launch_bounds__(kAtThreads) void attend_join_kernel(AttendArgs a) {
  constexpr int SF = (int)decode_slot_floats(G);
  constexpr int NT = kAtThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  if (!ACC || (int)blockIdx.x >= a.n_workers) {
    constexpr int LANES = NT / 32, BATCH = 16;    // parts side by side, parts per thread and round
    const int at = blockIdx.x - (ACC ? a.n_workers : 0), bh = at / G, g = at - bh * G;
    const ViewInfo vi = a.infos[bh];
    const int P = vi.n_parts;
    if (P <= 1) return;
    if (P <= kFewParts) {
      // few parts: the first head's workgroup joins all heads, one value per thread
      if (g > 0) return;
      const float* base = a.slots + (size_t)vi.first_slot * SF;
      for (int i = t; i < G * kD; i += NT) {
        const int gi = i / kD;
        float ms[kFewParts], ls[kFewParts], os[kFewParts];
        float M = kAtFloor, L = 0.f, O = 0.f;
#pragma unroll
        for (int p = 0; p < kFewParts; ++p) {
          const float* sl = base + (size_t)min(p, P - 1) * SF;
          ms[p] = p < P ? sl[G * kD + gi] : kAtFloor;
          ls[p] = p < P ? sl[G * kD + G + gi] : 0.f;
          os[p] = p < P ? sl[i] : 0.f;
          M = fmaxf(M, ms[p]);
        }
#pragma unroll
        for (int p = 0; p < kFewParts; ++p) {
          const float w = fast_exp2(ms[p] - M);
          L += w * ls[p];
          O += w * os[p];
        }
        a.out[(size_t)bh * G * kD + i] = L == 0.f ? 0.f : O / L;
        if (a.lse && i % kD == 0) a.lse[(size_t)bh * G + gi] = L == 0.f ? -INFINITY : kLn2 * M + logf(L * fast_exp2(-kShift));
      }
      return;
    }
    __shared__ float s_red[NT / 64];
    __shared__ float4 s_acc[LANES][32];
    __shared__ float s_l[LANES];
    const int pl = t >> 5, dq = t & 31;
    const float* base = a.slots + (size_t)vi.first_slot * SF;
    float M = kAtFloor, L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = pl; p0 < P; p0 += LANES * BATCH) {
      float ms[BATCH], ls[BATCH];
      float4 os[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int p = p0 + u * LANES;
        ms[u] = kAtFloor;
        ls[u] = 0.f;
        os[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p < P) {
          const float* sl = base + (size_t)p * SF;
          ms[u] = sl[G * kD + g];
          ls[u] = sl[G * kD + G + g];
          os[u] = *reinterpret_cast<const float4*>(sl + g * kD + 4 * dq);
        }
      }
      float mb = M;
#pragma unroll
      for (int u = 0; u < BATCH; ++u) mb = fmaxf(mb, ms[u]);
      const float ca = fast_exp2(M - mb);
      L *= ca;
      acc.x *= ca; acc.y *= ca; acc.z *= ca; acc.w *= ca;
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const float w = fast_exp2(ms[u] - mb);
        L += w * ls[u];
        acc.x += w * os[u].x; acc.y += w * os[u].y; acc.z += w * os[u].z; acc.w += w * os[u].w;
      }
      M = mb;
    }
    float Mx = max_xor32(M);
    if (lane == 0) s_red[wave] = Mx;
    __syncthreads();
    Mx = s_red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) Mx = fmaxf(Mx, s_red[w]);
    const float cs = fast_exp2(M - Mx);
    s_acc[pl][dq] = make_float4(acc.x * cs, acc.y * cs, acc.z * cs, acc.w * cs);
    if (dq == 0) s_l[pl] = L * cs;
    __syncthreads();
    if (t < 32) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float Lt = 0.f;
#pragma unroll
      for (int p = 0; p < LANES; ++p) {
        o.x += s_acc[p][t].x; o.y += s_acc[p][t].y; o.z += s_acc[p][t].z; o.w += s_acc[p][t].w;
        Lt += s_l[p];
      }
      const size_t row = (size_t)bh * G + g;
      const float inv = Lt == 0.f ? 0.f : 1.f / Lt;
      *reinterpret_cast<float4*>(a.out + row * kD + 4 * t) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      if (a.lse && t == 0) a.lse[row] = Lt == 0.f ? -INFINITY : kLn2 * Mx + logf(Lt * fast_exp2(-kShift));
    }
    return;
  }
  if constexpr (ACC) {
    __shared__ float s_m[NT / 64][G], s_s[NT / 64][G];
    const int w = blockIdx.x;
    const bool v2 = a.variant == kDecodeStreamV2;
    const V2Item* list = a.v2items + (size_t)w * kAtMaxSeg;
    const int seg_lo = v2 ? 0 : a.worker_seg[w];
    int seg_hi = v2 ? 1 : a.worker_seg[w + 1];    // (v2: the first entry tells)
    int64_t soff = 0;
    for (int s = seg_lo; s < seg_hi; ++s) {
      int bh, t0, t1;
      if (v2) {
        const V2Item it = list[s];
        bh = it.bh_n & 0xFFFFFF;
        t0 = it.t0;
        t1 = it.t1;
        seg_hi = (int)((uint32_t)it.bh_n >> 24);
      } else {
        const DecodeItem it = a.items[s];
        bh = it.bh;
        t0 = it.t0;
        t1 = it.t1;
      }
      const int srows = (t1 - t0 + 63) & ~63;
      const float* sc = a.scores + ((size_t)w * a.score_rows + soff) * G;
      soff += srows;
      int64_t len = a.lens[bh];
      len = len < 0 ? 0 : len;                    // as the stream kernel reads it: the low 32 bits mean nothing
      const ViewInfo vi = a.infos[bh];
      auto acc = (__attribute__((address_space(1))) float*)(a.acc[bh] + t0);
      const int n = (int)(len < (int64_t)t1 ? len : (int64_t)t1) - t0;
      if (n <= 0) continue;
      // the first rows' scores and weights, requested beside the parts
      constexpr int AHEAD = 4;
      float x[AHEAD][G], old[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = min(u * NT + t, n - 1);
#pragma unroll
        for (int g = 0; g < G; ++g) x[u][g] = sc[(size_t)g * srows + i];
        old[u] = acc[i];
      }
      // (M, L) of every head of the view, from all of its parts: thread t takes
      // head t % G of the parts t / G, t / G + NT / G, ...
      const float* base = a.slots + (size_t)vi.first_slot * SF + G * kD + (t & (G - 1));
      float M = kAtFloor, L = 0.f;
      for (int p = t / G; p < vi.n_parts; p += NT / G) {
        const float pm = base[(size_t)p * SF], pl = base[(size_t)p * SF + G];
        const float nm = fmaxf(M, pm);
        L = L * fast_exp2(M - nm) + pl * fast_exp2(pm - nm);
        M = nm;
      }
#pragma unroll
      for (int o = 32; o >= G; o >>= 1) {
        const float pm = shfl_xor(M, o), pl = shfl_xor(L, o);
        const float nm = fmaxf(M, pm);
        L = L * fast_exp2(M - nm) + pl * fast_exp2(pm - nm);
        M = nm;
      }
      barrier_lds_only();                         // the previous segment's values have been read
      if (lane < G) {
        s_m[wave][lane] = M;
        s_s[wave][lane] = L;
      }
      barrier_lds_only();
      float mg[G], ig[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float Mx = s_m[0][g];
#pragma unroll
        for (int u = 1; u < NT / 64; ++u) Mx = fmaxf(Mx, s_m[u][g]);
        float Lx = 0.f;
#pragma unroll
        for (int u = 0; u < NT / 64; ++u) Lx += s_s[u][g] * fast_exp2(s_m[u][g] - Mx);
        mg[g] = Mx;
        // a head whose rows all score -inf gives none of them weight (out 0, lse -inf)
        ig[g] = Lx == 0.f ? 0.f : fast_exp2(kShift) / (Lx * (float)G);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = u * NT + t;
        float wsum = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) wsum += fast_exp2(x[u][g] - mg[g]) * ig[g];
        if (i < n) acc[i] = a.decay > 0.f ? __builtin_fmaf(a.decay, old[u], wsum) : wsum;
      }
      for (int i = AHEAD * NT + t; i < n; i += NT) {
        float wsum = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) wsum += fast_exp2(sc[(size_t)g * srows + i] - mg[g]) * ig[g];
        acc[i] = a.decay > 0.f ? __builtin_fmaf(a.decay, acc[i], wsum) : wsum;
      }
    }
  }
}

// Static LDS of the stream kernel, rounded up generously.
constexpr size_t kAtMaxLds = 160 * 1024;
constexpr int64_t kStagedRows = 1200;
template <class K, int G>
constexpr size_t attend_static_lds() {
  return kAtMaxSeg * (sizeof(AtSeg) + G * kD * sizeof(typename K::T)) + 2 * kAtWaves * G * (kD + 2) * sizeof(float) + 1024;
}

template <class K, int G, bool ACC>
static hipError_t launch_attend_t(const AttendArgs& a, hipStream_t stream) {
  // The scores of a share of more than kStagedRows rows stay in LDS until its end, where
  // they fit beside the rest (4 heads: 6000 rows): stored tile by tile among the
  // loads they cost 5.8 us of a 128K bf16 step of 53, at the end 2.5.  us per step,
  // tile by tile / staged, by rows of a share: bf16 620: 24.0 / 24.0, 1200: 43.1 /
  // 41.0, 2050: 68.1 / 63.0; int8 830: 24.2 / 24.6, 1600: 35.4 / 34.2, 4700: 87.6 / 81.5.
  const size_t lds = ACC && a.variant == kDecodeStreamV2 && a.score_rows > kStagedRows
                         ? (size_t)a.score_rows * G * sizeof(float) : 0;
  const bool staged = lds > 0 && lds + attend_static_lds<K, G>() <= kAtMaxLds;
  AttendArgs b = a;
  b.staged = staged;
  hipLaunchKernelGGL((attend_stream_kernel<K, G, ACC>), dim3(a.n_workers), dim3(kAtThreads), staged ? lds : 0, stream, b);
  const hipError_t e = hipGetLastError();        // the join takes up what the stream kernel left
  if (e != hipSuccess) return e;
  const int n_joins = a.n_multi > 0 ? a.n_views * G : 0;
  const int blocks = n_joins + (ACC ? a.n_workers : 0);
  if (blocks > 0)
    hipLaunchKernelGGL((attend_join_kernel<G, ACC>), dim3(blocks), dim3(kAtThreads), 0, stream, a);
  return hipGetLastError();
}

template <class K, bool ACC>
static hipError_t launch_attend_g(int G, const AttendArgs& a, hipStream_t stream) {
  switch (G) {
    case 1: return launch_attend_t<K, 1, ACC>(a, stream);
    case 2: return launch_attend_t<K, 2, ACC>(a, stream);
    case 4: return launch_attend_t<K, 4, ACC>(a, stream);
    case 8: return launch_attend_t<K, 8, ACC>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace catekv
