// Attention of chunks of new tokens over caches in pages, bf16 (gfx950): bound by the
// matrix cores and, next to them, by the softmax on the vector unit.
//
// A workgroup of 8 waves, two per SIMD, takes 256 new rows of one view's group (row =
// token * G + head), 32 per wave, and walks over the view's cached rows in tiles of 64
// that global-to-LDS loads bring in, one tile ahead.
//
// Scores are S^T = K Q^T on v_mfma_f32_32x32x16_bf16: lane l holds new row l % 32 and,
// in register i, cached row 8 (i / 4) + 4 (l / 32) + i % 4 of 32.  A new row's maximum,
// sum and factor are then a lane's own but for one exchange of lane halves, and the
// registers are in place as the operand P^T of O^T = V^T P^T: a product does not ask in
// which order its terms come, and V is read in the same order.
//
// The softmax runs online, one tile behind: between the products of tile t + 1's scores
// the vector unit forms the weights of tile t, and while these meet V it takes the
// maxima of tile t + 1.  A wave issues in order, so the two are laid between each other
// in the program, and scheduling barriers keep them there.
#include <type_traits>

#include "paged_math.h"

namespace catekv {
namespace {

typedef pg_f32x16 f32x16;
typedef pg_bf16x8 bf16x8;
typedef pg_s16x4 s16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kTile = 64;                             // cached rows of a tile
constexpr int kRB = kD * 2;                           // bytes of a row
constexpr int kSeg = kRB / 16;                        // 16-byte chunks of a row
constexpr int kStage = kTile * kSeg;                  // chunks of a tile

__device__ __forceinline__ f32x16 mfma(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// K in LDS: chunk ch of row r at place ch ^ (r & 15), so that 16 rows' chunk ch lie in
// different banks.  The operand of step ks: dims 16 ks + 8 (l / 32) + [0, 8) of row 32 kb +
// l % 32, at k_lane() ^ 32 ks of a block of 32 rows.
__device__ __forceinline__ uint32_t k_lane(int lane) { return (lane & 31) * kRB + ((lane >> 5) ^ (lane & 15)) * 16; }
__device__ __forceinline__ uint4 k_op(const uint4* kt, int kb, int ks, uint32_t at) {
  return *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(kt) + (at ^ (ks * 32)) + kb * 32 * kRB);
}

// V in LDS: chunk ch of row r at place ch ^ (r & 3) << 2.  The operand of step st (16 cached
// rows): dims 32 db + l % 32 of rows 16 st + 4 (l / 32) + {0 .. 3, 8 .. 11}.  A transposing
// read takes 4 rows of 16 dims per 16 lanes and hands them out by dim.
__device__ __forceinline__ uint32_t v_lane(int lane) {
  const int i = lane & 15, row = (lane >> 5) * 4 + (i >> 2);
  return row * kRB + ((((lane >> 4) & 1) * 2 + ((i >> 1) & 1)) ^ ((i >> 2) << 2)) * 16 + (i & 1) * 8;
}
__device__ __forceinline__ uint4 v_op(const uint4* vt, int st, int db, uint32_t at) {
  const char* base = reinterpret_cast<const char*>(vt) + (at ^ (db * 64)) + st * 16 * kRB;
  const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)base));
  const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + 8 * kRB)));
  return make_uint4(x.x, x.y, y.x, y.y);
}

template <class F>
__device__ __forceinline__ uint4 each(uint4 v, F f) {
  return make_uint4(pg_both(v.x, f), pg_both(v.y, f), pg_both(v.z, f), pg_both(v.w, f));
}

// Weights of 16 cached rows, number h of 64, as an operand.
__device__ __forceinline__ uint4 pack16(const f32x16 (&x)[2], int h) {
  const f32x16& y = x[h >> 1];
  const int o = (h & 1) * 8;
  return make_uint4(pg_pack2(y[o], y[o + 1]), pg_pack2(y[o + 2], y[o + 3]), pg_pack2(y[o + 4], y[o + 5]), pg_pack2(y[o + 6], y[o + 7]));
}

template <int G>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_tile_kernel(PagedAttn a) {
  __shared__ uint4 s_k0[kStage], s_k1[kStage], s_v0[kStage], s_v1[kStage];

  const PagedCache& c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int w = a.workers[blockIdx.x]; w < a.workers[blockIdx.x + 1]; ++w) {
  uint32_t lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));                       // nothing of a piece is kept in registers for the next
  const int hi = lane >> 5;
  const PagedPiece pc = a.pieces[w];
  const int L = pg_rows(c, pc.view, pc.max_rows);
  const int n_rows = pc.n_new * G;
  const int see0 = L - pc.n_new + 1;                   // cached rows that the first new token sees
  const int r_end = min(pc.row0 + kTileRows, n_rows);  // past the piece's last new row
  const int t_end = min(pc.t1, see0 + (r_end - 1) / G);
  const int n_tiles = t_end > pc.t0 ? (t_end - pc.t0 + kTile - 1) / kTile : 0;
  // tiles that every new row of the piece sees in full come first, the others are masked
  const int n_full = max(0, min(n_tiles, (min(see0 + pc.row0 / G, t_end) - pc.t0) / kTile));
  const bool idle = pc.row0 + wave * 32 >= n_rows;     // none of the wave's rows exists

  const int h = pc.view % c.hkv;
  const int row = pc.row0 + wave * 32 + (lane & 31);   // this lane's new row and what it sees
  const bool mine = row < n_rows;
  const int tok = mine ? row / G : 0;
  const int see = mine ? see0 + tok : 0;
  const size_t qrow = ((size_t)(pc.tok0 + tok) * a.hq + h * G + (mine ? row - tok * G : 0)) * kRB;
  uint4 q[8];
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const uint4 x = ldg16(a.q + qrow + ks * 32 + hi * 16);
    q[ks] = mine ? x : make_uint4(0, 0, 0, 0);
  }

  // ---- tiles into LDS ------------------------------------------------------------
  // Load i of a wave fills rows 32 i + 4 wave + [0, 4) of a tile, which never lie in two
  // pages.  Rows past the view's come from where its table's clamped entries point; masked
  // tiles let none of them through.
  const int32_t* ids = c.table + (size_t)pc.view * c.max_pages;
  const int mask = (1 << c.page_log) - 1;
  const int wrow = wave * 4, lrow = wrow + (lane >> 4), place = lane & 15;
  const uint32_t k_off = (lane >> 4) * kRB + (place ^ (lrow & 15)) * 16;
  const uint32_t v_off = (lane >> 4) * kRB + (place ^ ((lrow & 3) << 2)) * 16;
  constexpr int kLoads = kStage / kTileThreads;        // per thread, K and V each
  struct Ids { int id[kLoads]; };
  auto fetch = [&](int t) __attribute__((always_inline)) {
    Ids x;
    const int r = pc.t0 + min(t, n_tiles - 1) * kTile + wrow;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x.id[i] = pg_entry(ids, min((r + 32 * i) >> c.page_log, c.max_pages - 1));
    return x;
  };
  auto issue = [&](const char* pool, uint32_t off, uint4* stage, int t, const Ids& x) __attribute__((always_inline)) {
    const int r = pc.t0 + min(t, n_tiles - 1) * kTile + wrow;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const char* base = pool + (pg_page(c, x.id[i]) + ((r + 32 * i) & mask)) * kRB;
      __builtin_amdgcn_global_load_lds(base + off, (lds_void*)&stage[i * kTileThreads + wave * 64], 16, 0, 0);
    }
  };

  // Places of the operands in LDS.  own() makes them new values to the compiler, which
  // would otherwise keep every step's in a register of its own through the loop.
  uint32_t ka = k_lane(lane), va = v_lane(lane);
  auto own = [&]() __attribute__((always_inline)) { asm volatile("" : "+v"(ka), "+v"(va)); };

  // ---- the softmax's state ---------------------------------------------------------
  f32x16 o[4] = {};
  float m = -INFINITY, l = 0.f;
  const float cs = a.log2_scale, thr = a.rise;
  float cw = cs;                                       // of the weights: pg_factor()

  auto scores = [&](const uint4* kt, f32x16 (&s)[2]) __attribute__((always_inline)) {
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = mfma(k_op(kt, kb, ks, ka), q[ks], s[kb]);
  };
  auto hide = [&](f32x16 (&s)[2], int t) __attribute__((always_inline)) {
    const int r = pc.t0 + t * kTile + 4 * hi;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = r + kb * 32 + 8 * (i >> 2) + (i & 3) < see ? s[kb][i] : -INFINITY;
  };
  auto maximum = [&](const f32x16 (&s)[2]) __attribute__((always_inline)) {
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
    return mx;
  };
  // a row's maximum moves where it grew by 8 powers of two (weights up to 2^8); from -inf always
  auto raise = [&](float mx) __attribute__((always_inline)) {
    mx = max_xor32(mx);
    if (__builtin_amdgcn_ballot_w64(mx > m && !(mx <= m + thr))) {
      const float corr = mx > m ? fast_exp2((m - mx) * cs) : 1.f;
      m = fmaxf(m, mx);
      cw = pg_factor(m, cs);
      l *= corr;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= corr;
    }
  };
  // weights of registers [4 j, 4 j + 4) of both score blocks laid end to end
  auto weights4 = [&](f32x16 (&s)[2], int j, float mc) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float w = fast_exp2(__builtin_fmaf(s[j >> 2][(j & 3) * 4 + e], cw, -mc));
      s[j >> 2][(j & 3) * 4 + e] = w;
      l += w;
    }
  };
  auto reference = [&]() __attribute__((always_inline)) { return m == -INFINITY ? 0.f : m * cw; };
  auto product = [&](const uint4* vt, const uint4 (&p)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = mfma(v_op(vt, st, d, va), p[st], o[d]);
  };
  // The same for a masked tile: 0 * NaN is NaN, so V that is not finite is taken as 0 in
  // the product and added, row by row, to the sums of the new rows that see it.
  auto product_masked = [&](const uint4* vt, const uint4 (&p)[4], int t) __attribute__((always_inline)) {
    uint32_t bad = 0;
#pragma unroll 1
    for (int i = 0; i < kStage / 64; ++i) {
      const uint4 x = each(vt[i * 64 + lane], pg_bad16);
      bad |= x.x | x.y | x.z | x.w;
    }
    if (!__builtin_amdgcn_ballot_w64(bad)) {
      product(vt, p);
      return;
    }
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = mfma(each(v_op(vt, st, d, va), pg_clean16), p[st], o[d]);
    const int r0 = pc.t0 + t * kTile;
#pragma unroll 1
    for (int r = 0; r < kTile; ++r) {
      const bool sees = r0 + r < see;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {                  // dims 32 d + 8 i + 4 hi + [0, 4)
          const char* at = reinterpret_cast<const char*>(vt) + (r * kSeg + ((4 * d + i) ^ ((r & 3) << 2))) * 16 + hi * 8;
          const uint2 w = *reinterpret_cast<const uint2*>(at);
          const float x[4] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * i + e] += sees && pg_bad32(x[e]) ? x[e] : 0.f;
        }
    }
  };

  // ---- the loop --------------------------------------------------------------------
  // At the head of turn t: tile t's scores are in s and their maxima taken in; K of t + 1
  // and V of t are in LDS or on their way.  Leaves tile t + 1's scores in s2.
  Ids next = {}, after = {};                           // pages of the tiles t + 1 and t + 2
  auto turn = [&](auto stage, auto mask_tag, int t, f32x16 (&s)[2], f32x16 (&s2)[2]) __attribute__((always_inline)) {
    constexpr bool B = decltype(stage)::value, MASK = decltype(mask_tag)::value;
    const uint4* kt = B ? s_k0 : s_k1;
    const uint4* vt = B ? s_v1 : s_v0;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    issue(c.k, k_off, B ? s_k1 : s_k0, t + 2, after);
    issue(c.v, v_off, B ? s_v0 : s_v1, t + 1, next);
    next = after;
    after = fetch(t + 3);
    if (idle) return;
    own();
    uint4 p[4];
    // Operands come in fours, one four ahead: their wait is then for reads that have had
    // four products' time (a wait counts all LDS reads on their way).
    const float mc = reference();
    uint4 f[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[0][i] = k_op(kt, i & 1, i >> 1, ka);
    s2[0] = s2[1] = f32x16{};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f[(x + 1) & 1][i] = x < 3 ? k_op(kt, i & 1, 2 * x + 2 + (i >> 1), ka) : v_op(vt, 0, i, va);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        s2[i & 1] = mfma(f[x & 1][i], q[2 * x + (i >> 1)], s2[i & 1]);
        if (i & 1) weights4(s, 2 * x + (i >> 1), mc);
      }
      p[x] = pack16(s, x);
    }
    if (MASK) {
      __builtin_amdgcn_sched_barrier(0);
      product_masked(vt, p, t);
      hide(s2, t + 1);
      raise(maximum(s2));
    } else {
      float mx = -INFINITY;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        __builtin_amdgcn_sched_barrier(0);
        if (x < 3)
#pragma unroll
          for (int i = 0; i < 4; ++i) f[(x + 1) & 1][i] = v_op(vt, x + 1, i, va);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          o[i] = mfma(f[x & 1][i], p[x], o[i]);
          const int y = 4 * x + i;
          mx = fmaxf(fmaxf(mx, s2[y >> 3][(y & 7) * 2]), s2[y >> 3][(y & 7) * 2 + 1]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      raise(mx);
    }
  };
  using B0 = std::false_type;
  using B1 = std::true_type;
  f32x16 sa[2], sb[2];
  __syncthreads();                                     // the piece before has left the LDS
  if (n_tiles > 0) {
    next = fetch(0);
    issue(c.k, k_off, s_k0, 0, next);
    issue(c.v, v_off, s_v0, 0, next);
    next = fetch(1);
    issue(c.k, k_off, s_k1, 1, next);
    after = fetch(2);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (!idle) {
      scores(s_k0, sa);
      if (n_full < 1) hide(sa, 0);
      raise(maximum(sa));
    }
    int t = 0;
    for (; t + 2 < n_full; t += 2) {
      turn(B0{}, std::false_type{}, t, sa, sb);
      turn(B1{}, std::false_type{}, t + 1, sb, sa);
    }
    for (; t + 2 < n_tiles; t += 2) {
      turn(B0{}, std::true_type{}, t, sa, sb);
      turn(B1{}, std::true_type{}, t + 1, sb, sa);
    }
    const bool odd = t + 1 < n_tiles;
    if (odd) {
      turn(B0{}, std::true_type{}, t++, sa, sb);
      sa[0] = sb[0];
      sa[1] = sb[1];
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (!idle) {
      uint4 p[4];
      const float mc = reference();
#pragma unroll
      for (int j = 0; j < 8; ++j) weights4(sa, j, mc);
#pragma unroll
      for (int h = 0; h < 4; ++h) p[h] = pack16(sa, h);
      if (odd) product_masked(s_v1, p, t);
      else product_masked(s_v0, p, t);
    }
  }

  // ---- results ---------------------------------------------------------------------
  if (!mine) continue;
  const float sum = add_xor32(l);                      // lanes l and l ^ 32 hold the same row
  const bool none = m == -INFINITY;
  const float mc = none ? -INFINITY : m * cs;
  if (pc.slot >= 0) {
    float* slot = a.slots + (size_t)pc.slot * 4;
    const int at = row - pc.row0;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(slot + (size_t)at * kD + d * 32 + 8 * i + 4 * hi) =
            make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
    if (hi == 0) {
      slot[kTileRows * kD + at] = mc;
      slot[kTileRows * (kD + 1) + at] = sum;
    }
    continue;
  }
  const float inv = none ? 0.f : 1.f / sum;
  char* out = a.out + qrow;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : o[d][4 * i + e] * inv;
      pg_put4((uint16_t*)nullptr, out + (d * 32 + 8 * i + 4 * hi) * 2, x[0], x[1], x[2], x[3]);
    }
  if (a.lse && hi == 0) a.lse[qrow / kRB] = none ? -INFINITY : (mc + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

template <int G>
hipError_t tile(const PagedAttn& a, hipStream_t stream) {
  paged_tile_kernel<G><<<a.n, kTileThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

static_assert(kTileRows == kTileThreads / 2, "32 new rows per wave");

hipError_t launch_paged_tile(int G, const PagedAttn& a, hipStream_t s) {
  return G == 1 ? tile<1>(a, s) : G == 2 ? tile<2>(a, s) : G == 4 ? tile<4>(a, s) : tile<8>(a, s);
}

}  // namespace catekv
