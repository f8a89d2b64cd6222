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
// Weights are rounded to bf16 for their product with V (2^-8 of each; their sum is of the
// unrounded ones): against 64 bits 0.0020, as a root mean square over the values', instead of
// the 0.0017 of the result's own rounding.  In two parts, as the few-token kernel has them, they would take three
// products where two bound the kernel now.
//
// The softmax runs online, one tile behind: between the products of tile t + 1's scores
// the vector unit forms the weights of tile t, and while these meet V it takes the
// maxima of tile t + 1.  A wave issues in order, so the two are laid between each other
// in the program, and scheduling barriers keep them there.
//
// 2048 new tokens, the last of 32768 rows, 32 heads over 8: 1065 GFLOP in 940 to 1030 us, 1.03 to
// 1.13 PFLOP/s where a large library product reaches 1.10 (products beside each other
// without softmax: 1.6 to 1.9).  The matrix cores are busy for 52% of the cycles, the vector
// unit issues in 45%; no LDS bank conflicts.  Larger tiles of new rows do not fit the
// registers; 128 to a workgroup would read K and V from LDS twice as often.
#include <type_traits>

#include "paged_stream.h"

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

// Weights of 16 cached rows, number h of 64, as an operand.
__device__ __forceinline__ uint4 pack16(const f32x16 (&x)[2], int h) {
  const f32x16& y = x[h >> 1];
  const int o = (h & 1) * 8;
  return make_uint4(pg_pack2(y[o], y[o + 1]), pg_pack2(y[o + 2], y[o + 3]), pg_pack2(y[o + 4], y[o + 5]), pg_pack2(y[o + 6], y[o + 7]));
}

constexpr int kMixedQ = kStreamWaves * R * kPad / 4;   // 16-byte units of the streaming waves' sums
static_assert(kTileThreads == kStreamThreads && kMixedQ >= kTileRows * kSeg, "one launch for both");

// What is the same for all lanes about a piece.
struct Piece {
  int32_t view, tok0, n_new, row0, t0, slot;
  int32_t see0;                                        // cached rows that the first new token sees
  int32_t n_tiles, n_full;                             // tiles; those that every new row sees in full come first
};

// MIXED: a batch with sequences of few new tokens, too; the workgroups behind those of the
// tiles take them.
template <int G, bool MIXED>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_tile_kernel(PagedAttn a) {
  // aligned so that they come first: their places fit the reads' 16-bit offsets
  __shared__ __attribute__((aligned(1024))) uint4 s_k0[kStage], s_k1[kStage], s_v0[kStage], s_v1[kStage];
  __shared__ uint4 s_q[MIXED ? kMixedQ : kTileRows * kSeg];   // new rows, laid out as K is
  __shared__ int s_bad;

  if (MIXED && (int)blockIdx.x >= a.n) {
    constexpr int BATCH = kStage / (R * kSeg);
    float (*ml)[kStreamWaves][R] = reinterpret_cast<float (*)[kStreamWaves][R]>(s_v0);
    const int32_t* share = a.seg_workers + ((int)blockIdx.x - a.n);
    stream_share<uint16_t, G, BATCH>(a, a.segs, share[0], share[1],
                                     {reinterpret_cast<Seg (*)[BATCH]>(s_v1), reinterpret_cast<uint4 (*)[BATCH][R][kSeg]>(s_k0),
                                      reinterpret_cast<float (*)[kStreamWaves][R][kPad]>(s_q), ml, ml + 1});
    return;
  }

  const PagedCache& c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int last = a.workers[blockIdx.x + 1];
  const int mask = (1 << c.page_log) - 1;
  const int wrow = wave * 4;
  const float cs = a.log2_scale, thr = a.rise;
  constexpr int kLoads = kStage / kTileThreads;        // DMA per thread and tile, K and V each

  uint32_t lane = threadIdx.x & 63;
  // Places of the operands in LDS, and of a lane's 16 bytes in 4 rows of a tile.  own() makes
  // them new values to the compiler, which would otherwise keep what it makes of them, and
  // every step's address, in registers of their own throughout.
  uint32_t ka = k_lane(lane), va = v_lane(lane);
  const char* k_at = c.k + (lane >> 4) * kRB + ((lane & 15) ^ ((wrow + (lane >> 4)) & 15)) * 16;
  const char* v_at = c.v + (lane >> 4) * kRB + ((lane & 15) ^ ((lane >> 4) << 2)) * 16;
  auto own = [&]() __attribute__((always_inline)) { asm volatile("" : "+v"(ka), "+v"(va), "+v"(lane)); };

  // ---- a piece's way in ------------------------------------------------------------
  auto open = [&](int w) __attribute__((always_inline)) {
    const PagedPiece p = pg_scalar(a.pieces + w);
    Piece x;
    x.view = p.view;
    x.tok0 = p.tok0;
    x.n_new = p.n_new;
    x.row0 = p.row0;
    x.t0 = p.t0;
    x.slot = p.slot;
    const int L = pg_rows(c, pg_scalar(c.lens + p.view), p.max_rows);
    x.see0 = L - p.n_new + 1;
    const int t_end = min(p.t1, x.see0 + (min(p.row0 + kTileRows, p.n_new * G) - 1) / G);
    // without a cached row that is seen: one tile, all of it masked
    x.n_tiles = max(1, (t_end - p.t0 + kTile - 1) / kTile);
    x.n_full = max(0, (min(x.see0 + p.row0 / G, t_end) - p.t0) / kTile);
    return x;
  };
  // Tile t's DMA: load i of a wave fills rows 32 i + 4 wave + [0, 4) of it, which never lie in
  // two pages.  Rows past the view's come from where its table's clamped entries point;
  // masked tiles let none of them through.
  struct Ids { int id[kLoads]; };
  auto fetch = [&](const Piece& x, int t) __attribute__((always_inline)) {
    Ids y;
    const int r = x.t0 + min(t, x.n_tiles - 1) * kTile + wrow;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      y.id[i] = pg_entry(c.table + (size_t)x.view * c.max_pages, min((r + 32 * i) >> c.page_log, c.max_pages - 1));
    return y;
  };
  auto issue = [&](const Piece& x, const char* at, uint4* stage, int t, const Ids& y) __attribute__((always_inline)) {
    const int r = x.t0 + min(t, x.n_tiles - 1) * kTile + wrow;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const size_t off = (pg_page(c, y.id[i]) + ((r + 32 * i) & mask)) * kRB;
      __builtin_amdgcn_global_load_lds(at + off, (lds_void*)&stage[i * kTileThreads + wave * 64], 16, 0, 0);
    }
  };

  // ---- the softmax's state and its steps ---------------------------------------------
  uint4 q[8];
  f32x16 o[4];
  float m, l, cw;                                      // cw: pg_factor()
  int see;                                             // cached rows that this lane's new row sees
  // The wave's new rows, 4 per load; those past the last are the first token's.
  auto queries = [&](const Piece& x) __attribute__((always_inline)) {
    const int n = x.n_new * G;
    const char* base = a.q + ((size_t)x.tok0 * a.hq + (x.view % c.hkv) * G) * kRB;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int y = 4 * i + (lane >> 4), r = x.row0 + wave * 32 + y;
      const int tok = r < n ? r / G : 0, g = r < n ? r - tok * G : 0;
      const char* from = base + ((size_t)tok * a.hq + g) * kRB + ((lane & 15) ^ (y & 15)) * 16;
      __builtin_amdgcn_global_load_lds(from, (lds_void*)&s_q[(wave * 32 + 4 * i) * kSeg], 16, 0, 0);
    }
  };
  auto scores = [&](const uint4* kt, f32x16 (&s)[2]) __attribute__((always_inline)) {
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = mfma(k_op(kt, kb, ks, ka), q[ks], s[kb]);
  };
  auto hide = [&](f32x16 (&s)[2], int r0) __attribute__((always_inline)) {
    const int d = see - r0 - 4 * (int)(lane >> 5);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = kb * 32 + 8 * (i >> 2) + (i & 3) < d ? s[kb][i] : -INFINITY;
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
  // weights of registers 2 j and 2 j + 1 of both score blocks laid end to end
  auto weights2 = [&](f32x16 (&s)[2], int j, float mc) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float w = fast_exp2(__builtin_fmaf(s[j >> 3][(j & 7) * 2 + e], cw, -mc));
      s[j >> 3][(j & 7) * 2 + e] = w;
      l += w;
    }
  };
  auto reference = [&]() __attribute__((always_inline)) { return m == -INFINITY ? 0.f : m * cw; };
  auto weights = [&](f32x16 (&s)[2], uint4 (&p)[4]) __attribute__((always_inline)) {
    const float mc = reference();
#pragma unroll
    for (int x = 0; x < 4; ++x) {
#pragma unroll
      for (int i = 0; i < 4; ++i) weights2(s, 4 * x + i, mc);
      p[x] = pack16(s, x);
    }
  };
  auto product = [&](const uint4* vt, const uint4 (&p)[4]) __attribute__((always_inline)) {
    uint4 f[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[0][i] = v_op(vt, 0, i, va);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      __builtin_amdgcn_sched_barrier(0);
      if (x < 3)
#pragma unroll
        for (int i = 0; i < 4; ++i) f[(x + 1) & 1][i] = v_op(vt, x + 1, i, va);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = mfma(f[x & 1][i], p[x], o[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // ---- V that is not finite in masked tiles ------------------------------------------
  // 0 * NaN is NaN: such values are taken out of the tile, and go into the sums of the new
  // rows that see them at the piece's end.  Every thread looks at its part of the tile; a
  // barrier later all waves know.
  int tag = 0;                                         // of the masked tile
  auto look = [&](const uint4* vt) __attribute__((always_inline)) {
    ++tag;
    pg_u16x2 top = {0, 0};                                // the largest magnitude, as bits
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint4 x = vt[i * kTileThreads + wave * 64 + lane];
      const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(pg_u16x2, y[e] & 0x7fff7fffu));
    }
    if (top[0] >= 0x7f80 || top[1] >= 0x7f80) s_bad = tag;
  };
  bool purged = false;                                 // a tile of the piece
  auto purge = [&](uint4* vt) __attribute__((always_inline)) {
    barrier_lds_only();
    if (s_bad != tag) return;
    purged = true;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      uint4& x = vt[i * kTileThreads + wave * 64 + lane];
      x = make_uint4(pg_both(x.x, pg_clean16), pg_both(x.y, pg_clean16), pg_both(x.z, pg_clean16), pg_both(x.w, pg_clean16));
    }
    barrier_lds_only();
  };
  Ids next = {}, after = {};                           // pages of the tile after the one whose scores are there, and of the one behind

  // ---- turns -----------------------------------------------------------------------
  // At the head of turn t: tile t's scores are in s and their maxima taken in; K of t + 1
  // and V of t are in LDS or on their way.  Leaves tile t + 1's scores in s2.
  // The first masked turn asks for the next piece's new rows.
  auto turn = [&](auto stage, auto mask_tag, Piece& x, const Piece* y, int t, bool idle, f32x16 (&s)[2], f32x16 (&s2)[2]) __attribute__((always_inline)) {
    constexpr bool B = decltype(stage)::value, MASK = decltype(mask_tag)::value;
    const uint4* kt = B ? s_k0 : s_k1;
    uint4* vt = B ? s_v1 : s_v0;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    issue(x, k_at, B ? s_k1 : s_k0, t + 2, after);
    issue(x, v_at, B ? s_v0 : s_v1, t + 1, next);
    next = after;
    after = fetch(x, t + 3);
    own();
    if (MASK && y) queries(*y);
    const bool part = MASK && t >= x.n_full;           // some new rows do not see all of V's tile
    if (part) look(vt);
    // Operands come in fours, one four ahead: their wait is then for reads that have had
    // four products' time (a wait counts all LDS reads on their way).  A product leaves the
    // vector unit room for four instructions or so: two weights beside each of the scores'
    // first twelve and of V's first four, the maxima beside V's (all weights beside the
    // scores' products, four beside every other one: 1.4% longer).
    uint4 p[4], f[2][4];
    if (!idle) {
      const float mc = reference();
#pragma unroll
      for (int i = 0; i < 4; ++i) f[0][i] = k_op(kt, i & 1, i >> 1, ka);
      s2[0] = s2[1] = f32x16{};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (y < 3) f[(y + 1) & 1][i] = k_op(kt, i & 1, 2 * y + 2 + (i >> 1), ka);
          else if (!MASK) f[0][i] = v_op(vt, 0, i, va);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          s2[i & 1] = mfma(f[y & 1][i], q[2 * y + (i >> 1)], s2[i & 1]);
          if (y < 3) weights2(s, 4 * y + i, mc);
        }
        if (y < 3) p[y] = pack16(s, y);
      }
      if (MASK) {
#pragma unroll
        for (int i = 0; i < 4; ++i) weights2(s, 12 + i, mc);
        p[3] = pack16(s, 3);
      }
    }
    if (part) purge(vt);
    if (idle) return;
    if (MASK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[0][i] = v_op(vt, 0, i, va);
      if (t + 1 >= x.n_full) hide(s2, x.t0 + (t + 1) * kTile);
    }
    const float mc = reference();
    float mx = -INFINITY;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      __builtin_amdgcn_sched_barrier(0);
      if (y < 3)
#pragma unroll
        for (int i = 0; i < 4; ++i) f[(y + 1) & 1][i] = v_op(vt, y + 1, i, va);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        o[i] = mfma(f[y & 1][i], p[y], o[i]);
        if (!MASK && y == 0) weights2(s, 12 + i, mc);
        if (!MASK && y == 1 && i == 0) p[3] = pack16(s, 3);
        const int z = 4 * y + i;
        mx = fmaxf(fmaxf(mx, s2[z >> 3][(z & 7) * 2]), s2[z >> 3][(z & 7) * 2 + 1]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    raise(mx);
  };
  using B0 = std::false_type;
  using B1 = std::true_type;

  // ---- the worker's pieces -----------------------------------------------------------
  // The next piece's new rows and K come in under this one's last turns and products, and its V under the
  // results' way out, which nothing waits for but the first turn.
  int w = a.workers[blockIdx.x];
  if (w >= last) return;                               // a worker without pieces
  Piece x = open(w);
  const Ids tile0 = fetch(x, 0);
  next = fetch(x, 1);
  queries(x);
  issue(x, k_at, s_k0, 0, tile0);
  issue(x, k_at, s_k1, 1, next);
  issue(x, v_at, s_v0, 0, tile0);
  if (threadIdx.x == 0) s_bad = 0;
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  for (;;) {
    own();
    {
      const int row = x.row0 + wave * 32 + (lane & 31);
      see = row < x.n_new * G ? x.see0 + row / G : 0;
    }
    const bool idle = x.row0 + wave * 32 >= x.n_new * G;   // none of the wave's rows exists
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] = f32x16{};
    m = -INFINITY;
    l = 0.f;
    cw = cs;
    f32x16 sa[2], sb[2];
    const bool more = w + 1 < last;
    const Piece y = open(more ? w + 1 : w);
    const Ids y0 = fetch(y, 0), y1 = fetch(y, 1);
    after = fetch(x, 2);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = k_op(s_q + wave * 32 * kSeg, 0, ks, ka);
    if (!idle) {
      scores(s_k0, sa);
      if (x.n_full < 1) hide(sa, x.t0);
      raise(maximum(sa));
    }
    int t = 0;
    for (; t + 2 < x.n_full; t += 2) {
      turn(B0{}, std::false_type{}, x, nullptr, t, idle, sa, sb);
      turn(B1{}, std::false_type{}, x, nullptr, t + 1, idle, sb, sa);
    }
    const int first = t;
    purged = false;
    for (; t + 2 < x.n_tiles; t += 2) {
      turn(B0{}, std::true_type{}, x, more && t == first ? &y : nullptr, t, idle, sa, sb);
      turn(B1{}, std::true_type{}, x, nullptr, t + 1, idle, sb, sa);
    }
    const bool odd = t + 1 < x.n_tiles;
    if (odd) {
      turn(B0{}, std::true_type{}, x, more && t == first ? &y : nullptr, t, idle, sa, sb);
      ++t;
      sa[0] = sb[0];
      sa[1] = sb[1];
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    own();
    if (more) {                                        // K's places are free
      if (t == first) queries(y);                      // there was no masked turn
      issue(y, k_at, s_k0, 0, y0);
      issue(y, k_at, s_k1, 1, y1);
    }
    uint4* vt = odd ? s_v1 : s_v0;
    uint4 p[4];
    look(vt);
    if (!idle) weights(sa, p);
    purge(vt);
    if (!idle) product(vt, p);
    if (more) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();                                 // they are there, and V's places are free
      issue(y, v_at, s_v0, 0, y0);
    }

    // ---- results -------------------------------------------------------------------
    const float sum = add_xor32(l);                    // lanes l and l ^ 32 hold the same row
    float sums[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) sums[i] = o[i >> 4][i & 15];
    const bool unusual = __builtin_amdgcn_ballot_w64(sum == sum && pg_unusual(sums));
    const int at = wave * 32 + (lane & 31), row = x.row0 + at;
    if (row < x.n_new * G) {
      const int hi = lane >> 5, tok = row / G;
      const size_t qrow = ((size_t)(x.tok0 + tok) * a.hq + (x.view % c.hkv) * G + (row - tok * G)) * kRB;
      const float top = pg_top(m, sum);
      const bool none = top == -INFINITY;
      if (x.slot >= 0) {
        float* slot = a.slots + (size_t)x.slot * 4;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<float4*>(slot + (size_t)at * kD + d * 32 + 8 * i + 4 * hi) =
                make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
        if (hi == 0) {
          slot[kTileRows * kD + at] = top;
          slot[kTileRows * (kD + 1) + at] = sum;
        }
      } else {
        const float inv = none ? 0.f : 1.f / sum;
        char* out = a.out + qrow;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 4; i += 2) {             // dims 32 d + 8 i + [0, 16): the lower lanes' 8, the upper ones' 8
            uint32_t y[2][2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int f = 0; f < 2; ++f) {
                const float u = o[d][4 * (i + e) + 2 * f] * inv, v = o[d][4 * (i + e) + 2 * f + 1] * inv;
                y[e][f] = none ? 0u : pg_pack2(u, v);
              }
            const auto lo = __builtin_amdgcn_permlane32_swap(y[0][0], y[1][0], false, false);
            const auto hi2 = __builtin_amdgcn_permlane32_swap(y[0][1], y[1][1], false, false);
            *reinterpret_cast<uint4*>(out + (d * 32 + 8 * (i + hi)) * 2) = make_uint4(lo[0], hi2[0], lo[1], hi2[1]);
          }
        if (a.lse && hi == 0) a.lse[qrow / kRB] = pg_lse(top, sum, cs);
      }
    }
    if (unusual || purged) {                           // only tiles that were looked at have V left out of finite sums
      const uint64_t fine = __builtin_amdgcn_ballot_w64(m > -INFINITY && sum == sum);
      const int n = x.n_new * G, end = min(x.t0 + x.n_tiles * kTile, x.see0 + (min(x.row0 + wave * 32 + 32, n) - 1) / G);
      const RestoreAt to = {unusual ? x.t0 : x.t0 + first * kTile, end, x.see0, x.row0 + wave * 32, 32, n, (int)~fine, a.hq,
                            (size_t)x.tok0 * a.hq + (x.view % c.hkv) * G,
                            x.slot >= 0 ? a.slots + (size_t)x.slot * 4 + (size_t)wave * 32 * kD : nullptr};
      pg_restore<uint16_t, G>(c, x.view, a.q, a.scale, a.out, to);
    }
    if (!more) break;
    ++w;
    x = y;
    next = y1;
  }
}

template <bool MIXED>
hipError_t tile(int G, const PagedAttn& a, hipStream_t stream) {
  const int n = a.n + (MIXED ? a.n_few : 0);
  if (G == 1) paged_tile_kernel<1, MIXED><<<n, kTileThreads, 0, stream>>>(a);
  else if (G == 2) paged_tile_kernel<2, MIXED><<<n, kTileThreads, 0, stream>>>(a);
  else if (G == 4) paged_tile_kernel<4, MIXED><<<n, kTileThreads, 0, stream>>>(a);
  else paged_tile_kernel<8, MIXED><<<n, kTileThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

static_assert(kTileRows == kTileThreads / 2, "32 new rows per wave");

hipError_t launch_paged_tile(int G, const PagedAttn& a, hipStream_t s) { return tile<false>(G, a, s); }
hipError_t launch_paged_mixed(int G, const PagedAttn& a, hipStream_t s) { return tile<true>(G, a, s); }

}  // namespace catekv
