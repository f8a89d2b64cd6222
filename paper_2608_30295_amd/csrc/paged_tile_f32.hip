// Attention of chunks of new tokens over caches in pages (gfx950).
//
// A workgroup of 8 waves takes 256 (fp32: 128) new rows of one view's group and walks over its
// cached rows in tiles, K and V staged in LDS by global-to-LDS loads, two stages.  The
// softmax runs online.
#include <type_traits>

#include "paged_math.h"

namespace catekv {
namespace {

typedef pg_f32x16 f32x16;
typedef pg_bf16x8 bf16x8;
typedef pg_s16x4 s16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// ---- what differs between the types ---------------------------------------------
// Scores: S^T = K Q^T, cached rows down, new rows across: lane l holds new row l % 32
// and, in register i, cached row 8 (i / 4) + 4 (l / 32) + i % 4 of a block of 32, so that
// a new row's maximum and sum are a lane's own but for one exchange of lane halves, and
// the registers are in place as the operand P^T of O^T = V^T P^T (a product does not
// ask in which order its terms come: the same order is taken for V).
template <typename T> struct Ops;

template <> struct Ops<float> {
  static constexpr int kWaves = 4, kTile = 32, kSeg = 32, kQ = 16;
  static constexpr int kVSwz = 0;
  // Q as the operand of 2 dims a step: register e of chunk u holds dim 8 u + 4 (l / 32) + e
  static __device__ __forceinline__ int q_off(int u, int hi) { return u * 32 + hi * 16; }
  static __device__ __forceinline__ float f(uint32_t x) { return __uint_as_float(x); }
  static __device__ __forceinline__ f32x16 score(const uint4* kt, const uint4 (&q)[kQ], int kb, int lane) {
    const int row = kb * 32 + (lane & 31), hi = lane >> 5;
    f32x16 s = {};
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const uint4 k = kt[row * kSeg + ((2 * u + hi) ^ (row & 15))];
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(f(k.x), f(q[u].x), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(f(k.y), f(q[u].y), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(f(k.z), f(q[u].z), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(f(k.w), f(q[u].w), s, 0, 0, 0);
    }
    return s;
  }
  struct P { f32x16 w; };
  static __device__ __forceinline__ void pack(P& p, const f32x16 (&s)[1]) { p.w = s[0]; }
  static constexpr int kSteps = 16;
  // step st: cached rows 8 (st / 4) + 4 (l / 32) + st % 4
  static __device__ __forceinline__ float v_op(const uint4* vt, int st, int db, int lane) {
    const int row = 8 * (st >> 2) + 4 * (lane >> 5) + (st & 3);
    return reinterpret_cast<const float*>(vt)[row * kD + db * 32 + (lane & 31)];
  }
  static __device__ __forceinline__ f32x16 pv(const uint4* vt, const P& p, int db, int lane, f32x16 o) {
#pragma unroll
    for (int st = 0; st < kSteps; ++st) o = __builtin_amdgcn_mfma_f32_32x32x2f32(v_op(vt, st, db, lane), p.w[st], o, 0, 0, 0);
    return o;
  }
  static __device__ __forceinline__ bool any_bad(const uint4* vt, int lane) {
    bool b = false;
    for (int st = 0; st < kSteps; ++st)
      for (int db = 0; db < 4; ++db) b = b || pg_bad32(v_op(vt, st, db, lane));
    return b;
  }
  static __device__ __forceinline__ f32x16 pv_clean(const uint4* vt, const P& p, const P& seen, int db, int lane, f32x16 o, f32x16& n) {
    n = f32x16{};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const float v = v_op(vt, st, db, lane);
      o = __builtin_amdgcn_mfma_f32_32x32x2f32(pg_bad32(v) ? 0.f : v, p.w[st], o, 0, 0, 0);
      n = __builtin_amdgcn_mfma_f32_32x32x2f32(pg_code32(v), seen.w[st], n, 0, 0, 0);
    }
    return o;
  }
};

template <typename T, int G>
__global__ __launch_bounds__(Ops<T>::kWaves * 64) void paged_tile_kernel(PagedAttn a) {
  using X = Ops<T>;
  constexpr int W = X::kWaves, NT = W * 64, TILE = X::kTile, SEG = X::kSeg, NB = TILE / 32;
  constexpr int RB = kD * (int)sizeof(T);              // bytes of a row
  constexpr int LD = TILE * SEG / NT;                  // loads of 16 bytes per thread, K and V each
  constexpr int RPW = 64 / SEG;                        // rows of a wave's load
  constexpr int R = W * 32;
  static_assert(LD * NT == TILE * SEG && 16 % RPW == 0, "");
  __shared__ uint4 s_k0[TILE * SEG], s_v0[TILE * SEG], s_k1[TILE * SEG], s_v1[TILE * SEG];

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
  const int r_end = min(pc.row0 + R, n_rows);          // past the piece's last new row
  const int t_end = min(pc.t1, see0 + (r_end - 1) / G);
  const int n_tiles = t_end > pc.t0 ? (t_end - pc.t0 + TILE - 1) / TILE : 0;

  const int r = pc.row0 + wave * 32 + (lane & 31);     // this lane's new row
  const bool mine = r < n_rows;
  const int tok = r / G;
  const int see = mine ? see0 + tok : 0;
  const bool idle = pc.row0 + wave * 32 >= n_rows;     // none of the wave's rows exists

  const int h = pc.view % c.hkv;
  const size_t qrow = mine ? ((size_t)(pc.tok0 + tok) * a.hq + h * G + (r - tok * G)) * RB : 0;
  uint4 q[X::kQ];
#pragma unroll
  for (int i = 0; i < X::kQ; ++i) {
    const uint4 x = ldg16(a.q + (mine ? qrow : (size_t)pc.tok0 * a.hq * RB) + X::q_off(i, hi));
    q[i] = mine ? pg_scale_q((const T*)nullptr, x, a.scale) : make_uint4(0, 0, 0, 0);
  }

  f32x16 o[4] = {};
  float m = -INFINITY, l = 0.f;
  const float cs = a.log2_scale, thr = a.rise;
  float cw = cs;                                       // of the weights: pg_factor()

  // thread x's load i fills chunk i NT + x of the stage: row (i NT + x) / SEG, place x % SEG
  const int32_t* ids = c.table + (size_t)pc.view * c.max_pages;
  const int mask = (1 << c.page_log) - 1;
  const int lrow = wave * RPW + lane / SEG, place = lane & (SEG - 1);
  auto page_base = [&](int t) -> size_t {              // of cached row t (uniform)
    return pg_page(c, pg_entry(ids, t >> c.page_log));
  };
  const size_t row_zero = n_tiles > 0 ? page_base(0) * RB : 0;
  auto issue = [&](uint4* ks, uint4* vs, int t0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int first = t0 + i * (NT / SEG) + wave * RPW;     // the wave's rows of this load
      const size_t base = page_base(min(first, L - 1));
      const int row = i * (NT / SEG) + lrow, t = t0 + row;
      const size_t at = t < L ? (base + (t & mask)) * RB : row_zero;   // rows past the view's are row 0
      const int kc = place ^ (row & 15), vc = X::kVSwz ? place ^ ((row & 3) << X::kVSwz) : place;
      __builtin_amdgcn_global_load_lds(c.k + at + kc * 16, (lds_void*)&ks[i * NT + wave * 64], 16, 0, 0);
      __builtin_amdgcn_global_load_lds(c.v + at + vc * 16, (lds_void*)&vs[i * NT + wave * 64], 16, 0, 0);
    }
  };

  auto use = [&](const uint4* ks, const uint4* vs, int t0, auto mask_tag) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mask_tag)::value;
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = X::score(ks, q, b, lane);
    if (MASK) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[b][i] = t0 + b * 32 + 8 * (i >> 2) + 4 * hi + (i & 3) < see ? s[b][i] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
    mx = max_xor32(mx);
    // the maximum moves where it grew by 8 powers of two (weights up to 2^8); from -inf always
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
    const float mc = m == -INFINITY ? 0.f : m * cw;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = fast_exp2(__builtin_fmaf(s[b][i], cw, -mc));
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) l += s[b][i];
    typename X::P p;
    X::pack(p, s);
    if (MASK && __builtin_amdgcn_ballot_w64(X::any_bad(vs, lane))) {
      typename X::P seen;
      f32x16 one[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) one[b][i] = t0 + b * 32 + 8 * (i >> 2) + 4 * hi + (i & 3) < see ? 1.f : 0.f;
      X::pack(seen, one);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f32x16 n;
        o[d] = X::pv_clean(vs, p, seen, d, lane, o[d], n);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] += pg_of_codes(n[i]);
      }
    } else {
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = X::pv(vs, p, d, lane, o[d]);
    }
  };

  // Tiles that every new row of the workgroup sees in full come first, the others are
  // masked.  One stage is used while the other is on its way; the barrier at a tile's
  // head says that it is there and that nobody reads the other any more.
  const int n_full = max(0, min(n_tiles, (min(see0 + pc.row0 / G, t_end) - pc.t0) / TILE));
  auto step = [&](auto stage, int t, auto mask_tag) __attribute__((always_inline)) {
    constexpr int B = decltype(stage)::value;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (t + 1 < n_tiles) issue(B ? s_k0 : s_k1, B ? s_v0 : s_v1, pc.t0 + (t + 1) * TILE);
    if (!idle) use(B ? s_k1 : s_k0, B ? s_v1 : s_v0, pc.t0 + t * TILE, mask_tag);
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  __syncthreads();                                     // the piece before has left the LDS
  if (n_tiles > 0) issue(s_k0, s_v0, pc.t0);
  int t = 0;
  for (; t + 2 <= n_full; t += 2) {
    step(S0{}, t, std::false_type{});
    step(S1{}, t + 1, std::false_type{});
  }
  for (; t < n_tiles; t += 2) {
    step(S0{}, t, std::true_type{});
    if (t + 1 < n_tiles) step(S1{}, t + 1, std::true_type{});
  }
  if (!mine) continue;
  l = add_xor32(l);                                    // lanes l and l ^ 32 hold the same row
  const float mc = m == -INFINITY ? -INFINITY : m * cs;
  if (pc.slot >= 0) {
    float* slot = a.slots + (size_t)pc.slot * 4;
    const int at = r - pc.row0;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(slot + (size_t)at * kD + d * 32 + 8 * i + 4 * hi) =
            make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
    if (hi == 0) {
      slot[R * kD + at] = mc;
      slot[R * (kD + 1) + at] = l;
    }
    continue;
  }
  const bool none = m == -INFINITY;
  const float inv = none ? 0.f : 1.f / l;
  char* out = a.out + qrow;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : o[d][4 * i + e] * inv;
      pg_put4((T*)nullptr, out + (d * 32 + 8 * i + 4 * hi) * (int)sizeof(T), x[0], x[1], x[2], x[3]);
    }
  if (a.lse && hi == 0)
    a.lse[(size_t)(pc.tok0 + tok) * a.hq + h * G + (r - tok * G)] = none ? -INFINITY : (mc + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

template <typename T, int G>
hipError_t tile(const PagedAttn& a, hipStream_t stream) {
  paged_tile_kernel<T, G><<<a.n, Ops<T>::kWaves * 64, 0, stream>>>(a);
  return hipGetLastError();
}
}  // namespace

static_assert(kTileRowsF32 == 32 * Ops<float>::kWaves, "");

hipError_t launch_paged_tile_f32(int G, const PagedAttn& a, hipStream_t s) {
  return G == 1 ? tile<float, 1>(a, s) : G == 2 ? tile<float, 2>(a, s) : G == 4 ? tile<float, 4>(a, s) : tile<float, 8>(a, s);
}

}  // namespace catekv
