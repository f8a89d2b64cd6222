// Attention of chunks of new tokens over caches in pages (gfx950).
//
// A workgroup of 8 waves takes 256 (fp32: 128) new rows of one view's group and walks over its
// cached rows in tiles, K and V staged in LDS by global-to-LDS loads, two stages.  The
// softmax runs online.
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

template <> struct Ops<uint16_t> {
  static constexpr int kWaves = 8, kTile = 64, kSeg = 16, kQ = 8;
  static constexpr int kVSwz = 2;                    // V: chunk ^ (row & 3) << 2
  // Q as the operand of 16 dims a step: dims 16 ks + 8 (l / 32) + [0, 8)
  static __device__ __forceinline__ int q_off(int ks, int hi) { return ks * 32 + hi * 16; }
  static __device__ __forceinline__ f32x16 score(const uint4* kt, const uint4 (&q)[kQ], int kb, int lane) {
    const int row = kb * 32 + (lane & 31), hi = lane >> 5;
    f32x16 s = {};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const uint4 k = kt[row * kSeg + ((2 * ks + hi) ^ (row & 15))];
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[ks]), s, 0, 0, 0);
    }
    return s;
  }
  // P of a tile as operands: 16 cached rows a step
  struct P { uint4 w[kTile / 16]; };
  static __device__ __forceinline__ void pack(P& p, const f32x16 (&s)[kTile / 32]) {
#pragma unroll
    for (int st = 0; st < kTile / 16; ++st) {
      const f32x16& x = s[st / 2];
      const int o = (st & 1) * 8;
      p.w[st] = make_uint4(pg_pack2(x[o], x[o + 1]), pg_pack2(x[o + 2], x[o + 3]), pg_pack2(x[o + 4], x[o + 5]), pg_pack2(x[o + 6], x[o + 7]));
    }
  }
  // V^T of dims 32 db + l % 32 for the cached rows of step st: a transposing read hands
  // each 16 lanes 4 rows x 16 dims, column by column
  static __device__ __forceinline__ uint4 v_op(const uint4* vt, int st, int db, int lane) {
    const int hi = lane >> 5, g = (lane >> 4) & 1, i = lane & 15;
    const int row = st * 16 + hi * 4 + (i >> 2);
    const int chunk = (db * 4 + g * 2 + ((i >> 1) & 1)) ^ ((row & 3) << 2);
    const char* base = reinterpret_cast<const char*>(vt) + (row * kSeg + chunk) * 16 + (i & 1) * 8;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)base);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + 8 * kSeg * 16));
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    return make_uint4(x.x, x.y, y.x, y.y);
  }
  static __device__ __forceinline__ f32x16 mul(uint4 v, uint4 p, f32x16 o) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p), o, 0, 0, 0);
  }
  static constexpr int kSteps = kTile / 16;
  static __device__ __forceinline__ f32x16 pv(const uint4* vt, const P& p, int db, int lane, f32x16 o) {
#pragma unroll
    for (int st = 0; st < kSteps; ++st) o = mul(v_op(vt, st, db, lane), p.w[st], o);
    return o;
  }
  template <class F>
  static __device__ __forceinline__ uint4 each(uint4 v, F f) {
    return make_uint4(pg_both(v.x, f), pg_both(v.y, f), pg_both(v.z, f), pg_both(v.w, f));
  }
  static __device__ __forceinline__ bool any_bad(const uint4* vt, int lane) {
    uint32_t bad = 0;
    for (int st = 0; st < kSteps; ++st)
      for (int db = 0; db < 4; ++db) {
        const uint4 b = each(v_op(vt, st, db, lane), pg_bad16);
        bad |= b.x | b.y | b.z | b.w;
      }
    return bad != 0;
  }
  // as pv(), with what is not finite taken as 0, and counted by code for the rows that see it
  static __device__ __forceinline__ f32x16 pv_clean(const uint4* vt, const P& p, const P& seen, int db, int lane, f32x16 o, f32x16& n) {
    n = f32x16{};
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const uint4 v = v_op(vt, st, db, lane);
      o = mul(each(v, pg_clean16), p.w[st], o);
      n = mul(each(v, pg_code16), seen.w[st], n);
    }
    return o;
  }
};

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

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hi = lane >> 5;
  const PagedPiece pc = a.pieces[blockIdx.x];
  const PagedCache& c = a.c;
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
  // all of the wave's new rows see the cached rows below
  const int see_all = see0 + (pc.row0 + wave * 32) / G;
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
  bool big = false;                                    // in the wave: kPgBig
  const float cs = pg_log2_scale<T>(a.scale), thr = 8.0f / cs;

  // thread x's load i fills chunk i NT + x of the stage: row (i NT + x) / SEG, place x % SEG
  const int32_t* ids = c.table + (size_t)pc.view * c.max_pages;
  const int mask = (1 << c.page_log) - 1;
  const int lrow = wave * RPW + lane / SEG, place = lane & (SEG - 1);
  auto page_base = [&](int t) -> size_t {              // of cached row t (uniform)
    return pg_page(c, pg_entry(ids, t >> c.page_log));
  };
  const size_t row_zero = n_tiles > 0 ? page_base(0) * RB : 0;
  auto issue = [&](uint4* ks, uint4* vs, int t0) {
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

  auto use = [&](const uint4* ks, const uint4* vs, int t0) {
    f32x16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = X::score(ks, q, b, lane);
    const bool masked = t0 + TILE > see_all;           // uniform in the wave
    if (masked) {
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
      big = __builtin_amdgcn_ballot_w64(fabsf(m) * cs > kPgBig && m != -INFINITY) != 0;
      l *= corr;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= corr;
    }
    const float m0 = m == -INFINITY ? 0.f : m, mc = m0 * cs;
    if (big) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = fast_exp2((s[b][i] - m0) * cs);
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = fast_exp2(__builtin_fmaf(s[b][i], cs, -mc));
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) l += s[b][i];
    typename X::P p;
    X::pack(p, s);
    if (masked && __builtin_amdgcn_ballot_w64(X::any_bad(vs, lane))) {
      // 0 * NaN: what is not finite reaches only the new rows that see it
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

  if (n_tiles > 0) issue(s_k0, s_v0, pc.t0);
  for (int t = 0; t < n_tiles; t += 2) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();                                   // stage 0 is there, and nobody reads stage 1 any more
    if (t + 1 < n_tiles) issue(s_k1, s_v1, pc.t0 + (t + 1) * TILE);
    if (!idle) use(s_k0, s_v0, pc.t0 + t * TILE);
    if (t + 1 >= n_tiles) break;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (t + 2 < n_tiles) issue(s_k0, s_v0, pc.t0 + (t + 2) * TILE);
    if (!idle) use(s_k1, s_v1, pc.t0 + (t + 1) * TILE);
  }
  if (!mine) return;
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
    return;
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

// Joins the partial slots of rows that were cut.  A row has 32 lanes per group (4 dims
// each) and S groups, which take every S-th part; a workgroup has 8 / S rows.
template <typename T, int G, int S>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedAttn a, int first, int blocks) {
  constexpr int ROWS = kJoinRows / S;
  __shared__ float s_x[S][ROWS][kD], s_l[S][ROWS], s_m[S][ROWS];
  const int ji = blockIdx.x / blocks;
  const PagedJoin j = a.joins[first + ji];
  const int lane = threadIdx.x & 31, row = (threadIdx.x >> 5) % ROWS, g = (threadIdx.x >> 5) / ROWS;
  const int at = (blockIdx.x - ji * blocks) * ROWS + row, r = j.row0 + at;
  const bool mine = at < j.rows && r < j.n_new * G;
  const float* slot = a.slots + (size_t)j.slot * 4;
  const size_t step = paged_slot_floats(j.rows);
  const float* ms = slot + (size_t)j.rows * kD + (mine ? at : 0);
  float M = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  if (mine) {
    // the largest of the group's parts, 32 at a time
    for (int p = g + lane * S; p < j.n_parts; p += 32 * S) M = fmaxf(M, ms[p * step]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
#pragma unroll 4
    for (int p = g; p < j.n_parts; p += S) {
      const float mp = ms[p * step], lp = ms[p * step + j.rows];
      const float4 v = *reinterpret_cast<const float4*>(slot + p * step + (size_t)at * kD + lane * 4);
      const bool some = mp != -INFINITY;               // a part without rows holds zeros
      const float w = some ? fast_exp2(mp - M) : 0.f;
      l += w * lp;
      x[0] += w * v.x;
      x[1] += w * v.y;
      x[2] += w * v.z;
      x[3] += w * v.w;
    }
  }
  if (S > 1) {
    *reinterpret_cast<float4*>(&s_x[g][row][lane * 4]) = make_float4(x[0], x[1], x[2], x[3]);
    if (lane == 0) {
      s_m[g][row] = M;
      s_l[g][row] = l;
    }
    __syncthreads();
    if (g > 0) return;
    M = -INFINITY;
#pragma unroll
    for (int i = 0; i < S; ++i) M = fmaxf(M, s_m[i][row]);
    l = x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const float mi = s_m[i][row], w = mi == -INFINITY ? 0.f : fast_exp2(mi - M);
      const float4 v = *reinterpret_cast<const float4*>(&s_x[i][row][lane * 4]);
      l += w * s_l[i][row];
      x[0] += w * v.x;
      x[1] += w * v.y;
      x[2] += w * v.z;
      x[3] += w * v.w;
    }
  }
  if (!mine) return;
  const bool none = M == -INFINITY;
  const float inv = none ? 0.f : 1.f / l;
  const int tok = r / G, h = j.view % a.c.hkv;
  const size_t q = (size_t)(j.tok0 + tok) * a.hq + h * G + (r - tok * G);
  pg_put4((T*)nullptr, a.out + (q * kD + lane * 4) * sizeof(T), x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if (a.lse && lane == 0) a.lse[q] = none ? -INFINITY : (M + __builtin_amdgcn_logf(l)) * kLn2;
}

template <typename T, int G>
hipError_t tile(const PagedAttn& a, hipStream_t stream) {
  paged_tile_kernel<T, G><<<a.n, Ops<T>::kWaves * 64, 0, stream>>>(a);
  return hipGetLastError();
}
// Joins first ... first + n of at most `rows` rows each.
template <typename T, int G>
hipError_t join(const PagedAttn& a, int first, int n, int rows, int parts, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const int per = paged_join_rows(parts), blocks = (rows + per - 1) / per;
  if (per == kJoinRows) paged_join_kernel<T, G, 1><<<n * blocks, kJoinThreads, 0, stream>>>(a, first, blocks);
  else paged_join_kernel<T, G, kJoinRows><<<n * blocks, kJoinThreads, 0, stream>>>(a, first, blocks);
  return hipGetLastError();
}
template <typename T>
hipError_t tile_g(int G, const PagedAttn& a, hipStream_t s) {
  return G == 1 ? tile<T, 1>(a, s) : G == 2 ? tile<T, 2>(a, s) : G == 4 ? tile<T, 4>(a, s) : tile<T, 8>(a, s);
}
template <typename T>
hipError_t join_g(int G, const PagedAttn& a, int first, int n, int rows, int parts, hipStream_t s) {
  return G == 1 ? join<T, 1>(a, first, n, rows, parts, s) : G == 2 ? join<T, 2>(a, first, n, rows, parts, s)
       : G == 4 ? join<T, 4>(a, first, n, rows, parts, s) : join<T, 8>(a, first, n, rows, parts, s);
}

}  // namespace

int paged_tile_rows(int dtype) { return 32 * (dtype == CATEKV_BF16 ? Ops<uint16_t>::kWaves : Ops<float>::kWaves); }

hipError_t launch_paged_tile(int dtype, int G, const PagedAttn& a, hipStream_t stream) {
  return dtype == CATEKV_BF16 ? tile_g<uint16_t>(G, a, stream) : tile_g<float>(G, a, stream);
}
hipError_t launch_paged_join(int dtype, int G, const PagedAttn& a, int first, int n, int rows, int parts, hipStream_t stream) {
  return dtype == CATEKV_BF16 ? join_g<uint16_t>(G, a, first, n, rows, parts, stream)
                              : join_g<float>(G, a, first, n, rows, parts, stream);
}

}  // namespace catekv
