// Attention of chunks of new tokens over caches in pages, fp32 (gfx950): bound by the
// fp32 products (v_mfma_f32_32x32x2_f32, 64 cycles for 4096 operations).
//
// A workgroup of 4 waves takes 128 new rows of one view's group (row = token * G + head),
// 32 per wave, and walks over the view's cached rows in tiles of 32 that global-to-LDS
// loads bring in, one tile ahead.  Two workgroups share a compute unit: what one waits for
// and its softmax lie under the other's products.
//
// Scores are S^T = K Q^T: lane l holds new row l % 32 and, in register i, cached row 8 (i / 4)
// + 4 (l / 32) + i % 4, which is how O^T = V^T P^T takes P: register i of both lane halves is
// a step of two cached rows, 8 (i / 4) + i % 4 and the one 4 behind it.
//
// 333 new tokens over 4099 rows, 32 heads over 8: 21.5 GFLOP in 200 us, 107 TFLOP/s where a
// large library product reaches 153; 6% are rows that only fill the last of 11 tiles of
// 128, and the matrix cores are busy for two thirds of the cycles (one workgroup of twice
// the rows per compute unit, with spills: 380 us).
#include <type_traits>

#include "paged_math.h"

namespace catekv {
namespace {

typedef pg_f32x16 f32x16;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr int kTile = 32;                             // cached rows of a tile
constexpr int kRB = kD * 4;                           // bytes of a row
constexpr int kSeg = kRB / 16;                        // 16-byte chunks of a row
constexpr int kStage = kTile * kSeg;                  // chunks of a tile
constexpr int kLoads = kStage / kThreads;             // DMA per thread and tile, K and V each
static_assert(kTileRowsF32 == kWaves * 32, "32 new rows per wave");

__device__ __forceinline__ float el(const uint4& v, int i) {
  return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
}
__device__ __forceinline__ f32x16 mfma(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

template <int G>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_tile_f32_kernel(PagedAttn a) {
  __shared__ uint4 s_k0[kStage], s_v0[kStage], s_k1[kStage], s_v1[kStage];
  __shared__ int s_bad;
  const PagedCache& c = a.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mask = (1 << c.page_log) - 1;
  const float cs = a.log2_scale, thr = a.rise;
  int tag = 0;                                         // of the masked tile
  if (threadIdx.x == 0) s_bad = 0;

  for (int w = a.workers[blockIdx.x]; w < a.workers[blockIdx.x + 1]; ++w) {
    uint32_t lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                     // nothing of a piece is kept in registers for the next
    const int hi = lane >> 5;
    const PagedPiece pc = a.pieces[w];
    const int L = __builtin_amdgcn_readfirstlane(pg_rows(c, c.lens[pc.view], pc.max_rows));
    const int n_rows = pc.n_new * G;
    const int see0 = L - pc.n_new + 1;                 // cached rows that the first new token sees
    const int t_end = min(pc.t1, see0 + (min(pc.row0 + kTileRowsF32, n_rows) - 1) / G);
    const int n_tiles = max(0, (t_end - pc.t0 + kTile - 1) / kTile);
    const int n_full = max(0, (min(see0 + pc.row0 / G, t_end) - pc.t0) / kTile);   // that all new rows see in full
    const bool idle = pc.row0 + wave * 32 >= n_rows;   // none of the wave's rows exists
    const int row = pc.row0 + wave * 32 + (lane & 31);
    const bool mine = row < n_rows;
    const int tok = mine ? row / G : 0, h = pc.view % c.hkv;
    const int see = mine ? see0 + tok : 0;
    const size_t qrow = ((size_t)(pc.tok0 + tok) * a.hq + h * G + (mine ? row - tok * G : 0)) * kRB;
    // Q as the operand of two dims a step: register e of chunk u holds dim 8 u + 4 hi + e
    uint4 q[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) q[u] = pg_scale_q((const float*)nullptr, ldg16(a.q + qrow + u * 32 + hi * 16), a.scale);

    // Load i of a wave fills rows 8 i + 2 wave + [0, 2) of a tile, which never lie in two pages.
    // K lies with chunk ch of row r at place ch ^ (r & 15), V as it is.
    const int32_t* ids = c.table + (size_t)pc.view * c.max_pages;
    const int wrow = wave * 2, y = lane >> 5, place = lane & 31;
    auto issue = [&](uint4* ks, uint4* vs, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = pc.t0 + t * kTile + 8 * i + wrow;
        const size_t at = (pg_page(c, pg_entry(ids, min(r >> c.page_log, c.max_pages - 1))) + (r & mask)) * kRB;
        const int kc = place ^ ((8 * i + wrow + y) & 15);
        __builtin_amdgcn_global_load_lds(c.k + at + (y * kSeg + kc) * 16, (lds_void*)&ks[i * kThreads + wave * 64], 16, 0, 0);
        __builtin_amdgcn_global_load_lds(c.v + at + (y * kSeg + place) * 16, (lds_void*)&vs[i * kThreads + wave * 64], 16, 0, 0);
      }
    };

    f32x16 o[4] = {};
    float m = -INFINITY, l = 0.f, cw = cs;             // cw: pg_factor()
    bool purged = false;

    auto step = [&](auto stage, int t) __attribute__((always_inline)) {
      constexpr int B = decltype(stage)::value;
      const uint4* kt = B ? s_k1 : s_k0;
      uint4* vt = B ? s_v1 : s_v0;
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();                                 // the tile is there, and nobody reads the other stage
      if (t + 1 < n_tiles) issue(B ? s_k0 : s_k1, B ? s_v0 : s_v1, t + 1);
      const int r0 = pc.t0 + t * kTile;
      if (t >= n_full) {
        // 0 * NaN is NaN: V that is not finite is taken out of a masked tile, and goes into the
        // sums of the new rows that see it at the piece's end.  A thread looks at its part.
        ++tag;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad = bad || pg_bad32(el(vt[i * kThreads + threadIdx.x], e));
        if (bad) s_bad = tag;
        barrier_lds_only();
        if (s_bad == tag) {
          purged = true;
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            uint4& x = vt[i * kThreads + threadIdx.x];
            x = make_uint4(pg_bad32(el(x, 0)) ? 0u : x.x, pg_bad32(el(x, 1)) ? 0u : x.y, pg_bad32(el(x, 2)) ? 0u : x.z,
                           pg_bad32(el(x, 3)) ? 0u : x.w);
          }
          barrier_lds_only();
        }
      }
      if (idle) return;
      f32x16 s = {};
      {
        const int kr = lane & 31;
        const char* base = reinterpret_cast<const char*>(kt) + kr * kRB;
        uint32_t x = (hi ^ (kr & 15)) * 16;
        asm volatile("" : "+v"(x));                    // places are formed anew, not kept
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          const uint4 k = *reinterpret_cast<const uint4*>(base + (x ^ (u * 32)));
#pragma unroll
          for (int e = 0; e < 4; ++e) s = mfma(el(k, e), el(q[u], e), s);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = r0 + 8 * (i >> 2) + 4 * hi + (i & 3) < see ? s[i] : -INFINITY;
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i]);
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
      for (int i = 0; i < 16; ++i) {
        s[i] = fast_exp2(__builtin_fmaf(s[i], cw, -mc));
        l += s[i];
      }
      const float* v = reinterpret_cast<const float*>(vt) + 4 * hi * kD + (lane & 31);
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] = mfma(v[(8 * (i >> 2) + (i & 3)) * kD + d * 32], s[i], o[d]);
    };
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;
    __syncthreads();                                   // the piece before has left the LDS
    if (n_tiles > 0) issue(s_k0, s_v0, 0);
    for (int t = 0; t < n_tiles; t += 2) {
      step(S0{}, t);
      if (t + 1 < n_tiles) step(S1{}, t + 1);
    }

    l = add_xor32(l);                                  // lanes l and l ^ 32 hold the same row
    float sums[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) sums[i] = o[i >> 4][i & 15];
    const bool unusual = __builtin_amdgcn_ballot_w64(l == l && pg_unusual(sums));
    if (mine) {
      const float top = pg_top(m, l);
      const bool none = top == -INFINITY;
      // a partial result is taken as it is, a whole one divided by its sum
      const bool part = pc.slot >= 0;
      const float inv = part ? 1.f : none ? 0.f : 1.f / l;
      const int at = row - pc.row0;
      float* out = part ? a.slots + (size_t)pc.slot * 4 + (size_t)at * kD : reinterpret_cast<float*>(a.out + qrow);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = !part && none ? 0.f : o[d][4 * i + e] * inv;
          *reinterpret_cast<float4*>(out + d * 32 + 8 * i + 4 * hi) = make_float4(f[0], f[1], f[2], f[3]);
        }
      if (hi == 0 && part) {
        float* slot = a.slots + (size_t)pc.slot * 4;
        slot[kTileRowsF32 * kD + at] = top;
        slot[kTileRowsF32 * (kD + 1) + at] = l;
      } else if (hi == 0 && a.lse) {
        a.lse[qrow / kRB] = pg_lse(top, l, cs);
      }
    }
    if (unusual || purged) {                           // only masked tiles have V left out of finite sums
      const uint64_t fine = __builtin_amdgcn_ballot_w64(m > -INFINITY && l == l);
      const int end = min(pc.t0 + n_tiles * kTile, see0 + (min(pc.row0 + wave * 32 + 32, n_rows) - 1) / G);
      const RestoreAt to = {unusual ? pc.t0 : pc.t0 + n_full * kTile, end, see0, pc.row0 + wave * 32, 32, n_rows, (int)~fine, a.hq,
                            (size_t)pc.tok0 * a.hq + h * G,
                            pc.slot >= 0 ? a.slots + (size_t)pc.slot * 4 + (size_t)wave * 32 * kD : nullptr};
      pg_restore<float, G>(c, pc.view, a.q, a.scale, a.out, to);
    }
  }
}

template <int G>
hipError_t tile(const PagedAttn& a, hipStream_t stream) {
  paged_tile_f32_kernel<G><<<a.n, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_tile_f32(int G, const PagedAttn& a, hipStream_t s) {
  return G == 1 ? tile<1>(a, s) : G == 2 ? tile<2>(a, s) : G == 4 ? tile<4>(a, s) : tile<8>(a, s);
}

}  // namespace catekv
