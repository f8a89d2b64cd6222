// Partial results of attention over pages joined (gfx950).
#include "paged_math.h"

namespace catekv {
namespace {

// Joins the partial slots of rows that were cut.  A row has 32 lanes per group (4 dims
// each) and S groups, which take every S-th part; a workgroup has 8 / S rows.  Bound by
// dependent loads: a group that goes through 96 parts alone takes 23 us, eight that share
// them 4.7; up to 8 parts are left to one (4 to 9 us).
template <typename T, int G, int S>
__device__ __forceinline__ void join_rows(const PagedAttn& a, const PagedJoin& j, int block, float* s_all) {
  constexpr int ROWS = kJoinRows / S;
  float (*s_x)[ROWS][kD] = reinterpret_cast<float (*)[ROWS][kD]>(s_all);
  float (*s_l)[ROWS] = reinterpret_cast<float (*)[ROWS]>(s_all + kJoinRows * kD);
  float (*s_m)[ROWS] = s_l + S;
  const int lane = threadIdx.x & 31, row = (threadIdx.x >> 5) % ROWS, g = (threadIdx.x >> 5) / ROWS;
  const int at = block * ROWS + row, r = j.row0 + at;
  const bool mine = at < j.rows && r < j.n_new * G;
  const float* slot = a.slots + (size_t)j.slot * 4;
  const size_t step = paged_slot_floats(j.rows);
  const float* ms = slot + (size_t)j.rows * kD + (mine ? at : 0);
  float M = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  // Sums that are not finite are formed anew, with what is not finite in parts as it is (with
  // both in one the 128K hybrid case's join took 5.6 us for 5.0).
  auto plain = [](float sum, float w, float v) { return __builtin_fmaf(w, v, sum); };
  auto odd = [](float sum, float w, float v) { return pg_bad32(v) ? sum + v : __builtin_fmaf(w, v, sum); };
  if (mine) {
    // the largest of the group's parts, 32 at a time
    for (int p = g + lane * S; p < j.n_parts; p += 32 * S) M = fmaxf(M, ms[p * step]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float f = pg_factor(M, a.log2_scale);
    auto sum = [&](auto add) __attribute__((always_inline)) {
      l = x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll 4
      for (int p = g; p < j.n_parts; p += S) {
        const float mp = ms[p * step], lp = ms[p * step + j.rows];
        const float4 v = *reinterpret_cast<const float4*>(slot + p * step + (size_t)at * kD + lane * 4);
        const float w = pg_share(mp, M, f);            // no finite score: zeros, or what V makes of rows without weight
        l += w * lp;
        x[0] = add(x[0], w, v.x);
        x[1] = add(x[1], w, v.y);
        x[2] = add(x[2], w, v.z);
        x[3] = add(x[3], w, v.w);
      }
    };
    sum(plain);
    if (__builtin_expect(pg_unusual(x), 0)) sum(odd);
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
    const float f = pg_factor(M, a.log2_scale);
    auto sum = [&](auto add) __attribute__((always_inline)) {
      l = x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const float w = pg_share(s_m[i][row], M, f);
        const float4 v = *reinterpret_cast<const float4*>(&s_x[i][row][lane * 4]);
        l += w * s_l[i][row];
        x[0] = add(x[0], w, v.x);
        x[1] = add(x[1], w, v.y);
        x[2] = add(x[2], w, v.z);
        x[3] = add(x[3], w, v.w);
      }
    };
    sum(plain);
    if (__builtin_expect(pg_unusual(x), 0)) sum(odd);
  }
  if (!mine) return;
  const bool none = M == -INFINITY;
  const float inv = none ? 0.f : 1.f / l;
  const int tok = r / G, h = j.view % a.c.hkv;
  const size_t q = (size_t)(j.tok0 + tok) * a.hq + h * G + (r - tok * G);
  pg_put4((T*)nullptr, a.out + (q * kD + lane * 4) * sizeof(T), none ? 0.f : x[0] * inv, none ? 0.f : x[1] * inv,
          none ? 0.f : x[2] * inv, none ? 0.f : x[3] * inv);
  if (a.lse && lane == 0) a.lse[q] = pg_lse(M, l, a.log2_scale);
}

// Workgroup b of a join: the tiles' come first, then those of few new rows.
template <typename T, int G>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedAttn a, JoinShape tile, JoinShape few) {
  __shared__ float s_all[kJoinRows * (kD + 2)];
  const int b = blockIdx.x, split = tile.n * tile.blocks;
  const JoinShape& x = b < split ? tile : few;
  const int i = (b < split ? b : b - split) / x.blocks, block = (b < split ? b : b - split) - i * x.blocks;
  const PagedJoin j = a.joins[b < split ? i : tile.n + i];
  if (x.deep) join_rows<T, G, kJoinRows>(a, j, block, s_all);
  else join_rows<T, G, 1>(a, j, block, s_all);
}

template <typename T>
hipError_t join(int G, const PagedAttn& a, const JoinShape& tile, const JoinShape& few, hipStream_t stream) {
  const unsigned n = (unsigned)(tile.n * tile.blocks + few.n * few.blocks);
  if (n == 0) return hipSuccess;
  if (G == 1) paged_join_kernel<T, 1><<<n, kJoinThreads, 0, stream>>>(a, tile, few);
  else if (G == 2) paged_join_kernel<T, 2><<<n, kJoinThreads, 0, stream>>>(a, tile, few);
  else if (G == 4) paged_join_kernel<T, 4><<<n, kJoinThreads, 0, stream>>>(a, tile, few);
  else paged_join_kernel<T, 8><<<n, kJoinThreads, 0, stream>>>(a, tile, few);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_join(int dtype, int G, const PagedAttn& a, const JoinShape& tile, const JoinShape& few, hipStream_t stream) {
  return dtype == CATEKV_BF16 ? join<uint16_t>(G, a, tile, few, stream) : join<float>(G, a, tile, few, stream);
}

}  // namespace catekv
