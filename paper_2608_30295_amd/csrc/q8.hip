// Caches in 8 bits: rows into codes with a scale per block of rows, back, and
// the append of a step's token.
//
// All three move bytes and little else (quantize: 2 row bytes read and one
// written per element pair), so a wave takes one block of K or of V whole: the
// rows go through its registers once, the maximum is taken of the bit patterns
// on the way, and both sides are read and written in whole lines (lanes with 32
// consecutive bytes of fp32, half a line per access: 4099 fp32 rows of 8 heads back
// from int8 15.2 -> 8.4 us).  131072 bf16 rows of 8 heads: 805 MB in 149 us into
// e4m3, in 147 us back (5.4 and 5.5 TB/s; a copy runs at 5.15), 136 and 117 right after
// one another (the codes then come partly from the Infinity Cache, it seems: the L2
// asks for all of their 269 MB).
#include "cache.h"
#include "common.h"

namespace catekv {

constexpr float kTinyMax = 7.888609052210118e-31f;   // 2^-100
constexpr int kQ8Waves = kQ8Threads / 64;

// The rows on their way into codes are read once (once16).  They and the rows written
// on the way back pass the caches by, which leaves these to the codes (8
// heads of 131072 bf16 rows into e4m3 and back 306 -> 258 us, of 32768 87 -> 71; one
// way alone 45 -> 39 and 47 -> 33 at 32768, 150 -> 149 and 155 -> 147 at 131072).

// 16 bytes of a row: kN elements.
template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
  static constexpr int kN = 8;
  uint4 w;
  __device__ __forceinline__ float get(int i) const {
    const uint32_t x = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return i & 1 ? bf16_hi(x) : bf16_lo(x);
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[0], f[1]}), b2));
    w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[2], f[3]}), b2));
    w.z = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[4], f[5]}), b2));
    w.w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[6], f[7]}), b2));
  }
};
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  uint4 w;
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w); }
  __device__ __forceinline__ void set(const float (&f)[4]) {
    w = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_ds_bpermute(((int)__lane_id() ^ o) << 2, (int)x);
    x = x > y ? x : y;
  }
  return x;
}

// Scale of a block whose largest |x| has these bits, and its reciprocal (0 for a
// block that is all 0 or not finite: its codes are 0).
template <int FMT>
__device__ __forceinline__ void block_scale(uint32_t big, float& scale, float& inv) {
  scale = inv = 0.f;
  if (big >= 0x7f800000u) {
    scale = __uint_as_float(0x7fc00000u);
  } else if (__uint_as_float(big) >= kTinyMax) {
    if constexpr (FMT == CATEKV_I8) {
      scale = __uint_as_float(big) * (1.0f / 127.0f);
      inv = 1.0f / scale;
    } else {
      // 448 = 1.75 * 2^8: m / 2^8, one power more if its fraction is above 1.75
      const uint32_t e = (big >> 23) - 8 + ((big & 0x7fffffu) > 0x600000u ? 1 : 0);
      scale = __uint_as_float(e << 23);
      inv = __uint_as_float((254u - e) << 23);
    }
  }
}

// Codes of a piece, one word per four elements.  int8: x inv is within 2^-15 of the
// quotient x / scale, which decides the rounding except next to a border between
// two codes; where the wave holds such an element (2 in 10^4 of normal values: 10% of
// its 512 elements of bf16, 5% of its 256 of fp32) all are divided in fp64, whose
// quotient lies on a border only if the exact one does.  e4m3: x inv is exact, the
// conversion rounds to nearest even.
template <int FMT, typename T>
__device__ __forceinline__ void piece_codes(const Piece<T>& x, float scale, float inv, uint32_t (&w)[Piece<T>::kN / 4]) {
  constexpr int N = Piece<T>::kN;
  if constexpr (FMT == CATEKV_I8) {
    float r[N];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = x.get(i) * inv;
      r[i] = __builtin_rintf(y);
      off = fmaxf(off, fabsf(y - r[i]));
    }
    if (__builtin_amdgcn_ballot_w64(off > 0.4999f)) {
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = (float)__builtin_rint((double)x.get(i) / (double)scale);
    }
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
      w[h] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[h] |= ((uint32_t)(int)r[4 * h + i] & 0xffu) << (8 * i);
    }
  } else {
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(x.get(4 * h) * inv, x.get(4 * h + 1) * inv, 0, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(x.get(4 * h + 2) * inv, x.get(4 * h + 3) * inv, c, true);
      w[h] = (uint32_t)c;
    }
  }
}

template <int W>
__device__ __forceinline__ void store_words(uint8_t* p, const uint32_t (&w)[W]) {
  if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// ROWS rows of a block in one wave, from row `first` on: a lane takes 16 bytes of
// every 64-lane load, which covers two fp32 rows or four bf16 rows whole.
// `row(r)`: address of the block's row r.
template <typename T, int ROWS>
struct BlockRows {
  static constexpr int kPer = kD / Piece<T>::kN;   // lanes of a row
  static constexpr int kStep = 64 / kPer;          // rows of a load
  static constexpr int N = ROWS / kStep;
  Piece<T> x[N];
  template <typename Row>
  __device__ __forceinline__ void load(Row row, int first) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i].w = once16(row(first + lane / kPer + kStep * i) + (lane % kPer) * 16);
  }
  // largest |x| of the wave's rows, as bits
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < Piece<T>::kN; ++j) {
        const uint32_t b = __float_as_uint(x[i].get(j)) & 0x7fffffffu;
        big = big > b ? big : b;
      }
    return wave_max(big);
  }
  template <int FMT>
  __device__ __forceinline__ void store(uint8_t* codes, int first, float scale, float inv) const {
    const int lane = threadIdx.x & 63;
    const bool zero = inv == 0.f;                  // 0 * inf is not 0
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t w[Piece<T>::kN / 4] = {};
      if (!zero) piece_codes<FMT, T>(x[i], scale, inv, w);
      store_words(codes + (first + lane / kPer + kStep * i) * kD + (lane % kPer) * Piece<T>::kN, w);
    }
  }
};

// grid: (groups of kQ8Waves blocks x views, views fastest; 1; K and V).  The wave
// behind a view's last whole block copies the remaining rows into the tail.
template <int FMT, typename T, int BLOCK>
__global__ __launch_bounds__(kQ8Threads) void q8_quantize_kernel(Q8Args a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views;
  const bool is_v = blockIdx.z;
  const int64_t len = a.lens[bh];
  if (len < 0 || len > a.max_rows) return;
  const int64_t whole = len / BLOCK, blk = (int64_t)group * kQ8Waves + wave;
  if (blk > whole) return;
  const catekv_q8_view view = a.views[bh];
  const catekv_kv_ptrs kv = a.kv[bh];
  const char* src = reinterpret_cast<const char*>(is_v ? kv.v : kv.k) + (size_t)blk * BLOCK * kD * sizeof(T);
  if (blk < whole) {
    BlockRows<T, BLOCK> rows;
    rows.load([&](int r) { return src + (size_t)r * kD * sizeof(T); }, 0);
    float scale, inv;
    block_scale<FMT>(rows.largest(), scale, inv);
    rows.template store<FMT>(reinterpret_cast<uint8_t*>(is_v ? view.v : view.k) + (size_t)blk * BLOCK * kD, 0, scale, inv);
    if (lane == 0) (is_v ? view.v_scale : view.k_scale)[blk] = scale;
    return;
  }
  char* dst = reinterpret_cast<char*>(is_v ? view.v_tail : view.k_tail);
  const int bytes = (int)(len - whole * BLOCK) * kD * (int)sizeof(T);
  for (int i = lane * 16; i < bytes; i += 64 * 16) *reinterpret_cast<uint4*>(dst + i) = ldg16(src + i);
}

template <int FMT, typename T, int BLOCK>
__global__ __launch_bounds__(kQ8Threads) void q8_dequantize_kernel(Q8Args a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int group = blockIdx.x / a.n_views, bh = blockIdx.x - group * a.n_views;
  const bool is_v = blockIdx.z;
  const int64_t len = a.lens[bh];
  if (len < 0 || len > a.max_rows) return;
  const int64_t whole = len / BLOCK, blk = (int64_t)group * kQ8Waves + wave;
  if (blk > whole) return;
  const catekv_q8_view view = a.views[bh];
  const catekv_kv_ptrs kv = a.kv[bh];
  char* dst = reinterpret_cast<char*>(const_cast<void*>(is_v ? kv.v : kv.k)) + (size_t)blk * BLOCK * kD * sizeof(T);
  if (blk < whole) {
    const char* src = reinterpret_cast<const char*>(is_v ? view.v : view.k) + (size_t)blk * BLOCK * kD;
    const float scale = (is_v ? view.v_scale : view.k_scale)[blk];
    // a lane takes the codes of 16 bytes of every 64-lane store
    constexpr int E = Piece<T>::kN, N = BLOCK * kD / E / 64;
    uint32_t c[N][E / 4];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t* p = reinterpret_cast<const uint32_t*>(src + (i * 64 + lane) * E);
#pragma unroll
      for (int h = 0; h < E / 4; ++h) c[i][h] = p[h];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float f[E];
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const uint32_t x = c[i][j >> 2];
        if constexpr (FMT == CATEKV_I8) {
          f[j] = (float)(int8_t)(x >> (8 * (j & 3)));
        } else {
          f[j] = (j & 3) == 0   ? __builtin_amdgcn_cvt_f32_fp8(x, 0)
                 : (j & 3) == 1 ? __builtin_amdgcn_cvt_f32_fp8(x, 1)
                 : (j & 3) == 2 ? __builtin_amdgcn_cvt_f32_fp8(x, 2)
                                : __builtin_amdgcn_cvt_f32_fp8(x, 3);
        }
        f[j] *= scale;
      }
      Piece<T> o;
      o.set(f);
      __builtin_nontemporal_store(u32x4_t{o.w.x, o.w.y, o.w.z, o.w.w}, reinterpret_cast<u32x4_t*>(dst + (size_t)(i * 64 + lane) * 16));
    }
    return;
  }
  const char* src = reinterpret_cast<const char*>(is_v ? view.v_tail : view.k_tail);
  const int bytes = (int)(len - whole * BLOCK) * kD * (int)sizeof(T);
  for (int i = lane * 16; i < bytes; i += 64 * 16) *reinterpret_cast<uint4*>(dst + i) = ldg16(src + i);
}

// One workgroup per view: four waves for K, four for V, a quarter of a block each
// when the new row fills it.  That row is taken from the call's arguments, not from
// the tail it was just stored in.
template <int FMT, typename T, int BLOCK>
__global__ __launch_bounds__(kAppendThreads) void q8_append_kernel(Q8Args a) {
  const int bh = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = wave & 3;
  const bool is_v = wave >= 4;
  __shared__ uint32_t s_big[8];
  const int64_t len = a.lens_rw[bh], cap = a.capacity[bh];
  const catekv_q8_view view = a.views[bh];
  if (len < 0 || len >= cap) {
    if (threadIdx.x == 0 && a.overflow) *a.overflow = 1;
    return;
  }
  const int64_t blk = len / BLOCK;
  const int at = (int)(len - blk * BLOCK);
  constexpr int kRow = kD * (int)sizeof(T), kRows = BLOCK / 4;
  const char* fresh = reinterpret_cast<const char*>(is_v ? a.v_new : a.k_new) + (size_t)bh * kRow;
  char* tail = reinterpret_cast<char*>(is_v ? view.v_tail : view.k_tail);
  const bool full = at == BLOCK - 1;
  BlockRows<T, kRows> rows;
  if (full) rows.load([&](int r) { return r == BLOCK - 1 ? fresh : tail + r * kRow; }, part * kRows);
  if (part == 0 && lane < kRow / 16) *reinterpret_cast<uint4*>(tail + at * kRow + lane * 16) = ldg16(fresh + lane * 16);
  if (full) {
    const uint32_t big = rows.largest();
    if (lane == 0) s_big[wave] = big;
  }
  __syncthreads();                                 // all waves have read the length, too
  if (full) {
    const uint32_t* b = s_big + (is_v ? 4 : 0);
    float scale, inv;
    block_scale<FMT>(max(max(b[0], b[1]), max(b[2], b[3])), scale, inv);
    rows.template store<FMT>(reinterpret_cast<uint8_t*>(is_v ? view.v : view.k) + (size_t)blk * BLOCK * kD, part * kRows, scale, inv);
    if (part == 0 && lane == 0) (is_v ? view.v_scale : view.k_scale)[blk] = scale;
  }
  if (threadIdx.x == 0) a.lens_rw[bh] = len + 1;
}

int64_t q8_groups(int64_t max_rows, int block) {
  return (max_rows / block + kQ8Waves) / kQ8Waves;   // one wave more than whole blocks, for the tail
}

enum Q8Op { kQuantize, kDequantize, kAppend };

template <int FMT, typename T, int BLOCK>
static hipError_t launch_q8_t(Q8Op op, const Q8Args& a, hipStream_t stream) {
  const dim3 grid((unsigned)(q8_groups(a.max_rows, BLOCK) * a.n_views), 1, 2), block(kQ8Threads);
  if (op == kQuantize)
    hipLaunchKernelGGL((q8_quantize_kernel<FMT, T, BLOCK>), grid, block, 0, stream, a);
  else if (op == kDequantize)
    hipLaunchKernelGGL((q8_dequantize_kernel<FMT, T, BLOCK>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_append_kernel<FMT, T, BLOCK>), dim3(a.n_views), dim3(kAppendThreads), 0, stream, a);
  return hipGetLastError();
}

template <int FMT, typename T>
static hipError_t launch_q8_b(Q8Op op, const Q8Args& a, hipStream_t stream) {
  return a.block == 32 ? launch_q8_t<FMT, T, 32>(op, a, stream) : launch_q8_t<FMT, T, 64>(op, a, stream);
}

static hipError_t launch_q8(Q8Op op, int fmt, int dtype, const Q8Args& a, hipStream_t stream) {
  if (fmt == CATEKV_I8)
    return dtype == CATEKV_BF16 ? launch_q8_b<CATEKV_I8, uint16_t>(op, a, stream)
                                : launch_q8_b<CATEKV_I8, float>(op, a, stream);
  return dtype == CATEKV_BF16 ? launch_q8_b<CATEKV_E4M3, uint16_t>(op, a, stream)
                              : launch_q8_b<CATEKV_E4M3, float>(op, a, stream);
}

hipError_t launch_q8_quantize(int fmt, int dtype, const Q8Args& a, hipStream_t s) { return launch_q8(kQuantize, fmt, dtype, a, s); }
hipError_t launch_q8_dequantize(int fmt, int dtype, const Q8Args& a, hipStream_t s) { return launch_q8(kDequantize, fmt, dtype, a, s); }
hipError_t launch_q8_append(int fmt, int dtype, const Q8Args& a, hipStream_t s) { return launch_q8(kAppend, fmt, dtype, a, s); }

}  // namespace catekv
