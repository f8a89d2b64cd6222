// The few-token kernel by itself: batches without chunks, and fp32 (gfx950).
#include "paged_stream.h"

namespace catekv {
namespace {

template <typename T, int G>
__global__ __launch_bounds__(kStreamThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_stream_kernel(PagedAttn a) {
  constexpr int BATCH = 8;
  __shared__ Seg s_seg[BATCH];
  __shared__ uint4 s_q[BATCH][R][kD * sizeof(T) / 16];
  __shared__ float s_o[kStreamWaves][R][kPad];
  __shared__ float s_m[kStreamWaves][R], s_l[kStreamWaves][R];
  stream_share<T, G, BATCH>(a, a.segs, a.seg_workers[blockIdx.x], a.seg_workers[blockIdx.x + 1],
                            {&s_seg, &s_q, &s_o, &s_m, &s_l});
}

template <typename T, int G>
hipError_t stream_tg(const PagedAttn& a, hipStream_t stream) {
  paged_stream_kernel<T, G><<<a.n_few, kStreamThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <typename T>
hipError_t stream_t(int G, const PagedAttn& a, hipStream_t s) {
  return G == 1 ? stream_tg<T, 1>(a, s) : G == 2 ? stream_tg<T, 2>(a, s) : G == 4 ? stream_tg<T, 4>(a, s) : stream_tg<T, 8>(a, s);
}

}  // namespace

hipError_t launch_paged_stream(int dtype, int G, const PagedAttn& a, hipStream_t stream) {
  return dtype == CATEKV_BF16 ? stream_t<uint16_t>(G, a, stream) : stream_t<float>(G, a, stream);
}

}  // namespace catekv
