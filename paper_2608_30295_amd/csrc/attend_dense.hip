// Attention with weights over bf16 and fp32 views (attend.h).
#include "attend.h"

namespace catekv {

hipError_t launch_attend_dense(int dtype, int G, const AttendArgs& a, hipStream_t stream) {
  return dtype == CATEKV_BF16 ? launch_attend_g<KindBf16, true>(G, a, stream)
                              : launch_attend_g<KindF32, true>(G, a, stream);
}

}  // namespace catekv
