// Attention over 8-bit views of e4m3 codes, with and without weights (attend.h).
#include "attend.h"

namespace catekv {

hipError_t launch_attend_e4m3(int dtype, int G, const AttendArgs& a, hipStream_t stream) {
  typedef Kind8<CATEKV_E4M3, uint16_t> KB;
  typedef Kind8<CATEKV_E4M3, float> KF;
  if (dtype == CATEKV_BF16)
    return a.acc ? launch_attend_g<KB, true>(G, a, stream) : launch_attend_g<KB, false>(G, a, stream);
  return a.acc ? launch_attend_g<KF, true>(G, a, stream) : launch_attend_g<KF, false>(G, a, stream);
}

}  // namespace catekv
