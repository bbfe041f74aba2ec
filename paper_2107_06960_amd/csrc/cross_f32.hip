// cross_f32.hip -- the cross attention kernels of cross_fast.h in float32 (heads up to 128).
#include "cross_fast.h"

namespace mafat {

hipError_t launch_cross_f32(const CrossArgs& a, const CrossPlan& p, hipStream_t stream) {
  if (a.head_dim <= 64) return launch_fast<MAFAT_F32, 64>(a, p, stream);
  if (a.head_dim <= 96) return launch_fast<MAFAT_F32, 96>(a, p, stream);
  return launch_fast<MAFAT_F32, 128>(a, p, stream);
}

}  // namespace mafat
