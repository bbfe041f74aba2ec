// cross_bf16.hip -- the cross attention kernels of cross_fast.h in bfloat16.
#include "cross_fast.h"

namespace mafat {

hipError_t launch_cross_bf16(const CrossArgs& a, const CrossPlan& p, hipStream_t stream) {
  if (a.head_dim <= 64) return launch_fast<MAFAT_BF16, 64>(a, p, stream);
  if (a.head_dim <= 96) return launch_fast<MAFAT_BF16, 96>(a, p, stream);
  if (a.head_dim <= 128) return launch_fast<MAFAT_BF16, 128>(a, p, stream);
  return launch_fast<MAFAT_BF16, 256>(a, p, stream);
}

}  // namespace mafat
