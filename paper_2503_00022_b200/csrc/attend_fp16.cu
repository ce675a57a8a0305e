// attend_mma.cuh for caches of this type (a file for each, so that they compile side by side).
#include "attend_mma.cuh"

namespace kvc {

int launch_attend_fp16(AttendArgs a, cudaStream_t stream) { return att::launch_width<KVCRUSH_FP16, KVCRUSH_FP16>(a, stream); }

}  // namespace kvc
