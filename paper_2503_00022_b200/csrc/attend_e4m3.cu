// attend_mma.cuh for caches of this type (a file for each, so that they compile side by side).
#include "attend_mma.cuh"

namespace kvc {

int launch_attend_e4m3(AttendArgs a, cudaStream_t stream) { return att::launch_queries<KVCRUSH_E4M3>(a, stream); }

}  // namespace kvc
