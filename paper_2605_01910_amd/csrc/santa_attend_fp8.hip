// santa_attend_fp8.hip -- instantiations of the chunk attention kernels
// (santa_attend.h) for fp8 caches.
#include "santa_attend.h"
#include "santa_kernels.h"

namespace santa {
template hipError_t launch_attend_e<uint8_t>(const AttendPlan &, const AttendArgs &, hipStream_t);
}  // namespace santa
