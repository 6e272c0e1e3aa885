// santa_attend_bf16.hip -- instantiations of the chunk attention kernels
// (santa_attend.h) for bf16 caches.
#include "santa_attend.h"
#include "santa_kernels.h"

namespace santa {
template hipError_t launch_attend_e<uint16_t>(const AttendPlan &, const AttendArgs &, hipStream_t);
}  // namespace santa
