// santa_attend_f32.hip -- instantiations of the chunk attention kernels
// (santa_attend.h) for f32 caches.
#include "santa_attend.h"
#include "santa_kernels.h"

namespace santa {
template hipError_t launch_attend_e<float>(const AttendPlan &, const AttendArgs &, hipStream_t);
}  // namespace santa
