// The attention kernels for heads of 256 elements.
#include "attend.h"

namespace moecache {
template hipError_t launch_attend<256>(const AttendArgs &, bool, int, hipStream_t);
template hipError_t launch_plan<256>(const AttendArgs &, int, hipStream_t);
template hipError_t launch_join<256>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
