// The attention kernels for heads of 128 elements.
#include "attend.h"

namespace moecache {
template hipError_t launch_attend<128>(const AttendArgs &, bool, int, hipStream_t);
template hipError_t launch_plan<128>(const AttendArgs &, int, hipStream_t);
template hipError_t launch_join<128>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
