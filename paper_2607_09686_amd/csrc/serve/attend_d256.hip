// The attention kernels for heads of 256 elements.
#include "attend.h"

namespace moecache {
template hipError_t launch_attend<256>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
