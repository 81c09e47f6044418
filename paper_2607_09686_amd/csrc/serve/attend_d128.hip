// The attention kernels for heads of 128 elements.
#include "attend.h"

namespace moecache {
template hipError_t launch_attend<128>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
