// The attention kernels for heads of 64 elements.
#include "attend.h"

namespace moecache {
template hipError_t launch_attend<64>(const AttendArgs &, bool, bool, hipStream_t);
}  // namespace moecache
