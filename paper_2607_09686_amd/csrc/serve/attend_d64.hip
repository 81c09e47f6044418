// The attention kernels for heads of 64 elements.
#include "attend.h"

namespace moecache {
uint64_t attend_work_bytes(const AttendArgs &a, int rows, int dim) { return attend_work_size(a, rows, dim); }
template hipError_t launch_attend<64>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
