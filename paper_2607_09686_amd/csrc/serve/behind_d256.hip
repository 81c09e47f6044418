// Attention over a cache of 8 bits and behind shared tokens, for heads of 256 elements.
#include "behind.h"

namespace moecache {
template hipError_t launch_attend_ext<256>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
