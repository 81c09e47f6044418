// Attention over a cache of 8 bits and behind shared tokens, for heads of 64 elements.
#include "behind.h"

namespace moecache {
uint64_t front_bytes(const AttendArgs &a, int dim) {
  return (uint64_t)a.prefix_tiles * a.prefix_splits * a.kv.kv_heads * a.prefix_rows * (dim + 2) * sizeof(float);
}
template hipError_t launch_attend_ext<64>(const AttendArgs &, bool, int, hipStream_t);
}  // namespace moecache
