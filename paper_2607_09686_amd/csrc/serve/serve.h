// Internal interface of the serving operators: appending rotated keys and values to a paged
// cache, attention over it, sampling.  Launch wrappers return the launch's own status.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace moecache {

// One layer's paged cache and the batch of new tokens, as the kernels see them.
struct KvView {
  uint16_t *keys, *values;   // pools (elements of 16 bits)
  const int32_t *pages;      // [n_seqs][max_pages]
  const int32_t *starts;     // [n_seqs + 1]
  const int32_t *lengths;    // [n_seqs]
  int32_t *status;           // nullable
  int n_seqs, n_tokens, heads, kv_heads, group;
  int page_shift, n_pages, max_pages;
};

// bits of *status
constexpr int kKvBadPage = 1, kKvBadLength = 2;

struct AppendArgs {
  KvView kv;
  const void *q, *k, *v;             // q nullable
  void *q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements from token to token
  const double *freq;                // [rope_dim / 2] radians per position
  int dim, rope_dim, adjacent;
};

struct AttendArgs {
  KvView kv;
  const void *q;
  void *out;
  int64_t q_stride, out_stride;
  int window;          // 0: none
  float scale_log2;    // scale * log2(e)
  int target_log2;     // of the work units aimed at over all KV heads
  int min_keys;        // fewest keys of a unit, a multiple of 64
  int max_units;       // grid units per KV head
  int max_slots;       // partial-result slots per KV head
  int max_tiles;       // split tiles
  bool nearest;        // how a tile's units are rounded, see units_of
  void *work;          // attend_work_bytes
};

// in_f32: q, k, v hold fp32 instead of the cache's type; half: the cache's type is fp16
hipError_t launch_append(const AppendArgs &a, bool half, bool in_f32, hipStream_t s);

// rows: of a tile, 32, 64 or 128
uint64_t attend_work_bytes(const AttendArgs &a, int rows, int dim);
template <int D>
hipError_t launch_attend(const AttendArgs &a, bool half, int rows, hipStream_t s);

struct SampleArgs {
  const void *logits;
  int64_t stride;  // elements from row to row
  int rows, vocab;
  const float *temperature, *top_p, *min_p;  // [rows], nullable
  const int32_t *top_k;                      // [rows], nullable
  const float *u;                            // [rows]
  int32_t *token;                            // [rows]
  float *prob;                               // [rows], nullable
  void *work;                                // sample_work_bytes
};
size_t sample_work_bytes(int rows, int vocab);
// type of the logits: 0 fp32, 1 bf16, 2 fp16
hipError_t launch_sample(const SampleArgs &a, int type, hipStream_t s);

}  // namespace moecache
