// C entries of the serving operators (include/moecache.h): argument checks, launch shapes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../../include/moecache.h"
#include "serve.h"

void moecache_set_last_error(const char *msg);

using namespace moecache;

namespace {

int fail(int code, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    moecache_set_last_error(buf);
  } catch (...) {  // no memory for the message: the code still stands
  }
  return code;
}

int hip_fail(const char *what, hipError_t e) {
  return fail(MOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// Makes the stream's device current while a call launches on it (the null stream's is current).
struct DeviceScope {
  int before = -1;
  hipError_t enter(hipStream_t s) {
    if (!s) return hipSuccess;
    hipDevice_t dev;
    int now;
    hipError_t e = hipStreamGetDevice(s, &dev);
    if (e == hipSuccess) e = hipGetDevice(&now);
    if (e != hipSuccess || dev == now) return e;
    e = hipSetDevice(dev);
    if (e == hipSuccess) before = now;
    return e;
  }
  ~DeviceScope() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

bool aligned(const void *p) { return (uintptr_t)p % 16 == 0; }

// A grid holds less than 2^32 threads: at most 2^24 blocks of 256 per call.
constexpr int64_t kMaxRows = 1 << 27, kMaxTokens = 1 << 24, kMaxSeqHeads = 1 << 22;
constexpr int kMaxSampleRows = 65535;  // rows are a grid's second dimension
// Attention units aimed at: what the card holds at once (256 CUs of two blocks; few rows with heads of
// 256: of one), or with few rows twice that where half as many tiles are there already, so that a
// long and a short sequence's units even out.  Keys below which a tile isn't split.
constexpr int kResident = 512;
constexpr int kFewMinKeys = 256, kManyMinKeys = 512;

int check_kv(const moe_kv_batch *b, const char *who, KvView *kv) {
  if (!b) return fail(MOE_EINVAL, "%s: the batch is NULL", who);
  if (b->dtype != MOE_BF16 && b->dtype != MOE_F16) return fail(MOE_EINVAL, "%s: dtype must be MOE_BF16 or MOE_F16", who);
  if (b->head_dim != 64 && b->head_dim != 128 && b->head_dim != 256)
    return fail(MOE_EINVAL, "%s: head_dim must be 64, 128 or 256", who);
  if (b->n_kv_heads < 1 || b->n_heads < b->n_kv_heads || b->n_heads % b->n_kv_heads || b->n_heads > 1024)
    return fail(MOE_EINVAL, "%s: n_heads must be a multiple of n_kv_heads, 1..1024", who);
  const int P = b->page_tokens;
  if (P < 16 || P > 1024 || (P & (P - 1))) return fail(MOE_EINVAL, "%s: page_tokens must be a power of two in [16, 1024]", who);
  if (b->n_pages < 1) return fail(MOE_EINVAL, "%s: n_pages must be >= 1", who);
  if (b->n_seqs < 0 || b->n_seqs > 65536 || b->n_tokens < 0 || b->n_tokens > kMaxTokens)
    return fail(MOE_EINVAL, "%s: n_seqs must be in [0, 65536] and n_tokens in [0, 2^24]", who);
  if ((int64_t)b->n_tokens * b->n_heads > kMaxRows || (int64_t)b->n_seqs * b->n_kv_heads > kMaxSeqHeads)
    return fail(MOE_EINVAL, "%s: n_tokens * n_heads must be <= 2^27 and n_seqs * n_kv_heads <= 2^22", who);
  if (b->max_pages < 1 || (int64_t)b->max_pages * P > (1 << 30))
    return fail(MOE_EINVAL, "%s: max_pages must be >= 1, max_pages * page_tokens <= 2^30", who);
  if (!b->keys || !b->values || !aligned(b->keys) || !aligned(b->values))
    return fail(MOE_EINVAL, "%s: keys and values must be 16-byte aligned device pointers", who);
  if (b->n_seqs && b->n_tokens && (!b->pages || !b->starts || !b->lengths))
    return fail(MOE_EINVAL, "%s: pages, starts and lengths must not be NULL", who);
  int shift = 0;
  while (1 << shift < P) ++shift;
  *kv = KvView{(uint16_t *)b->keys, (uint16_t *)b->values, b->pages, b->starts, b->lengths, b->status,
               b->n_seqs, b->n_tokens, b->n_heads, b->n_kv_heads, b->n_heads / b->n_kv_heads,
               shift, b->n_pages, b->max_pages};
  return MOE_OK;
}

// A row of `heads` heads every `stride` elements of `size` bytes.
bool rows_ok(const void *p, int64_t stride, int heads, int dim, int size) {
  return p && aligned(p) && stride >= (int64_t)heads * dim && stride * size % 16 == 0 && stride <= (int64_t)1 << 32;
}

// Rows (new tokens times the query heads of a KV head) of an attention tile.  New tokens per sequence
// are known on the device only, so the rule goes by their mean.  Tiles of 32 and 64 rows read the
// cache at full rate, once for every tile of a sequence.  In a tile of 128 the waves share the keys
// through LDS and split the rows, and those without rows have nothing to do.  A batch of both kinds takes one
// size for all, which costs no more than a call for each: 63 single tokens over 4000 keys with a chunk of 2048 behind
// 4000 (128) 294 us, in two calls 105 + 194; 255 with a chunk of 512 (32) 408, in two 365 + 71.
int tile_rows(const KvView &kv) {
  const int64_t rows = (int64_t)kv.n_tokens * kv.group;
  return rows <= (int64_t)32 * kv.n_seqs ? 32 : rows <= (int64_t)64 * kv.n_seqs ? 64 : 128;
}

int plan(AttendArgs *a, uint64_t *bytes, int dim) {
  const KvView &kv = a->kv;
  const int rows = tile_rows(kv);
  const bool few = rows < 128;
  const int resident = few && dim > 128 ? kResident / 2 : kResident;
  // a sequence's tiles number ceil(rows / M), all sequences' together at most all rows / M + n_seqs
  const int64_t tiles = (int64_t)kv.n_tokens * kv.group / rows + kv.n_seqs;
  const int target = few && 2 * tiles * kv.kv_heads >= resident ? 2 * resident : resident;
  a->target_log2 = 0;
  while (1 << a->target_log2 < target) ++a->target_log2;
  a->nearest = few && 4 * tiles * kv.kv_heads >= resident;
  a->min_keys = few ? kFewMinKeys : kManyMinKeys;
  // units: a tile's keys / C, to the nearest whole number; with C >= all tiles' keys / (target /
  // kv_heads) that is at most target / kv_heads in all, and one more per tile; nor can a tile
  // have more than its table's keys give.  A split tile's units, x + 1/2 at x >= 3/2, are fewer than 2 x.
  const int64_t share = target / kv.kv_heads + 1;
  const int64_t most = (((int64_t)kv.max_pages << kv.page_shift) + a->min_keys / 2) / a->min_keys + 1;
  a->max_units = (int)std::min(share + tiles, tiles * most);
  a->max_slots = (int)std::min(2 * share, tiles * most);
  a->max_tiles = (int)std::min(share, tiles);
  *bytes = attend_work_bytes(*a, rows, dim);
  return rows;
}

}  // namespace

extern "C" {

int moe_kv_append(const moe_kv_batch *b, const moe_kv_rope *rope, int32_t in_dtype, const void *k, int64_t k_stride,
                  const void *v, int64_t v_stride, const void *q, int64_t q_stride, void *q_out,
                  int64_t q_out_stride) {
  AppendArgs a{};
  const int rc = check_kv(b, "moe_kv_append", &a.kv);
  if (rc) return rc;
  if (in_dtype != MOE_F32 && in_dtype != b->dtype)
    return fail(MOE_EINVAL, "moe_kv_append: in_dtype must be the cache's dtype or MOE_F32");
  if (rope) {
    if (rope->dim < 0 || rope->dim > b->head_dim || rope->dim % 16)
      return fail(MOE_EINVAL, "moe_kv_append: rope dim must be a multiple of 16 up to head_dim");
    if (rope->dim && !rope->freq) return fail(MOE_EINVAL, "moe_kv_append: rope freq is NULL");
  }
  if (b->n_tokens == 0 || b->n_seqs == 0) return MOE_OK;
  const int size = in_dtype == MOE_F32 ? 4 : 2;
  if (!rows_ok(k, k_stride, b->n_kv_heads, b->head_dim, size) || !rows_ok(v, v_stride, b->n_kv_heads, b->head_dim, size))
    return fail(MOE_EINVAL, "moe_kv_append: k and v must be 16-byte aligned rows of n_kv_heads * head_dim elements");
  if (q && (!rows_ok(q, q_stride, b->n_heads, b->head_dim, size) ||
            !rows_ok(q_out, q_out_stride, b->n_heads, b->head_dim, 2)))
    return fail(MOE_EINVAL, "moe_kv_append: q and q_out must be 16-byte aligned rows of n_heads * head_dim elements");
  a.q = q, a.k = k, a.v = v, a.q_out = q_out;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
  a.freq = rope ? rope->freq : nullptr;
  a.dim = b->head_dim;
  a.rope_dim = rope ? rope->dim : 0;
  a.adjacent = rope ? rope->adjacent != 0 : 0;
  const hipStream_t s = (hipStream_t)b->hip_stream;
  DeviceScope scope;
  hipError_t e = scope.enter(s);
  if (e == hipSuccess) e = launch_append(a, b->dtype == MOE_F16, in_dtype == MOE_F32, s);
  return e == hipSuccess ? MOE_OK : hip_fail("moe_kv_append", e);
}

int moe_kv_attend_workspace(const moe_kv_batch *b, uint64_t *bytes) {
  AttendArgs a{};
  if (!bytes) return fail(MOE_EINVAL, "moe_kv_attend_workspace: bytes is NULL");
  const int rc = check_kv(b, "moe_kv_attend_workspace", &a.kv);
  if (rc) return rc;
  plan(&a, bytes, b->head_dim);
  return MOE_OK;
}

int moe_kv_attend(const moe_kv_batch *b, int32_t window, float scale, const void *q, int64_t q_stride, void *out,
                  int64_t out_stride, void *workspace, uint64_t workspace_bytes) {
  AttendArgs a{};
  const int rc = check_kv(b, "moe_kv_attend", &a.kv);
  if (rc) return rc;
  if (window < 0) return fail(MOE_EINVAL, "moe_kv_attend: window must be >= 0");
  a.scale_log2 = scale * 1.44269504088896340736f;
  if (!(scale > 0.f) || !std::isfinite(a.scale_log2))
    return fail(MOE_EINVAL, "moe_kv_attend: scale must be positive and finite, and its log2(e)-fold too");
  if (b->n_tokens == 0 || b->n_seqs == 0) return MOE_OK;
  if (!rows_ok(q, q_stride, b->n_heads, b->head_dim, 2) || !rows_ok(out, out_stride, b->n_heads, b->head_dim, 2))
    return fail(MOE_EINVAL, "moe_kv_attend: q and out must be 16-byte aligned rows of n_heads * head_dim elements");
  uint64_t bytes;
  const int rows = plan(&a, &bytes, b->head_dim);
  if (!workspace || !aligned(workspace) || workspace_bytes < bytes)
    return fail(MOE_EINVAL, "moe_kv_attend: the workspace must be 16-byte aligned and of at least %llu bytes",
                (unsigned long long)bytes);
  a.q = q, a.out = out, a.q_stride = q_stride, a.out_stride = out_stride;
  a.window = window;
  a.work = workspace;
  const hipStream_t s = (hipStream_t)b->hip_stream;
  DeviceScope scope;
  hipError_t e = scope.enter(s);
  const bool half = b->dtype == MOE_F16;
  if (e == hipSuccess)
    e = b->head_dim == 64    ? launch_attend<64>(a, half, rows, s)
        : b->head_dim == 128 ? launch_attend<128>(a, half, rows, s)
                             : launch_attend<256>(a, half, rows, s);
  return e == hipSuccess ? MOE_OK : hip_fail("moe_kv_attend", e);
}

int moe_sample_workspace(const moe_sample_batch *b, uint64_t *bytes) {
  if (!b || !bytes) return fail(MOE_EINVAL, "moe_sample_workspace: the batch or bytes is NULL");
  if (b->n_rows < 0 || b->n_rows > kMaxSampleRows || b->vocab < 1 || b->vocab > 1 << 20)
    return fail(MOE_EINVAL, "moe_sample_workspace: n_rows must be in [0, 65535] and vocab in [1, 2^20]");
  *bytes = sample_work_bytes(b->n_rows, b->vocab);
  return MOE_OK;
}

int moe_sample(const moe_sample_batch *b, int32_t *token, float *prob, void *workspace, uint64_t workspace_bytes) {
  if (!b) return fail(MOE_EINVAL, "moe_sample: the batch is NULL");
  if (b->dtype != MOE_F32 && b->dtype != MOE_BF16 && b->dtype != MOE_F16)
    return fail(MOE_EINVAL, "moe_sample: dtype must be MOE_F32, MOE_BF16 or MOE_F16");
  if (b->vocab < 1 || b->vocab > 1 << 20) return fail(MOE_EINVAL, "moe_sample: vocab must be in [1, 2^20]");
  if (b->n_rows < 0 || b->n_rows > kMaxSampleRows) return fail(MOE_EINVAL, "moe_sample: n_rows must be in [0, 65535]");
  if (b->n_rows == 0) return MOE_OK;
  if (!b->logits || !b->u || !token) return fail(MOE_EINVAL, "moe_sample: logits, u and token must not be NULL");
  if (b->row_stride < b->vocab || b->row_stride > (int64_t)1 << 32)
    return fail(MOE_EINVAL, "moe_sample: row_stride must be at least vocab");
  const uint64_t bytes = sample_work_bytes(b->n_rows, b->vocab);
  if (bytes && (!workspace || !aligned(workspace) || workspace_bytes < bytes))
    return fail(MOE_EINVAL, "moe_sample: the workspace must be 16-byte aligned and of at least %llu bytes",
                (unsigned long long)bytes);
  const uintptr_t size = b->dtype == MOE_F32 ? 4 : 2;
  if ((uintptr_t)b->logits % size) return fail(MOE_EINVAL, "moe_sample: logits are not aligned to their elements");
  const SampleArgs a{b->logits, b->row_stride, b->n_rows, b->vocab, b->temperature, b->top_p, b->min_p,
                     b->top_k,  b->u,          token,     prob,     workspace};
  const hipStream_t s = (hipStream_t)b->hip_stream;
  DeviceScope scope;
  hipError_t e = scope.enter(s);
  if (e == hipSuccess) e = launch_sample(a, b->dtype == MOE_F32 ? 0 : b->dtype == MOE_BF16 ? 1 : 2, s);
  return e == hipSuccess ? MOE_OK : hip_fail("moe_sample", e);
}

}  // extern "C"
