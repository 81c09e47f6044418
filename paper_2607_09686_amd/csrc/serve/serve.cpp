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
constexpr int kFewMinKeys = 256, kManyMinKeys = 512, kShortMinKeys = 192;

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
               shift, b->n_pages, b->max_pages, nullptr, nullptr};
  return MOE_OK;
}

// The same with the scales of pools of 8 bits, if given.
int check_kv_ext(const moe_kv_batch *b, const moe_kv_scales *scales, const char *who, KvView *kv) {
  const int rc = check_kv(b, who, kv);
  if (rc || !scales) return rc;
  if (!scales->keys || !scales->values || !aligned(scales->keys) || !aligned(scales->values))
    return fail(MOE_EINVAL, "%s: the scales must be 16-byte aligned device pointers", who);
  kv->key_scales = scales->keys, kv->value_scales = scales->values;
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

// The launch over what all sequences begin with: tiles of all rows together, each cut into units alike.  A unit's
// time goes with its keys, and each unit more leaves a tile's partial results to write and to read; with x tiles (of all
// KV heads) of S keys the two balance at sqrt(S x) units, up to a factor that measured as about 0.45: n = 0.45 sqrt(S / x)
// to a tile, to the nearest power of two (5 n^2 x <= 2 S).  us with half as many, as many, and twice: 64 sequences behind
// 8192 (16 tiles, 8 units each) 61, 41, 46; 8 behind 65536 in 8 bits (4, 64) 40, 29, 39; 24 windows behind 2992 (16, 8) 25,
// 22, 28; 16 behind 4096 (4, 16) 21, 17, 17; 32 behind 32768 (8, 32) 54, 37, 43; 8 chunks of 50 to 200 behind 8192 (256, 2)
// 186, 148, 146.  Not more than the card holds twice, for the workspace's sake.
// S is what the prefix's pages hold, its count is on the device.
constexpr int kPrefixMinKeys = 128;
void plan_prefix(AttendArgs *a) {
  const KvView &kv = a->kv;
  const int64_t rows = (int64_t)kv.n_tokens * kv.group, keys = (int64_t)a->prefix_pages << kv.page_shift;
  a->prefix_rows = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  a->prefix_tiles = (int)((rows + a->prefix_rows - 1) / a->prefix_rows);
  const int64_t tiles = (int64_t)a->prefix_tiles * kv.kv_heads;
  int64_t n = 1;
  const auto fits = [&](int64_t n) {
    return 5 * n * n * tiles <= 2 * keys && keys / n >= kPrefixMinKeys && n * tiles <= 2 * kResident;
  };
  while (fits(2 * n)) n *= 2;
  a->prefix_splits = (int)n;
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
  // Keys of 8 bits, where there are tiles of few rows enough, are as many again: 64 sequences of 50 to 1500, 24.8 us, with
  // 256 keys 28.5.  Few tiles of 128 rows over 8 bits or behind shared tokens are cut finer (kShortMinKeys, 512 keys): 60
  // tokens over 460 with heads of 256 27 and 38 us, 3 chunks of 108 to 210 behind 800 shared and 580 to 819 own 36 and 55,
  // 4 of 10 to 26 behind 1312 and 333 to 409 23 and 29; with more tiles it costs, 5 chunks of 65 to 438 60 and 47.
  const bool ext = kv.key_scales || a->shared;
  const bool wide = few && kv.key_scales && target > resident, fine = !few && ext && 4 * tiles * kv.kv_heads <= resident;
  a->min_keys = fine ? kShortMinKeys : few && !wide ? kFewMinKeys : kManyMinKeys;
  // units: a tile's keys / C, to the nearest whole number; with C >= all tiles' keys / (target /
  // kv_heads) that is at most target / kv_heads in all, and one more per tile; nor can a tile
  // have more than its table's keys give.  A split tile's units, x + 1/2 at x >= 3/2, are fewer than 2 x.
  const int64_t share = target / kv.kv_heads + 1;
  const int64_t most = (((int64_t)kv.max_pages << kv.page_shift) + a->min_keys / 2) / a->min_keys + 1;
  a->max_units = (int)std::min(share + tiles, tiles * most);
  a->max_slots = (int)std::min(2 * share, tiles * most);
  a->max_tiles = (int)std::min(share, tiles);
  if (a->shared) {  // every tile's units leave partial results, and a note
    a->max_slots = a->max_units;
    a->max_tiles = (int)tiles;
    plan_prefix(a);
  }
  *bytes = attend_work_bytes(*a, rows, dim);
  if (a->shared) *bytes += front_bytes(*a, dim);
  return rows;
}

int check_prefix(const moe_kv_prefix *p, const char *who, AttendArgs *a) {
  if (!p) return MOE_OK;
  if (!p->pages || !p->tokens) return fail(MOE_EINVAL, "%s: the prefix's pages and tokens must not be NULL", who);
  if (p->n_pages < 1 || ((int64_t)p->n_pages << a->kv.page_shift) > (1 << 30))
    return fail(MOE_EINVAL, "%s: the prefix's n_pages must be >= 1, n_pages * page_tokens <= 2^30", who);
  a->prefix = p->pages, a->shared = p->tokens, a->prefix_pages = p->n_pages;
  return MOE_OK;
}

// What the two forms of appending have in common, from the checked view on.
int append(AppendArgs &a, const moe_kv_batch *b, const moe_kv_rope *rope, int32_t in_dtype, const void *k,
           int64_t k_stride, const void *v, int64_t v_stride, const void *q, int64_t q_stride, void *q_out,
           int64_t q_out_stride, const char *who) {
  if (in_dtype != MOE_F32 && in_dtype != b->dtype)
    return fail(MOE_EINVAL, "%s: in_dtype must be the cache's dtype or MOE_F32", who);
  if (rope) {
    if (rope->dim < 0 || rope->dim > b->head_dim || rope->dim % 16)
      return fail(MOE_EINVAL, "%s: rope dim must be a multiple of 16 up to head_dim", who);
    if (rope->dim && !rope->freq) return fail(MOE_EINVAL, "%s: rope freq is NULL", who);
  }
  if (b->n_tokens == 0 || b->n_seqs == 0) return MOE_OK;
  const int size = in_dtype == MOE_F32 ? 4 : 2;
  if (!rows_ok(k, k_stride, b->n_kv_heads, b->head_dim, size) || !rows_ok(v, v_stride, b->n_kv_heads, b->head_dim, size))
    return fail(MOE_EINVAL, "%s: k and v must be 16-byte aligned rows of n_kv_heads * head_dim elements", who);
  if (q && (!rows_ok(q, q_stride, b->n_heads, b->head_dim, size) ||
            !rows_ok(q_out, q_out_stride, b->n_heads, b->head_dim, 2)))
    return fail(MOE_EINVAL, "%s: q and q_out must be 16-byte aligned rows of n_heads * head_dim elements", who);
  a.q = q, a.k = k, a.v = v, a.q_out = q_out;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
  a.freq = rope ? rope->freq : nullptr;
  a.dim = b->head_dim;
  a.rope_dim = rope ? rope->dim : 0;
  a.adjacent = rope ? rope->adjacent != 0 : 0;
  const hipStream_t s = (hipStream_t)b->hip_stream;
  const bool half = b->dtype == MOE_F16, in_f32 = in_dtype == MOE_F32;
  DeviceScope scope;
  hipError_t e = scope.enter(s);
  if (e == hipSuccess)
    e = a.q_norm || a.k_norm || a.kv.key_scales ? launch_append_ext(a, half, in_f32, s) : launch_append(a, half, in_f32, s);
  return e == hipSuccess ? MOE_OK : hip_fail(who, e);
}

// And of attention: the plan, the launches.
int attend(AttendArgs &a, const moe_kv_batch *b, int32_t window, float scale, const void *q, int64_t q_stride, void *out,
           int64_t out_stride, void *workspace, uint64_t workspace_bytes, const char *who) {
  if (window < 0) return fail(MOE_EINVAL, "%s: window must be >= 0", who);
  a.scale_log2 = scale * 1.44269504088896340736f;
  if (!(scale > 0.f) || !std::isfinite(a.scale_log2))
    return fail(MOE_EINVAL, "%s: scale must be positive and finite, and its log2(e)-fold too", who);
  if (b->n_tokens == 0 || b->n_seqs == 0) return MOE_OK;
  if (!rows_ok(q, q_stride, b->n_heads, b->head_dim, 2) || !rows_ok(out, out_stride, b->n_heads, b->head_dim, 2))
    return fail(MOE_EINVAL, "%s: q and out must be 16-byte aligned rows of n_heads * head_dim elements", who);
  uint64_t bytes;
  const int rows = plan(&a, &bytes, b->head_dim);
  if (!workspace || !aligned(workspace) || workspace_bytes < bytes)
    return fail(MOE_EINVAL, "%s: the workspace must be 16-byte aligned and of at least %llu bytes", who,
                (unsigned long long)bytes);
  a.q = q, a.out = out, a.q_stride = q_stride, a.out_stride = out_stride;
  a.window = window;
  a.work = workspace;
  const bool half = b->dtype == MOE_F16, ext = a.shared || a.kv.key_scales;
  if (a.shared) a.front = (float *)((uint8_t *)workspace + attend_work_bytes(a, rows, b->head_dim));
  const hipStream_t s = (hipStream_t)b->hip_stream;
  DeviceScope scope;
  hipError_t e = scope.enter(s);
  if (e == hipSuccess) {
    if (b->head_dim == 64)
      e = ext ? launch_attend_ext<64>(a, half, rows, s) : launch_attend<64>(a, half, rows, s);
    else if (b->head_dim == 128)
      e = ext ? launch_attend_ext<128>(a, half, rows, s) : launch_attend<128>(a, half, rows, s);
    else
      e = ext ? launch_attend_ext<256>(a, half, rows, s) : launch_attend<256>(a, half, rows, s);
  }
  return e == hipSuccess ? MOE_OK : hip_fail(who, e);
}

}  // namespace

extern "C" {

int moe_kv_append(const moe_kv_batch *b, const moe_kv_rope *rope, int32_t in_dtype, const void *k, int64_t k_stride,
                  const void *v, int64_t v_stride, const void *q, int64_t q_stride, void *q_out,
                  int64_t q_out_stride) {
  AppendArgs a{};
  const int rc = check_kv(b, "moe_kv_append", &a.kv);
  return rc ? rc : append(a, b, rope, in_dtype, k, k_stride, v, v_stride, q, q_stride, q_out, q_out_stride, "moe_kv_append");
}

int moe_kv_append_ext(const moe_kv_batch *b, const moe_kv_scales *scales, const moe_kv_rope *rope, const moe_kv_norm *norm,
                      int32_t in_dtype, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *q,
                      int64_t q_stride, void *q_out, int64_t q_out_stride) {
  const char *who = "moe_kv_append_ext";
  AppendArgs a{};
  const int rc = check_kv_ext(b, scales, who, &a.kv);
  if (rc) return rc;
  if (norm) {
    if (norm->dtype != MOE_F32 && norm->dtype != b->dtype)
      return fail(MOE_EINVAL, "%s: the norm's dtype must be the cache's or MOE_F32", who);
    if (!(norm->eps >= 0.f) || !std::isfinite(norm->eps))
      return fail(MOE_EINVAL, "%s: the norm's eps must not be negative, and finite", who);
    if (!aligned(norm->q_weight) || !aligned(norm->k_weight))
      return fail(MOE_EINVAL, "%s: the norm's weights must be 16-byte aligned device pointers", who);
    if (norm->q_weight && !q && b->n_tokens && b->n_seqs) return fail(MOE_EINVAL, "%s: a norm of q without q", who);
    a.q_norm = norm->q_weight, a.k_norm = norm->k_weight;
    a.norm_f32 = norm->dtype == MOE_F32, a.eps = norm->eps;
  }
  return append(a, b, rope, in_dtype, k, k_stride, v, v_stride, q, q_stride, q_out, q_out_stride, who);
}

int moe_kv_read(const moe_kv_batch *b, const moe_kv_scales *scales, void *k, int64_t k_stride, void *v, int64_t v_stride) {
  ReadArgs a{};
  const int rc = check_kv_ext(b, scales, "moe_kv_read", &a.kv);
  if (rc) return rc;
  if (b->n_tokens == 0 || b->n_seqs == 0) return MOE_OK;
  if (!rows_ok(k, k_stride, b->n_kv_heads, b->head_dim, 2) || !rows_ok(v, v_stride, b->n_kv_heads, b->head_dim, 2))
    return fail(MOE_EINVAL, "moe_kv_read: k and v must be 16-byte aligned rows of n_kv_heads * head_dim elements");
  a.k = k, a.v = v, a.k_stride = k_stride, a.v_stride = v_stride, a.dim = b->head_dim;
  const hipStream_t s = (hipStream_t)b->hip_stream;
  DeviceScope scope;
  hipError_t e = scope.enter(s);
  if (e == hipSuccess) e = launch_read(a, b->dtype == MOE_F16, s);
  return e == hipSuccess ? MOE_OK : hip_fail("moe_kv_read", e);
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
  return rc ? rc : attend(a, b, window, scale, q, q_stride, out, out_stride, workspace, workspace_bytes, "moe_kv_attend");
}

int moe_kv_attend_ext_workspace(const moe_kv_batch *b, const moe_kv_scales *scales, const moe_kv_prefix *prefix,
                                uint64_t *bytes) {
  const char *who = "moe_kv_attend_ext_workspace";
  AttendArgs a{};
  if (!bytes) return fail(MOE_EINVAL, "%s: bytes is NULL", who);
  int rc = check_kv_ext(b, scales, who, &a.kv);
  if (!rc) rc = check_prefix(prefix, who, &a);
  if (rc) return rc;
  plan(&a, bytes, b->head_dim);
  return MOE_OK;
}

int moe_kv_attend_ext(const moe_kv_batch *b, const moe_kv_scales *scales, const moe_kv_prefix *prefix, int32_t window,
                      float scale, const void *q, int64_t q_stride, void *out, int64_t out_stride, void *workspace,
                      uint64_t workspace_bytes) {
  const char *who = "moe_kv_attend_ext";
  AttendArgs a{};
  int rc = check_kv_ext(b, scales, who, &a.kv);
  if (!rc) rc = check_prefix(prefix, who, &a);
  if (rc) return rc;
  if (prefix && window) return fail(MOE_EINVAL, "%s: a window and a prefix do not go together", who);
  return attend(a, b, window, scale, q, q_stride, out, out_stride, workspace, workspace_bytes, who);
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
