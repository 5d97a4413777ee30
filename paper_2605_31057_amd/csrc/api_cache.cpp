// api_cache.cpp -- the C ABI of the rotary positions, the 8-bit K/V cache and the
// attention over it (lvsa.h): argument checks and dispatch.
#include <atomic>
#include <climits>
#include <cmath>

#include "values.h"

namespace lvsa {
namespace {

// Whether two of a tensor's rows share an element: rows (h, t) and (h', t') do where
// |(h - h') stride_head - (t - t') stride_token| < 128.
bool rows_overlap(const lvsa_tensor& t, int32_t heads, int32_t n) {
  const __int128 sh = t.stride_head, st = t.stride_token;
  if ((n > 1 && st < 128) || (heads > 1 && sh < 128)) return true;
  if (heads == 1 || n == 1) return false;
  // One axis clears the other, as in every ordinary layout.
  if (sh >= (n - 1) * st + 128 || st >= (heads - 1) * sh + 128) return false;
  for (int32_t h = 1; h < heads; ++h) {
    const __int128 at = h * sh, before = at / st;   // the tokens on both sides of it
    if (before > n - 1) break;
    if (at - before * st < 128 || (before + 1 < n && (before + 1) * st - at < 128)) return true;
  }
  return false;
}

}  // namespace

lvsa_status check_output(const lvsa_tensor* t, int32_t heads, int32_t n) {
  const lvsa_status st = check_tensor(t, heads, n);
  if (st != LVSA_OK) return st;
  return rows_overlap(*t, heads, n) ? LVSA_EINVAL : LVSA_OK;
}

namespace {

constexpr int32_t kMaxCacheHeads = 65535;          // a launch's second dimension
constexpr int64_t kMaxQueryRows = (int64_t)1 << 27; // heads * tokens of one attention call

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

lvsa_status check_rope_grid(const lvsa_rope* r) {
  if (!r) return LVSA_EINVAL;
  if (r->frames < 1 || r->height < 1 || r->width < 1) return LVSA_EINVAL;
  const int64_t plane = (int64_t)r->height * r->width;
  if (plane > INT32_MAX || plane * r->frames > INT32_MAX) return LVSA_EINVAL;
  for (int32_t p : r->pairs)
    if (p < 0 || p > 64) return LVSA_EINVAL;
  const int32_t sum = r->pairs[0] + r->pairs[1] + r->pairs[2];
  if (sum < 1 || sum > 64) return LVSA_EINVAL;
  if (r->layout != LVSA_ROPE_PAIRS && r->layout != LVSA_ROPE_HALVES) return LVSA_EINVAL;
  return LVSA_OK;
}

int64_t table_entries(const lvsa_rope& r) {
  return (int64_t)r.frames * r.pairs[0] + (int64_t)r.height * r.pairs[1] +
         (int64_t)r.width * r.pairs[2];
}

// The kernels' form of *r; entries are counted in 32 bits there.
lvsa_status rope_args(const lvsa_rope* r, RopeArgs* out) {
  const lvsa_status st = check_rope_grid(r);
  if (st != LVSA_OK) return st;
  if (!r->table) return LVSA_EINVAL;
  if (!aligned(r->table, 8) || table_entries(*r) > INT32_MAX) return LVSA_EUNSUPPORTED;
  out->table = r->table;
  out->grid = r->frames * r->height * r->width;
  out->plane = r->height * r->width;
  out->width = r->width;
  out->p0 = r->pairs[0];
  out->p01 = r->pairs[0] + r->pairs[1];
  out->p012 = out->p01 + r->pairs[2];
  out->at_row = r->frames * r->pairs[0];
  out->at_col = out->at_row + r->height * r->pairs[1];
  out->halves = r->layout == LVSA_ROPE_HALVES;
  return LVSA_OK;
}

bool known_type(int32_t dtype) {
  return dtype == LVSA_BF16 || dtype == LVSA_F16 || dtype == LVSA_F32;
}

// A tensor that is read: its own heads and tokens, at least one of each.
lvsa_status check_input(const lvsa_tensor* t) {
  if (!t || t->heads < 1 || t->n_tokens < 1) return LVSA_EINVAL;
  return check_tensor(t, t->heads, t->n_tokens);
}

lvsa_status check_cache(const lvsa_kv_cache* c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return LVSA_EINVAL;
  if (c->heads < 1 || c->capacity < 1 || c->n_tokens < 0 || c->n_tokens > c->capacity)
    return LVSA_EINVAL;
  if (c->block != 64 && c->block != 128) return LVSA_EUNSUPPORTED;
  if (c->capacity % 128 != 0 || c->capacity > LVSA_MAX_CACHE_TOKENS) return LVSA_EUNSUPPORTED;
  if (c->heads > kMaxCacheHeads) return LVSA_EUNSUPPORTED;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4))
    return LVSA_EUNSUPPORTED;
  return LVSA_OK;
}

lvsa_status run_rope(const lvsa_tensor* x, int32_t dtype, int32_t start, const lvsa_rope* rope,
                     lvsa_tensor* y, float sign, void* stream) {
  if (!y || !known_type(dtype) || start < 0) return LVSA_EINVAL;
  lvsa_status st;
  if ((st = check_input(x)) != LVSA_OK) return st;
  if ((st = check_output(y, x->heads, x->n_tokens)) != LVSA_OK) return st;
  if ((int64_t)start + x->n_tokens > INT32_MAX) return LVSA_EINVAL;
  if (x->heads > kMaxCacheHeads || x->n_tokens > (1 << 28)) return LVSA_EUNSUPPORTED;
  if (x->data == y->data &&
      ((x->n_tokens > 1 && x->stride_token != y->stride_token) ||
       (x->heads > 1 && x->stride_head != y->stride_head)))
    return LVSA_EINVAL;
  RopeArgs r;
  if ((st = rope_args(rope, &r)) != LVSA_OK) return st;
  return launch_rope(r, *x, *y, dtype, start, sign, (hipStream_t)stream) == hipSuccess
             ? LVSA_OK
             : LVSA_EDEVICE;
}

// Checks the arguments of an attention call but for out and workspace.
lvsa_status cache_attention_args(const lvsa_tensor* q, int32_t q_start,
                                 const lvsa_kv_cache* cache, const lvsa_block_mask* mask,
                                 CacheAttnArgs* a) {
  lvsa_status st;
  if ((st = check_input(q)) != LVSA_OK) return st;
  if ((st = check_cache(cache)) != LVSA_OK) return st;
  if (q_start < 0 || q->heads % cache->heads != 0) return LVSA_EINVAL;
  if ((int64_t)q->heads * q->n_tokens > kMaxQueryRows) return LVSA_EUNSUPPORTED;
  a->row_ptr = nullptr;
  a->col_idx = nullptr;
  a->mask_block = 0;
  a->mask_blocks = 0;
  if (mask) {
    if (!mask->row_ptr || !mask->col_idx) return LVSA_EINVAL;
    if (mask->block != 64 && mask->block != 128) return LVSA_EUNSUPPORTED;
    if (mask->n_tokens != cache->n_tokens || mask->n_tokens < 1) return LVSA_EINVAL;
    const int32_t nb = (mask->n_tokens + mask->block - 1) / mask->block;
    if (mask->n_q_blocks != nb || mask->n_kv_blocks != nb) return LVSA_EINVAL;
    if (nb > kMaxSparseBlocks) return LVSA_EUNSUPPORTED;
    if ((int64_t)q_start + q->n_tokens > cache->n_tokens) return LVSA_EINVAL;
    a->row_ptr = mask->row_ptr;
    a->col_idx = mask->col_idx;
    a->mask_block = mask->block;
    a->mask_blocks = nb;
  }
  a->q = q->data;
  a->q_sh = q->stride_head, a->q_st = q->stride_token;
  a->o = nullptr;
  a->o_sh = a->o_st = 0;
  a->heads = cache->heads;
  a->group = q->heads / cache->heads;
  a->n = q->n_tokens;
  a->q_start = q_start;
  a->n_tokens = cache->n_tokens;
  a->capacity = cache->capacity;
  a->scale_shift = cache->block == 64 ? 6 : 7;
  a->k = (const uint8_t*)cache->k;
  a->v = (const uint8_t*)cache->v;
  a->k_scale = cache->k_scale;
  a->v_scale = cache->v_scale;
  a->workspace = nullptr;
  return LVSA_OK;
}

// Compute units of the current device (asked for once per device).
lvsa_status compute_units(int32_t* cus) {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return LVSA_EDEVICE;
  if (dev < kDevices) n = known[dev].load(std::memory_order_relaxed);
  if (n < 1) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
        n < 1)
      return LVSA_EDEVICE;
    if (dev < kDevices) known[dev].store(n, std::memory_order_relaxed);
  }
  *cus = n;
  return LVSA_OK;
}

}  // namespace
}  // namespace lvsa

using namespace lvsa;

extern "C" {

lvsa_status lvsa_rope_table_size(const lvsa_rope* r, int64_t* entries) {
  if (!entries) return LVSA_EINVAL;
  const lvsa_status st = check_rope_grid(r);
  if (st != LVSA_OK) return st;
  *entries = table_entries(*r);
  return LVSA_OK;
}

lvsa_status lvsa_rope_table(const lvsa_rope* r, double theta, float* table, int64_t capacity) {
  if (!table || !(theta > 0.0) || !std::isfinite(theta)) return LVSA_EINVAL;
  const lvsa_status st = check_rope_grid(r);
  if (st != LVSA_OK) return st;
  if (capacity < table_entries(*r)) return LVSA_EINVAL;
  const int32_t size[3] = {r->frames, r->height, r->width};
  for (int axis = 0; axis < 3; ++axis)
    for (int32_t pos = 0; pos < size[axis]; ++pos)
      for (int32_t m = 0; m < r->pairs[axis]; ++m) {
        const double angle = pos * std::pow(theta, -(double)m / r->pairs[axis]);
        *table++ = (float)std::cos(angle);
        *table++ = (float)std::sin(angle);
      }
  return LVSA_OK;
}

lvsa_status lvsa_rope_forward(const lvsa_tensor* x, int32_t dtype, int32_t start,
                              const lvsa_rope* rope, lvsa_tensor* out, void* stream) {
  return run_rope(x, dtype, start, rope, out, 1.f, stream);
}

lvsa_status lvsa_rope_backward(const lvsa_tensor* grad_out, int32_t dtype, int32_t start,
                               const lvsa_rope* rope, lvsa_tensor* grad_in, void* stream) {
  return run_rope(grad_out, dtype, start, rope, grad_in, -1.f, stream);
}

lvsa_status lvsa_kv_write(lvsa_kv_cache* cache, const lvsa_tensor* k, const lvsa_tensor* v,
                          int32_t dtype, int32_t start, const lvsa_rope* rope, void* stream) {
  lvsa_status st;
  if ((st = check_cache(cache)) != LVSA_OK) return st;
  if (!known_type(dtype)) return LVSA_EINVAL;
  if ((st = check_input(k)) != LVSA_OK) return st;
  if (k->heads != cache->heads) return LVSA_EINVAL;
  if ((st = check_tensor(v, k->heads, k->n_tokens)) != LVSA_OK) return st;
  if (start < 0 || start > cache->n_tokens || (int64_t)start + k->n_tokens > cache->capacity)
    return LVSA_EINVAL;
  RopeArgs r = {};
  if (rope && (st = rope_args(rope, &r)) != LVSA_OK) return st;
  if (launch_kv_write(*cache, cache->n_tokens, *k, *v, dtype, start, r, (hipStream_t)stream) !=
      hipSuccess)
    return LVSA_EDEVICE;
  if (start + k->n_tokens > cache->n_tokens) cache->n_tokens = start + k->n_tokens;
  return LVSA_OK;
}

lvsa_status lvsa_kv_read(const lvsa_kv_cache* cache, int32_t start, lvsa_tensor* k,
                         lvsa_tensor* v, int32_t dtype, void* stream) {
  lvsa_status st;
  if ((st = check_cache(cache)) != LVSA_OK) return st;
  if (!known_type(dtype) || (!k && !v) || start < 0) return LVSA_EINVAL;
  const int32_t n = k ? k->n_tokens : v->n_tokens;
  if (n < 1 || (int64_t)start + n > cache->n_tokens) return LVSA_EINVAL;
  if (k && (st = check_output(k, cache->heads, n)) != LVSA_OK) return st;
  if (v && (st = check_output(v, cache->heads, n)) != LVSA_OK) return st;
  if (k && v && k->data == v->data) return LVSA_EINVAL;
  return launch_kv_read(*cache, start, k, v, n, dtype, (hipStream_t)stream) == hipSuccess
             ? LVSA_OK
             : LVSA_EDEVICE;
}

lvsa_status lvsa_attention_cache_workspace(const lvsa_tensor* q, int32_t q_start,
                                           const lvsa_kv_cache* cache,
                                           const lvsa_block_mask* mask, int64_t* bytes) {
  if (!bytes) return LVSA_EINVAL;
  CacheAttnArgs a;
  lvsa_status st;
  if ((st = cache_attention_args(q, q_start, cache, mask, &a)) != LVSA_OK) return st;
  int32_t cus = 0;
  if ((st = compute_units(&cus)) != LVSA_OK) return st;
  *bytes = cache_attention_workspace(a, cus);
  return LVSA_OK;
}

lvsa_status lvsa_attention_cache(const lvsa_tensor* q, int32_t q_start,
                                 const lvsa_kv_cache* cache, const lvsa_block_mask* mask,
                                 lvsa_tensor* out, void* workspace, int64_t workspace_bytes,
                                 void* stream) {
  CacheAttnArgs a;
  lvsa_status st;
  if (!out) return LVSA_EINVAL;
  if ((st = cache_attention_args(q, q_start, cache, mask, &a)) != LVSA_OK) return st;
  if ((st = check_output(out, q->heads, q->n_tokens)) != LVSA_OK) return st;
  if (out->data == q->data || out->data == cache->k || out->data == cache->v) return LVSA_EINVAL;
  int32_t cus = 0;
  if ((st = compute_units(&cus)) != LVSA_OK) return st;
  const int64_t need = cache_attention_workspace(a, cus);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return LVSA_EINVAL;
    if (!aligned(workspace, 16)) return LVSA_EUNSUPPORTED;
  }
  a.o = out->data;
  a.o_sh = out->stride_head, a.o_st = out->stride_token;
  a.workspace = (float*)workspace;
  return launch_cache_attention(a, cus, (hipStream_t)stream) == hipSuccess ? LVSA_OK
                                                                           : LVSA_EDEVICE;
}

}  // extern "C"
