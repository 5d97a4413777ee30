// api_train.cpp -- the C ABI of attention's gradients and of the residual step with its
// gradients (lvsa.h): argument checks and dispatch.
#include <climits>
#include <utility>

#include "residual_norm.h"

namespace lvsa {
namespace {

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

bool known_type(int32_t dtype) {
  return dtype == LVSA_BF16 || dtype == LVSA_F16 || dtype == LVSA_F32;
}
bool known_norm(int32_t kind) {
  return kind == LVSA_NORM_NONE || kind == LVSA_NORM_LAYER || kind == LVSA_NORM_RMS;
}

// A tensor that attention's gradients read: [heads, n, 128], with 32-bit offsets within a
// head.
lvsa_status check_read(const lvsa_tensor* t, int32_t heads, int32_t n) {
  const lvsa_status st = check_tensor(t, heads, n);
  if (st != LVSA_OK) return st;
  return ((int64_t)n + 127) / 128 * 128 * t->stride_token * 2 >= ((int64_t)1 << 32)
             ? LVSA_EUNSUPPORTED
             : LVSA_OK;
}

// The rows' statistics take four work-items a row: below 2^31 in a launch.  (The items' launch
// has its own bound, attention_backward_workspace.)
bool too_long(int32_t heads, int32_t n) { return (int64_t)heads * n >= (int64_t)1 << 29; }

// The step's parameters and the rows of each frame; n rows.
lvsa_status norm_args(const lvsa_residual_norm* p, int32_t n, bool backward, NormArgs* a) {
  if (!p || n < 1) return LVSA_EINVAL;
  if (p->dim < 1 || p->frame_tokens < 0 || !known_norm(p->norm) || !known_norm(p->post) ||
      !known_type(p->stream_type) || !known_type(p->block_type) || !known_type(p->param_type) ||
      !(p->eps >= 0.f) || !(p->eps < __builtin_inff()))
    return LVSA_EINVAL;
  if (!p->scale != !p->shift) return LVSA_EINVAL;
  if (p->norm == LVSA_NORM_NONE && (p->scale || p->weight || p->bias)) return LVSA_EINVAL;
  if (p->post == LVSA_NORM_NONE && p->post_weight) return LVSA_EINVAL;
  if (p->dim % 8 != 0 || p->dim > LVSA_MAX_NORM_DIM) return LVSA_EUNSUPPORTED;
  if (p->stream_type != p->block_type && p->stream_type != LVSA_F32) return LVSA_EUNSUPPORTED;
  for (const void* x : {p->gate, p->scale, p->shift, p->weight, p->bias, p->post_weight})
    if (!aligned(x, 16)) return LVSA_EUNSUPPORTED;
  *a = NormArgs{};
  a->n = n;
  a->dim = p->dim;
  const bool frames = p->gate || p->scale;
  a->frame = frames && p->frame_tokens > 0 && p->frame_tokens < n ? p->frame_tokens : n;
  for (auto [x, st] : {std::pair{p->gate, p->gate_stride}, std::pair{p->scale, p->scale_stride},
                       std::pair{p->shift, p->shift_stride}})
    if (x && a->frame < n) {
      if (st < 0) return LVSA_EINVAL;
      if (st % 8 != 0) return LVSA_EUNSUPPORTED;
    }
  a->frames = (int32_t)(((int64_t)n + a->frame - 1) / a->frame);
  a->norm = p->norm, a->post = p->post, a->param_type = p->param_type;
  a->eps = p->eps, a->a = p->residual;
  a->gate = p->gate, a->scale = p->scale, a->shift = p->shift;
  a->gate_st = p->gate_stride, a->scale_st = p->scale_stride, a->shift_st = p->shift_stride;
  a->weight = p->weight, a->bias = p->bias, a->post_weight = p->post_weight;
  norm_units(*a, backward);
  // Work-items of a launch; back, of that which adds up frames too.
  if (backward && a->frames > 1 << 22) return LVSA_EUNSUPPORTED;
  if ((int64_t)a->frames * a->units * norm_team(a->dim).threads + 1024 > INT32_MAX)
    return LVSA_EUNSUPPORTED;
  return LVSA_OK;
}

lvsa_status check_rows(const lvsa_rows* t, int32_t n) {
  if (!t || !t->data || t->n != n) return LVSA_EINVAL;
  if (n > 1 && t->stride < 0) return LVSA_EINVAL;
  if (!aligned(t->data, 16) || (n > 1 && t->stride % 8 != 0)) return LVSA_EUNSUPPORTED;
  return LVSA_OK;
}
// Rows that are written: they share no elements, nor any with `same` unless they are it.
lvsa_status check_written(const lvsa_rows* t, int32_t n, int32_t dim) {
  const lvsa_status st = check_rows(t, n);
  if (st != LVSA_OK) return st;
  return n > 1 && t->stride < dim ? LVSA_EINVAL : LVSA_OK;
}
bool in_place(const lvsa_rows* in, const lvsa_rows* out) {
  return in->n == 1 || in->stride == out->stride;
}

}  // namespace
}  // namespace lvsa

using namespace lvsa;

extern "C" {

lvsa_status lvsa_attention_backward_workspace(const lvsa_tensor* q, const lvsa_block_mask* mask,
                                              int64_t* bytes) {
  if (!q || !bytes || q->heads < 1 || q->n_tokens < 1) return LVSA_EINVAL;
  if (too_long(q->heads, q->n_tokens)) return LVSA_EUNSUPPORTED;
  int32_t nb = (int32_t)(((int64_t)q->n_tokens + 127) / 128);
  bool sparse = false;
  if (mask) {
    if (mask->block != 64 && mask->block != 128) return LVSA_EUNSUPPORTED;
    if (mask->n_tokens != q->n_tokens || !mask->row_ptr != !mask->col_idx) return LVSA_EINVAL;
    nb = (int32_t)(((int64_t)q->n_tokens + mask->block - 1) / mask->block);
    if (mask->n_q_blocks != nb || mask->n_kv_blocks != nb) return LVSA_EINVAL;
    sparse = mask->row_ptr != nullptr;
    if (sparse && nb > kMaxSparseBlocks) return LVSA_EUNSUPPORTED;
    if (!sparse) nb = (int32_t)(((int64_t)q->n_tokens + 127) / 128);
  }
  const int64_t need = attention_backward_workspace(q->heads, q->n_tokens, nb, sparse);
  if (need < 0) return LVSA_EUNSUPPORTED;
  *bytes = need;
  return LVSA_OK;
}

lvsa_status lvsa_attention_backward(const lvsa_tensor* grad_out, const lvsa_tensor* q,
                                    const lvsa_tensor* k, const lvsa_tensor* v,
                                    const lvsa_tensor* out, const float* lse,
                                    const lvsa_block_mask* mask, lvsa_tensor* grad_q,
                                    lvsa_tensor* grad_k, lvsa_tensor* grad_v, void* workspace,
                                    int64_t workspace_bytes, void* stream) {
  if (!out || !lse || !grad_out) return LVSA_EINVAL;
  AttnBackArgs a;
  lvsa_tensor o = *out;
  lvsa_status st;
  if ((st = train_attention_args(q, k, v, mask, &o, &a.f)) != LVSA_OK) return st;
  const int32_t H = q->heads, n = q->n_tokens;
  if (too_long(H, n)) return LVSA_EUNSUPPORTED;
  if ((st = check_read(q, H, n)) != LVSA_OK) return st;
  if ((st = check_read(grad_out, H, n)) != LVSA_OK) return st;
  if (!aligned(lse, 4)) return LVSA_EUNSUPPORTED;
  const void* const in[] = {grad_out->data, q->data, k->data, v->data, out->data, lse};
  lvsa_tensor* const grads[] = {grad_q, grad_k, grad_v};
  for (lvsa_tensor* g : grads) {
    if ((st = check_output(g, H, n)) != LVSA_OK) return st;
    for (const void* x : in)
      if (g->data == x) return LVSA_EINVAL;
  }
  if (grad_q->data == grad_k->data || grad_q->data == grad_v->data ||
      grad_k->data == grad_v->data)
    return LVSA_EINVAL;
  a.block = mask ? mask->block : 128;
  if (!a.f.row_ptr) {   // every block: the walk is of 128-token ones
    a.block = 128;
    a.f.n_blocks = (int32_t)(((int64_t)n + 127) / 128);
  }
  const int64_t need = attention_backward_workspace(H, n, a.f.n_blocks, a.f.row_ptr != nullptr);
  if (need < 0) return LVSA_EUNSUPPORTED;
  if (!workspace || workspace_bytes < need) return LVSA_EINVAL;
  if (!aligned(workspace, 16)) return LVSA_EUNSUPPORTED;
  a.f.lse = const_cast<float*>(lse);
  a.go = grad_out->data, a.go_sh = grad_out->stride_head, a.go_st = grad_out->stride_token;
  a.gq = grad_q->data, a.gq_sh = grad_q->stride_head, a.gq_st = grad_q->stride_token;
  a.gk = grad_k->data, a.gk_sh = grad_k->stride_head, a.gk_st = grad_k->stride_token;
  a.gv = grad_v->data, a.gv_sh = grad_v->stride_head, a.gv_st = grad_v->stride_token;
  a.workspace = (char*)workspace;
  return launch_attention_backward(a, (hipStream_t)stream) == hipSuccess ? LVSA_OK : LVSA_EDEVICE;
}

lvsa_status lvsa_residual_norm_forward(const lvsa_residual_norm* p, const lvsa_rows* x,
                                       const lvsa_rows* y, lvsa_rows* r, lvsa_rows* h,
                                       void* stream) {
  if (!p || !x) return LVSA_EINVAL;
  NormArgs a;
  lvsa_status st;
  if ((st = norm_args(p, x->n, false, &a)) != LVSA_OK) return st;
  if ((st = check_rows(x, x->n)) != LVSA_OK) return st;
  if (p->norm == LVSA_NORM_NONE ? h != nullptr : h == nullptr) return LVSA_EINVAL;
  if (y) {
    if ((st = check_rows(y, x->n)) != LVSA_OK) return st;
    if ((st = check_written(r, x->n, p->dim)) != LVSA_OK) return st;
    if (r->data == y->data || (r->data == x->data && !in_place(x, r))) return LVSA_EINVAL;
    a.y = y->data, a.y_st = y->stride;
    a.r = r->data, a.r_st = r->stride;
  } else if (r || p->gate || p->post != LVSA_NORM_NONE || p->residual != 1.f ||
             p->norm == LVSA_NORM_NONE) {
    return LVSA_EINVAL;
  }
  if (h) {
    if ((st = check_written(h, x->n, p->dim)) != LVSA_OK) return st;
    if (r && h->data == r->data) return LVSA_EINVAL;
    if (y && h->data == y->data && !in_place(y, h)) return LVSA_EINVAL;
    if (h->data == x->data && (y || !in_place(x, h) || p->stream_type != p->block_type))
      return LVSA_EINVAL;
    a.h = h->data, a.h_st = h->stride;
  }
  a.x = x->data, a.x_st = x->stride;
  return launch_norm_forward(a, p->stream_type, p->block_type, (hipStream_t)stream) == hipSuccess
             ? LVSA_OK
             : LVSA_EDEVICE;
}

namespace {

// The step's arguments with the gradients that are wanted.
lvsa_status norm_grads(const lvsa_residual_norm* p, int32_t n, const lvsa_residual_norm_grads* g,
                       NormArgs* a) {
  if (!p || !g) return LVSA_EINVAL;
  const lvsa_status st = norm_args(p, n, true, a);
  if (st != LVSA_OK) return st;
  const std::pair<const void*, void*> given[] = {
      {p->gate, g->gate}, {p->scale, g->scale}, {p->shift, g->shift},
      {p->weight, g->weight}, {p->bias, g->bias}, {p->post_weight, g->post_weight}};
  for (auto [x, grad] : given) {
    if (grad && (!x || grad == x)) return LVSA_EINVAL;
    if (!aligned(grad, 16)) return LVSA_EUNSUPPORTED;
  }
  a->d_gate = g->gate, a->d_scale = g->scale, a->d_shift = g->shift;
  a->d_weight = g->weight, a->d_bias = g->bias, a->d_post_weight = g->post_weight;
  return LVSA_OK;
}

}  // namespace

lvsa_status lvsa_residual_norm_workspace(const lvsa_residual_norm* p, int32_t n,
                                         const lvsa_residual_norm_grads* grads, int64_t* bytes) {
  if (!bytes) return LVSA_EINVAL;
  NormArgs a;
  const lvsa_status st = norm_grads(p, n, grads, &a);
  if (st != LVSA_OK) return st;
  *bytes = norm_workspace(a);
  return LVSA_OK;
}

lvsa_status lvsa_residual_norm_backward(const lvsa_residual_norm* p, const lvsa_rows* grad_h,
                                        const lvsa_rows* grad_r, const lvsa_rows* r,
                                        const lvsa_rows* y,
                                        const lvsa_residual_norm_grads* grads, void* workspace,
                                        int64_t workspace_bytes, void* stream) {
  if (!p || !grads) return LVSA_EINVAL;
  // Without a norm the gradients do not depend on r, which may then be NULL.
  const lvsa_rows* const some = p->norm == LVSA_NORM_NONE ? grad_r : r;
  if (!some) return LVSA_EINVAL;
  const int32_t n = some->n;
  NormArgs a;
  lvsa_status st;
  if ((st = norm_grads(p, n, grads, &a)) != LVSA_OK) return st;
  if (p->norm == LVSA_NORM_NONE ? grad_h != nullptr : grad_h == nullptr) return LVSA_EINVAL;
  const lvsa_rows* const in[] = {grad_h, grad_r, r, y};
  for (const lvsa_rows* t : in)
    if (t && (st = check_rows(t, n)) != LVSA_OK) return st;
  const lvsa_rows *gx = grads->x.data ? &grads->x : nullptr,
                  *gy = grads->y.data ? &grads->y : nullptr;
  if (!y && (gy || p->gate || p->post != LVSA_NORM_NONE || p->residual != 1.f ||
             p->norm == LVSA_NORM_NONE))
    return LVSA_EINVAL;
  if (gx) {
    if ((st = check_written(gx, n, p->dim)) != LVSA_OK) return st;
    for (const lvsa_rows* t : in)
      if (t && t->data == gx->data && (t != grad_r || !in_place(t, gx))) return LVSA_EINVAL;
    a.r = gx->data, a.r_st = gx->stride;
  }
  if (gy) {
    if ((st = check_written(gy, n, p->dim)) != LVSA_OK) return st;
    for (const lvsa_rows* t : in)
      if (t && t->data == gy->data && (t != grad_h || !in_place(t, gy))) return LVSA_EINVAL;
    if (gx && gx->data == gy->data) return LVSA_EINVAL;
    a.h = gy->data, a.h_st = gy->stride;
  }
  if (r) a.x = r->data, a.x_st = r->stride;
  if (y) a.y = y->data, a.y_st = y->stride;
  if (grad_h) a.gh = grad_h->data, a.gh_st = grad_h->stride;
  if (grad_r) a.gr = grad_r->data, a.gr_st = grad_r->stride;
  const int64_t need = norm_workspace(a);
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return LVSA_EINVAL;
    if (!aligned(workspace, 16)) return LVSA_EUNSUPPORTED;
    a.partial = (float*)workspace;
  }
  return launch_norm_backward(a, p->stream_type, p->block_type, (hipStream_t)stream) == hipSuccess
             ? LVSA_OK
             : LVSA_EDEVICE;
}

}  // extern "C"
