// extern "C" entry points of the gradient operators: argument checks, then the launchers of iso_grad.h on the caller's
// stream.  Declarations and the meaning of every argument are in include/iso.h.
#include <hip/hip_runtime.h>

#include <cmath>

#include "iso.h"
#include "iso_device.h"
#include "iso_grad.h"

using namespace iso;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool is_dtype(int dt) { return dt == ISO_F32 || dt == ISO_BF16; }
bool is_flag(int v) { return v == 0 || v == 1; }

// Limits of one matrix, its padding and stride included: a launch of a workgroup per 2048 elements holds fewer than
// 2^32 threads.
constexpr int64_t kMaxDim = 1 << 24;
constexpr int64_t kMaxElems = 1ll << 34;
bool too_large(int64_t rows, int64_t ld) { return rows > 0 && ld > kMaxElems / rows; }

iso_status check_ptr(const void* p) {
  if (p == nullptr) return ISO_ERR_INVALID_ARG;
  return aligned16(p) ? ISO_OK : ISO_ERR_ALIGNMENT;
}

iso_status check_ws(const void* ws, size_t bytes, size_t need) {
  if (ws == nullptr) return ISO_ERR_WORKSPACE;
  if (((uintptr_t)ws & 255u) != 0) return ISO_ERR_ALIGNMENT;
  return bytes < need ? ISO_ERR_WORKSPACE : ISO_OK;
}

iso_status check_embed_sizes(const iso_embed* e) {
  if (e == nullptr) return ISO_ERR_INVALID_ARG;
  if (e->id_type != ISO_I32 && e->id_type != ISO_I64) return ISO_ERR_INVALID_ARG;
  if (e->tokens < 0 || e->vocab < 1 || e->dim < 1) return ISO_ERR_INVALID_ARG;
  if (e->tokens >= (1ll << 31) || e->vocab > ISO_EMBED_MAX_VOCAB || e->dim > ISO_EMBED_MAX_DIM) return ISO_ERR_UNSUPPORTED;
  return ISO_OK;
}

iso_status check_embed(const iso_embed* e) {
  iso_status st = check_embed_sizes(e);
  if (st != ISO_OK) return st;
  if (!std::isfinite((float)e->scale)) return ISO_ERR_INVALID_ARG;
  if (e->tokens == 0) return ISO_OK;
  if (e->ids == nullptr || e->ld_x < e->dim) return ISO_ERR_INVALID_ARG;
  if (((uintptr_t)e->ids & (e->id_type == ISO_I64 ? 7u : 3u)) != 0) return ISO_ERR_ALIGNMENT;
  if (too_large(e->tokens, e->ld_x)) return ISO_ERR_UNSUPPORTED;
  return check_ptr(e->x);
}

iso_status check_ckpt(const iso_ckpt& c) {
  if (c.rows < 0 || c.cols < 0) return ISO_ERR_INVALID_ARG;
  if (c.cols > kMaxDim || too_large(c.rows, ckpt_ld(c.cols))) return ISO_ERR_UNSUPPORTED;
  if (c.rows == 0 || c.cols == 0) return ISO_OK;
  iso_status st = check_ptr(c.q);
  return st != ISO_OK ? st : check_ptr(c.e);
}

iso_status check_ckpts(const iso_ckpt* c, int n, int dt) {
  if (n < 0 || (n > 0 && c == nullptr) || !is_dtype(dt)) return ISO_ERR_INVALID_ARG;
  for (int j = 0; j < n; ++j) {
    iso_status st = check_ckpt(c[j]);
    if (st != ISO_OK) return st;
    if (c[j].rows == 0 || c[j].cols == 0) continue;
    if (c[j].ld_x < c[j].cols) return ISO_ERR_INVALID_ARG;
    if (too_large(c[j].rows, c[j].ld_x)) return ISO_ERR_UNSUPPORTED;
    if ((st = check_ptr(c[j].x)) != ISO_OK) return st;
  }
  return ISO_OK;
}

// Sizes only with pointers == false (workspace queries).
iso_status check_weight_grads(const iso_weight_grad* g, int n, int dt, bool pointers) {
  if (n < 0 || (n > 0 && g == nullptr) || !is_dtype(dt)) return ISO_ERR_INVALID_ARG;
  for (int j = 0; j < n; ++j) {
    const iso_weight_grad& x = g[j];
    if (x.rows < 0 || x.in.rows < 0 || x.in.cols < 0) return ISO_ERR_INVALID_ARG;
    if (x.rows > kMaxDim || x.in.cols > kMaxDim || x.in.rows >= (1ll << 31) || too_large(x.rows, x.in.cols) ||
        too_large(x.in.rows, ckpt_ld(x.in.cols)))
      return ISO_ERR_UNSUPPORTED;
    if (x.rows == 0 || x.in.cols == 0) continue;
    if (x.in.rows > 0) {
      if (x.ld_dy < x.rows) return ISO_ERR_INVALID_ARG;
      if (too_large(x.in.rows, x.ld_dy)) return ISO_ERR_UNSUPPORTED;
    }
    if (!pointers) continue;
    iso_status st = check_ptr(x.grad);
    if (st != ISO_OK) return st;
    if (x.in.rows == 0) continue;
    if ((st = check_ckpt(x.in)) != ISO_OK) return st;
    if ((st = check_ptr(x.dy)) != ISO_OK) return st;
  }
  return ISO_OK;
}

// Rows of `cols` values with a stride that kernels read by 16 bytes.
iso_status check_rows(const void* p, int64_t ld, int64_t cols, int dt, bool pointers) {
  if (ld < cols) return ISO_ERR_INVALID_ARG;
  if (ld > ISO_ATTN_MAX_LD) return ISO_ERR_UNSUPPORTED;
  if (ld % (dt == ISO_BF16 ? 8 : 4) != 0) return ISO_ERR_ALIGNMENT;
  return pointers ? check_ptr(p) : ISO_OK;
}

iso_status check_words(const void* p) {
  if (p == nullptr) return ISO_ERR_INVALID_ARG;
  return ((uintptr_t)p & 3u) == 0 ? ISO_OK : ISO_ERR_ALIGNMENT;
}

// Sizes only with pointers == false (workspace queries, which read no strides either).
iso_status check_attn(const iso_attn* a, int dt, int grad, bool pointers) {
  if (a == nullptr || !is_dtype(dt) || !is_flag(grad)) return ISO_ERR_INVALID_ARG;
  if (a->sequences < 0 || a->tokens_q < 0 || a->tokens_k < 0 || a->heads < 1 || a->heads_kv < 1 || a->dim < 1)
    return ISO_ERR_INVALID_ARG;
  if (a->heads % a->heads_kv != 0 || !is_flag(a->causal) || a->window < 0) return ISO_ERR_INVALID_ARG;
  if (!std::isfinite((float)a->scale) || !((float)a->scale > 0.0f)) return ISO_ERR_INVALID_ARG;
  if (a->dim % 8 != 0 || a->dim > ISO_ATTN_MAX_DIM || a->sequences > ISO_ATTN_MAX_SEQUENCES) return ISO_ERR_UNSUPPORTED;
  if (a->heads > ISO_ATTN_MAX_LD / a->dim || !attend_fits(*a)) return ISO_ERR_UNSUPPORTED;
  if (!pointers || a->sequences == 0) return ISO_OK;
  const int64_t wide = (int64_t)a->heads * a->dim, narrow = (int64_t)a->heads_kv * a->dim;
  iso_status st;
  if ((st = check_words(a->start_q)) != ISO_OK || (st = check_words(a->start_k)) != ISO_OK) return st;
  if (a->tokens_q > 0) {
    if ((st = check_rows(a->q, a->ld_q, wide, dt, true)) != ISO_OK) return st;
    if ((st = check_rows(a->out, a->ld_out, wide, dt, true)) != ISO_OK) return st;
    if ((st = check_ptr(a->lse)) != ISO_OK) return st;
    if (grad != 0) {
      if ((st = check_rows(a->dout, a->ld_dout, wide, dt, true)) != ISO_OK) return st;
      if ((st = check_rows(a->dq, a->ld_dq, wide, dt, true)) != ISO_OK) return st;
    }
  }
  if (a->tokens_k > 0) {
    if ((st = check_rows(a->k, a->ld_k, narrow, dt, true)) != ISO_OK) return st;
    if ((st = check_rows(a->v, a->ld_v, narrow, dt, true)) != ISO_OK) return st;
    if (grad != 0) {
      if ((st = check_rows(a->dk, a->ld_dk, narrow, dt, true)) != ISO_OK) return st;
      if ((st = check_rows(a->dv, a->ld_dv, narrow, dt, true)) != ISO_OK) return st;
    }
  }
  return ISO_OK;
}

iso_status check_distill_sizes(const iso_distill* d) {
  if (d == nullptr || d->tokens < 0 || d->vocab < 1 || d->top < 1) return ISO_ERR_INVALID_ARG;
  if (d->id_type != ISO_I32 && d->id_type != ISO_I64) return ISO_ERR_INVALID_ARG;
  if (d->tokens > ISO_DISTILL_MAX_TOKENS || d->vocab > ISO_EMBED_MAX_VOCAB || d->top > ISO_DISTILL_MAX_TOP) return ISO_ERR_UNSUPPORTED;
  return ISO_OK;
}

iso_status check_distill(const iso_distill* d, int dt, bool loss, bool grad) {
  iso_status st = check_distill_sizes(d);
  if (st != ISO_OK) return st;
  const float t = (float)d->temperature, inv = (float)(1.4426950408889634 / d->temperature);   // log2(e) / T, the kernels' factor
  if (!is_dtype(dt) || !std::isfinite(t) || !(t > 0.0f) || !std::isfinite(inv) || !(inv > 0.0f)) return ISO_ERR_INVALID_ARG;
  if (d->tokens == 0) return ISO_OK;
  if (d->ids == nullptr || d->ld < d->vocab) return ISO_ERR_INVALID_ARG;
  if (((uintptr_t)d->ids & (d->id_type == ISO_I64 ? 7u : 3u)) != 0) return ISO_ERR_ALIGNMENT;
  if (too_large(d->tokens, d->ld)) return ISO_ERR_UNSUPPORTED;
  if ((st = check_ptr(d->logits)) != ISO_OK || (st = check_ptr(d->teacher)) != ISO_OK || (st = check_ptr(d->lse)) != ISO_OK) return st;
  if (d->weight != nullptr && (st = check_ptr(d->weight)) != ISO_OK) return st;
  if (loss && (st = check_ptr(d->loss)) != ISO_OK) return st;
  if (!grad) return ISO_OK;
  if (d->ld_grad < d->vocab || (d->grad == d->logits && d->ld_grad != d->ld)) return ISO_ERR_INVALID_ARG;
  if (too_large(d->tokens, d->ld_grad)) return ISO_ERR_UNSUPPORTED;
  return check_ptr(d->grad);
}

iso_status from_hip(hipError_t e) { return e == hipSuccess ? ISO_OK : ISO_ERR_HIP; }

}  // namespace

extern "C" {

size_t iso_workspace_size_embed(const iso_embed* e) {
  if (check_embed_sizes(e) != ISO_OK) return 0;
  return embed_plan(e->tokens, e->vocab, e->dim).total;
}

iso_status iso_embed_lookup(const iso_embed* e, int dt, void* ws, size_t ws_bytes, void* stream) {
  iso_status st = check_embed(e);
  if (st != ISO_OK) return st;
  if (!is_dtype(dt)) return ISO_ERR_INVALID_ARG;
  if ((st = check_ptr(e->table)) != ISO_OK) return st;
  if ((st = check_ws(ws, ws_bytes, kStatusBytes)) != ISO_OK) return st;
  return from_hip(run_embed_lookup(*e, dt, (uint8_t*)ws, (hipStream_t)stream));
}

iso_status iso_embed_grad(const iso_embed* e, int dt, int dt_grad, int accumulate, void* ws, size_t ws_bytes,
                          void* stream) {
  iso_status st = check_embed(e);
  if (st != ISO_OK) return st;
  if (!is_dtype(dt) || !is_dtype(dt_grad) || !is_flag(accumulate)) return ISO_ERR_INVALID_ARG;
  if ((st = check_ptr(e->grad)) != ISO_OK) return st;
  if ((st = check_ws(ws, ws_bytes, embed_plan(e->tokens, e->vocab, e->dim).total)) != ISO_OK) return st;
  return from_hip(run_embed_grad(*e, dt, dt_grad, accumulate != 0, (uint8_t*)ws, (hipStream_t)stream));
}

int64_t iso_ckpt_ld(int64_t cols) { return cols < 0 || cols > INT64_MAX - ISO_CKPT_GROUP ? -1 : ckpt_ld(cols); }

iso_status iso_ckpt_pack(const iso_ckpt* c, int n, int dt, void* stream) {
  const iso_status st = check_ckpts(c, n, dt);
  return st != ISO_OK ? st : from_hip(run_ckpt_pack(c, n, dt, (hipStream_t)stream));
}

iso_status iso_ckpt_unpack(const iso_ckpt* c, int n, int dt, void* stream) {
  const iso_status st = check_ckpts(c, n, dt);
  return st != ISO_OK ? st : from_hip(run_ckpt_unpack(c, n, dt, (hipStream_t)stream));
}

iso_status iso_ckpt_gate_grad(const iso_gate_grad* g, int n, int dt, void* stream) {
  if (n < 0 || (n > 0 && g == nullptr) || !is_dtype(dt)) return ISO_ERR_INVALID_ARG;
  for (int j = 0; j < n; ++j) {
    const iso_gate_grad& x = g[j];
    iso_status st = check_ckpt(x.gate);
    if (st != ISO_OK || (st = check_ckpt(x.up)) != ISO_OK) return st;
    if (x.gate.rows != x.up.rows || x.gate.cols != x.up.cols) return ISO_ERR_INVALID_ARG;
    if (x.gate.rows == 0 || x.gate.cols == 0) continue;
    if (x.ld < x.gate.cols) return ISO_ERR_INVALID_ARG;
    if (too_large(x.gate.rows, x.ld)) return ISO_ERR_UNSUPPORTED;
    const void* const p[3] = {x.dh, x.dgate, x.dup};
    for (const void* v : p)
      if ((st = check_ptr(v)) != ISO_OK) return st;
  }
  return from_hip(run_gate_grad(g, n, dt, (hipStream_t)stream));
}

size_t iso_workspace_size_weight_grad(const iso_weight_grad* g, int n, int dt) {
  if (check_weight_grads(g, n, dt, false) != ISO_OK) return 0;
  return weight_grad_workspace_bytes(g, n, dt);
}

iso_status iso_ckpt_weight_grad(const iso_weight_grad* g, int n, int dt, int dt_grad, int accumulate, void* ws,
                                size_t ws_bytes, void* stream) {
  iso_status st = check_weight_grads(g, n, dt, true);
  if (st != ISO_OK) return st;
  if (!is_dtype(dt_grad) || !is_flag(accumulate)) return ISO_ERR_INVALID_ARG;
  if ((st = check_ws(ws, ws_bytes, weight_grad_workspace_bytes(g, n, dt))) != ISO_OK) return st;
  return from_hip(run_weight_grad(g, n, dt, dt_grad, accumulate != 0, (uint8_t*)ws, (hipStream_t)stream));
}

size_t iso_workspace_size_attend(const iso_attn* a, int dt, int grad) {
  if (check_attn(a, dt, grad, false) != ISO_OK) return 0;
  return attend_workspace_bytes(*a, dt, grad != 0);
}

iso_status iso_attend(const iso_attn* a, int dt, void* ws, size_t ws_bytes, void* stream) {
  iso_status st = check_attn(a, dt, 0, true);
  if (st != ISO_OK) return st;
  if ((st = check_ws(ws, ws_bytes, attend_workspace_bytes(*a, dt, false))) != ISO_OK) return st;
  return from_hip(run_attend(*a, dt, (uint8_t*)ws, (hipStream_t)stream));
}

iso_status iso_attend_grad(const iso_attn* a, int dt, void* ws, size_t ws_bytes, void* stream) {
  iso_status st = check_attn(a, dt, 1, true);
  if (st != ISO_OK) return st;
  if ((st = check_ws(ws, ws_bytes, attend_workspace_bytes(*a, dt, true))) != ISO_OK) return st;
  return from_hip(run_attend_grad(*a, dt, (uint8_t*)ws, (hipStream_t)stream));
}

size_t iso_workspace_size_distill(const iso_distill* d) {
  return check_distill_sizes(d) == ISO_OK ? distill_workspace_bytes() : 0;
}

iso_status iso_distill_loss(const iso_distill* d, int dt, void* ws, size_t ws_bytes, void* stream) {
  iso_status st = check_distill(d, dt, true, d != nullptr && d->grad != nullptr);
  if (st != ISO_OK) return st;
  if ((st = check_ws(ws, ws_bytes, distill_workspace_bytes())) != ISO_OK) return st;
  return from_hip(run_distill_loss(*d, dt, (uint8_t*)ws, (hipStream_t)stream));
}

iso_status iso_distill_grad(const iso_distill* d, int dt, void* ws, size_t ws_bytes, void* stream) {
  iso_status st = check_distill(d, dt, false, true);
  if (st != ISO_OK) return st;
  if ((st = check_ws(ws, ws_bytes, distill_workspace_bytes())) != ISO_OK) return st;
  return from_hip(run_distill_grad(*d, dt, (uint8_t*)ws, (hipStream_t)stream));
}

}  // extern "C"
