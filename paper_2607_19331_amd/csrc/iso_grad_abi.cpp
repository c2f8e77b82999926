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

}  // extern "C"
