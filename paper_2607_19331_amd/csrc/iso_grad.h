// Host-side launchers of the gradient operators: embeddings and 8-bit activation checkpoints (internal to
// the library; arguments are checked in iso_grad_abi.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "iso.h"

namespace iso {

// Workspace regions of the embedding's gradient (many tokens; few take the status block alone).
struct EmbedPlan {
  int64_t tiles = 0, tile = 0;     // tokens are counted and scattered by tiles of `tile`
  int64_t most_runs = 0;           // partial sums of ids with many tokens
  size_t bad = 0, hist = 0, bucket0 = 0, pairs = 0, perm = 0, listed = 0, ids = 0, runs = 0, many = 0, part = 0, total = 0;
};

EmbedPlan embed_plan(int64_t tokens, int64_t vocab, int64_t dim);
hipError_t run_embed_lookup(const iso_embed& e, int dt, uint8_t* ws, hipStream_t s);
hipError_t run_embed_grad(const iso_embed& e, int dt, int dt_grad, bool accumulate, uint8_t* ws, hipStream_t s);

inline int64_t ckpt_ld(int64_t cols) { return (cols + ISO_CKPT_GROUP - 1) / ISO_CKPT_GROUP * ISO_CKPT_GROUP; }

hipError_t run_ckpt_pack(const iso_ckpt* c, int n, int dt, hipStream_t s);
hipError_t run_ckpt_unpack(const iso_ckpt* c, int n, int dt, hipStream_t s);
hipError_t run_gate_grad(const iso_gate_grad* g, int n, int dt, hipStream_t s);

size_t weight_grad_workspace_bytes(const iso_weight_grad* g, int n, int dt);
hipError_t run_weight_grad(const iso_weight_grad* g, int n, int dt, int dt_grad, bool accumulate, uint8_t* ws,
                           hipStream_t s);

}  // namespace iso
