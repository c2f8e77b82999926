// Host-side launchers of the gradient operators: embeddings, 8-bit activation checkpoints, attention and distillation
// (internal to the library; arguments are checked in iso_grad_abi.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "iso.h"
#include "iso_grad_plan.h"

namespace iso {

hipError_t run_embed_lookup(const iso_embed& e, int dt, uint8_t* ws, hipStream_t s);
hipError_t run_embed_grad(const iso_embed& e, int dt, int dt_grad, bool accumulate, uint8_t* ws, hipStream_t s);

hipError_t run_ckpt_pack(const iso_ckpt* c, int n, int dt, hipStream_t s);
hipError_t run_ckpt_unpack(const iso_ckpt* c, int n, int dt, hipStream_t s);
hipError_t run_gate_grad(const iso_gate_grad* g, int n, int dt, hipStream_t s);

hipError_t run_weight_grad(const iso_weight_grad* g, int n, int dt, int dt_grad, bool accumulate, uint8_t* ws,
                           hipStream_t s);

hipError_t run_attend(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s);
hipError_t run_attend_grad(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s);

hipError_t run_distill_loss(const iso_distill& d, int dt, uint8_t* ws, hipStream_t s);
hipError_t run_distill_grad(const iso_distill& d, int dt, uint8_t* ws, hipStream_t s);

}  // namespace iso
