// Element access shared by the gradient operators' kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iso_device.h"

namespace iso {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// V consecutive elements of storage type DT from element index i on, widened to binary32.  V = 1 or i * size a
// multiple of min(16, V * size) bytes.
template <int DT, int V>
__device__ __forceinline__ void load_elems(const void* p, int64_t i, float* v) {
  if constexpr (DT == ISO_BF16) {
    const auto* q = gmem((const uint16_t*)p) + i;
    if constexpr (V == 1) {
      v[0] = f32_from_bits((uint32_t)*q << 16);
    } else {
      uint32_t w[V / 2];
      if constexpr (V == 4) {
        const u32x2_t t = *(const __attribute__((address_space(1))) u32x2_t*)q;
        w[0] = t.x, w[1] = t.y;
      } else {
        static_assert(V == 8, "bf16 vectors hold 4 or 8");
        const u32x4_t t = *(const __attribute__((address_space(1))) u32x4_t*)q;
        w[0] = t.x, w[1] = t.y, w[2] = t.z, w[3] = t.w;
      }
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        v[2 * j] = f32_from_bits(w[j] << 16);
        v[2 * j + 1] = f32_from_bits(w[j] & 0xFFFF0000u);
      }
    }
  } else {
    const auto* q = gmem((const float*)p) + i;
    if constexpr (V == 1) {
      v[0] = *q;
    } else {
#pragma unroll
      for (int j = 0; j < V / 4; ++j) {
        const f32x4_t t = ((const __attribute__((address_space(1))) f32x4_t*)q)[j];
        v[4 * j] = t.x, v[4 * j + 1] = t.y, v[4 * j + 2] = t.z, v[4 * j + 3] = t.w;
      }
    }
  }
}

// Two values to bf16, round to nearest even (NaN stays NaN), lo in bits 0-15.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const iso_f32x2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, iso_bf16x2_t));
}

// V values rounded to storage type DT; STREAM: not kept in the caches (outputs larger than these).
template <int DT, int V, bool STREAM = false>
__device__ __forceinline__ void store_elems(void* p, int64_t i, const float* v) {
  if constexpr (DT == ISO_BF16) {
    auto* q = gmem((uint16_t*)p) + i;
    if constexpr (V == 1) {
      *q = (uint16_t)pack_bf16(v[0], 0.0f);
    } else if constexpr (V == 4) {
      const u32x2_t t = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
      auto* o = (__attribute__((address_space(1))) u32x2_t*)q;
      if constexpr (STREAM) __builtin_nontemporal_store(t, o);
      else *o = t;
    } else {
      static_assert(V == 8, "bf16 vectors hold 4 or 8");
      const u32x4_t t = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
      auto* o = (__attribute__((address_space(1))) u32x4_t*)q;
      if constexpr (STREAM) __builtin_nontemporal_store(t, o);
      else *o = t;
    }
  } else {
    auto* q = gmem((float*)p) + i;
    if constexpr (V == 1) {
      *q = v[0];
    } else {
#pragma unroll
      for (int j = 0; j < V / 4; ++j) {
        const f32x4_t t = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
        auto* o = (__attribute__((address_space(1))) f32x4_t*)q + j;
        if constexpr (STREAM) __builtin_nontemporal_store(t, o);
        else *o = t;
      }
    }
  }
}

// Whether rows of `dim` elements at stride ld can be read V at a time from a 16-byte aligned base.
inline bool vector_rows(int64_t dim, int64_t ld, int v) { return dim % v == 0 && ld % v == 0; }

}  // namespace iso
