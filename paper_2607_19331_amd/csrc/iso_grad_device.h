// Element access shared by the gradient operators' kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iso_device.h"

namespace iso {

// Vectors at any element's address: rows of odd length or stride are read and written 16 bytes a lane like others (global
// memory takes them; a vector that crosses a line costs one more request).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

template <class T>
using global_ptr = __attribute__((address_space(1))) T*;

// 16 bytes hold kVec<DT> elements.
template <int DT>
constexpr int kVec = DT == ISO_BF16 ? 8 : 4;

// The 16 bytes from element i on; of the `left` elements before the row's end where these are fewer, zeros after.
template <int DT>
__device__ __forceinline__ u32x4_t load_raw(const void* p, int64_t i, int64_t left = 16) {
  using bits = typename Fmt<DT>::bits_t;
  const auto q = gmem((const bits*)p) + i;
  if (left >= kVec<DT>) return *(global_ptr<const u32x4_any>)q;
  u32x4_t w = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < kVec<DT>; ++j) {
    if (j >= left) continue;
    if constexpr (DT == ISO_BF16) w[j / 2] |= (uint32_t)q[j] << (16 * (j & 1));
    else w[j] = q[j];
  }
  return w;
}

template <int DT>
__device__ __forceinline__ void unpack_raw(u32x4_t w, float* v) {
#pragma unroll
  for (int j = 0; j < kVec<DT>; ++j) {
    if constexpr (DT == ISO_BF16) v[j] = f32_from_bits((j & 1) ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    else v[j] = f32_from_bits(w[j]);
  }
}

// Two values to bf16, round to nearest even (NaN stays NaN), lo in bits 0-15.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const iso_f32x2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, iso_bf16x2_t));
}

// V elements (a multiple of 4) from element i on as binary32, those past the first `left` zero.
template <int DT, int V>
__device__ __forceinline__ void load_elems(const void* p, int64_t i, float* v, int64_t left = V) {
  if constexpr (V > kVec<DT>) {
    load_elems<DT, V / 2>(p, i, v, left);
    load_elems<DT, V / 2>(p, i + V / 2, v + V / 2, left - V / 2);
  } else if constexpr (V == kVec<DT>) {
    unpack_raw<DT>(load_raw<DT>(p, i, left), v);
  } else {
    static_assert(DT == ISO_BF16 && V == 4, "vectors hold 4 or 8 elements");
    const auto q = gmem((const uint16_t*)p) + i;
    u32x2_t w = {0, 0};
    if (left >= V) {
      w = *(global_ptr<const u32x2_any>)q;
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < left) w[j / 2] |= (uint32_t)q[j] << (16 * (j & 1));
    }
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = f32_from_bits((j & 1) ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
  }
}

template <bool STREAM>
__device__ __forceinline__ void put(u32x4_any w, global_ptr<u32x4_any> to) {
  if constexpr (STREAM) __builtin_nontemporal_store(w, to);
  else *to = w;
}
template <bool STREAM>
__device__ __forceinline__ void put(u32x2_any w, global_ptr<u32x2_any> to) {
  if constexpr (STREAM) __builtin_nontemporal_store(w, to);
  else *to = w;
}

// Outputs that the L2 caches (8 x 4 MiB) do not hold are written past them: a lookup of 117 MB takes 28 instead of 40 us,
// 1.7 GB of checkpoints there and back 285 instead of 299.  Smaller ones are left there for whoever reads them next.
inline bool streamed(int64_t bytes) { return bytes > (32ll << 20); }

// V values (a multiple of 4) rounded to storage type DT, of them the first `left`; STREAM: written past the caches.
template <int DT, int V, bool STREAM = false>
__device__ __forceinline__ void store_elems(void* p, int64_t i, const float* v, int64_t left = V) {
  using bits = typename Fmt<DT>::bits_t;
  const auto q = gmem((bits*)p) + i;
  if constexpr (V > kVec<DT>) {
    store_elems<DT, V / 2, STREAM>(p, i, v, left);
    store_elems<DT, V / 2, STREAM>(p, i + V / 2, v + V / 2, left - V / 2);
  } else if (left >= V) {
    if constexpr (DT == ISO_F32) {
      const u32x4_any w = {bits_from_f32(v[0]), bits_from_f32(v[1]), bits_from_f32(v[2]), bits_from_f32(v[3])};
      put<STREAM>(w, (global_ptr<u32x4_any>)q);
    } else if constexpr (V == 8) {
      const u32x4_any w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
      put<STREAM>(w, (global_ptr<u32x4_any>)q);
    } else {
      const u32x2_any w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
      put<STREAM>(w, (global_ptr<u32x2_any>)q);
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (j >= left) continue;
      if constexpr (DT == ISO_F32) q[j] = bits_from_f32(v[j]);
      else q[j] = (uint16_t)pack_bf16(v[j], 0.0f);
    }
  }
}

}  // namespace iso
