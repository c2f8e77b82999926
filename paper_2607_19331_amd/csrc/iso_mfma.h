// Matrix instructions and loads straight into LDS, as the kernels that feed them by hand use them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iso_device.h"

namespace iso {

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t* lds_frag;
typedef __attribute__((address_space(3))) f32x4_t* lds_f32x4;
typedef uint32_t lds_u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) const lds_u32x2_t* lds_pair;
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// v minus both bf16 values of a pair.
__device__ __forceinline__ float minus_pair(uint32_t pair, float v) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), __builtin_bit_cast(bf16x2_t, 0xBF80BF80u), v, false);
}

// Descriptor of a buffer of `left` bytes: reads past its end give zeros.
__device__ __forceinline__ u32x4_t buffer_of(const uint8_t* p, int64_t left) {
  const uint64_t a = (uint64_t)p;
  const uint32_t n = left <= 0 ? 0u : left > 0xFFFFFFF0ll ? 0xFFFFFFF0u : (uint32_t)left;
  return u32x4_t{(uint32_t)a, (uint32_t)(a >> 32) & 0xFFFFu, n, 0x00027000u};
}

// The same with the scalar unit alone (it compares no 64 bits), for at most 2 GiB: offsets from there on are outside.
__device__ __forceinline__ u32x4_t scalar_buffer_of(const uint8_t* p, int64_t left) {
  const uint64_t a = (uint64_t)p;
  const int32_t hi = (int32_t)(left >> 32);
  const uint32_t lo = (uint32_t)left, n = hi < 0 ? 0u : hi > 0 || lo > 0x80000000u ? 0x80000000u : lo;
  u32x4_t b = {(uint32_t)a, (uint32_t)(a >> 32) & 0xFFFFu, n, 0x00027000u};
#pragma unroll
  for (int j = 0; j < 4; ++j) b[j] = __builtin_amdgcn_readfirstlane(b[j]);
  return b;
}

// 16 bytes a lane from the buffer into LDS, the wave's 1024 bytes one after another from byte `lds` on.  An instruction
// of its own because the compiler waits for every such load before the next LDS read, whatever that reads; the kernels
// count them themselves.  It has no destination register; m0 needs one instruction between its write and its use.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 among the clobbers
__device__ __forceinline__ void load_lds(u32x4_t buffer, uint32_t lds, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(buffer)
               : "m0");
}
#pragma clang diagnostic pop

}  // namespace iso
