// Workspace layout of all calls.  Plain C++ (no HIP), so that host-side planning can be compiled by itself.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace iso {

// [0, 256)            status block (u32 flags)
// [256, ...)          per-call tables and scratch, each region 256-byte aligned
constexpr size_t kStatusBytes = 256;
constexpr uint32_t kStatusNonFinite = 1u;
constexpr uint32_t kStatusInternal = 2u;   // a kernel found counts that cannot occur; results invalid
constexpr uint32_t kStatusIndex = 4u;      // a token id outside the vocabulary

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace iso
