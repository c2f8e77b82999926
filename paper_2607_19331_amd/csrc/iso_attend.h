// What the attention kernels share: their arguments, the rows and keys of a sequence, and the row-by-row forms.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "iso.h"
#include "iso_device.h"
#include "iso_grad_device.h"
#include "iso_grad_plan.h"

namespace iso {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// A row's running maximum is only followed where it has grown by more than this (in powers of two): sums stay below
// 2^8 times their terms, and most tiles scale nothing.
constexpr float kSlack = 8.0f;

struct AttnArgs {
  const void *q, *k, *v;
  int64_t ld_q, ld_k, ld_v;           // row strides, elements
  const int32_t *start_q, *start_k;
  int64_t tokens_q, tokens_k;
  int32_t sequences, heads, heads_kv, group, dim;
  int32_t causal;
  int64_t window;
  float scale, scale2;                // scale, and scale log2(e)
  void* out;
  int64_t ld_out;
  float* lse;
  const void* dout;
  int64_t ld_dout;
  void *dq, *dk, *dv;
  int64_t ld_dq, ld_dk, ld_dv;
  float* stat;                        // for every row of a group's list, kv head by kv head: L log2(e), then D
  Pieces pieces, key_pieces;          // that a tile's keys are shared out to, and the rows of a tile of keys
  float *part, *key_part;             // their sums: pieces x tokens_q x heads (tokens_k x heads_kv x 2) x kPartLd
  uint32_t* status;
};

inline AttnArgs args_of(const iso_attn& a, uint8_t* ws) {
  AttnArgs A{};
  A.q = a.q, A.k = a.k, A.v = a.v, A.ld_q = a.ld_q, A.ld_k = a.ld_k, A.ld_v = a.ld_v;
  A.start_q = a.start_q, A.start_k = a.start_k, A.tokens_q = a.tokens_q, A.tokens_k = a.tokens_k;
  A.sequences = (int32_t)a.sequences, A.heads = a.heads, A.heads_kv = a.heads_kv, A.group = a.heads / a.heads_kv, A.dim = a.dim;
  A.causal = a.causal, A.window = std::min(a.window, (int64_t)1 << 30);   // past every distance, and sums with it hold
  A.scale = (float)a.scale, A.scale2 = (float)(a.scale * 1.4426950408889634);
  A.out = a.out, A.ld_out = a.ld_out, A.lse = a.lse, A.dout = a.dout, A.ld_dout = a.ld_dout;
  A.dq = a.dq, A.dk = a.dk, A.dv = a.dv, A.ld_dq = a.ld_dq, A.ld_dk = a.ld_dk, A.ld_dv = a.ld_dv;
  A.status = (uint32_t*)ws;
  return A;
}

// One sequence: first rows and lengths.  The queries of a kv head's group are taken as one list of `rows` = nq group rows,
// row r being query r / group of head r % group of the group: rows next to each other see (almost) the same keys.
struct Seq {
  int64_t q0, k0;
  int32_t nq, nk;
};

__device__ __forceinline__ bool seq_range(const int32_t* start, int64_t s, int64_t tokens, int64_t& first, int32_t& n) {
  const auto g = gmem(start) + s;
  const int32_t a = g[0], b = g[1];
  const bool ok = a >= 0 && a <= b && b <= tokens;
  first = ok ? a : 0;
  n = ok ? b - a : 0;
  return ok;
}

// Whether both offsets of a sequence are ranges; if not, it has no rows.
__device__ __forceinline__ bool seq_of(const AttnArgs& A, int64_t s, Seq& r) {
  const bool q = seq_range(A.start_q, s, A.tokens_q, r.q0, r.nq), k = seq_range(A.start_k, s, A.tokens_k, r.k0, r.nk);
  if (!q || !k) r = Seq{0, 0, 0, 0};
  return q && k;
}
__device__ __forceinline__ Seq seq_of(const AttnArgs& A, int64_t s) {
  Seq r;
  seq_of(A, s, r);
  return r;
}

// The last rows that sequences have taken: one that begins before them is left out too, so that no two share a row.  That takes offsets
// that do not ascend, and then some sequence's are no range.
struct Taken {
  int64_t q = 0, k = 0;
  __device__ __forceinline__ bool free(const Seq& s) const { return s.q0 >= q && s.k0 >= k; }
  __device__ __forceinline__ void add(const Seq& s) { q = max(q, s.q0 + s.nq), k = max(k, s.k0 + s.nk); }
};

// The keys that query i of the sequence sees: [lo, hi), and the queries that see key j.
__device__ __forceinline__ void keys_of(const AttnArgs& A, const Seq& s, int64_t i, int32_t& lo, int32_t& hi) {
  const int64_t p = i + s.nk - s.nq;
  int64_t a = 0, b = s.nk;
  if (A.causal) b = min(b, p + 1);
  if (A.window > 0) a = max(a, p - A.window + 1), b = min(b, p + A.window);
  b = max(b, (int64_t)0);
  a = min(a, b);
  lo = (int32_t)a, hi = (int32_t)b;
}

__device__ __forceinline__ void queries_of(const AttnArgs& A, const Seq& s, int64_t j, int32_t& lo, int32_t& hi) {
  const int64_t i = j - (s.nk - s.nq);   // the query at position j
  int64_t a = 0, b = s.nq;
  if (A.causal) a = max(a, i);
  if (A.window > 0) a = max(a, i - A.window + 1), b = min(b, i + A.window);
  b = max(b, (int64_t)0);
  a = min(a, b);
  lo = (int32_t)a, hi = (int32_t)b;
}

// Writes the status word of a call: whether all offsets are ranges of the rows, and ascend.  One workgroup.
__device__ __forceinline__ void check_starts(const AttnArgs& A) {
  bool bad = false;
  for (int64_t s = threadIdx.x; s < A.sequences; s += blockDim.x) {
    int64_t f;
    int32_t n;
    bad |= !seq_range(A.start_q, s, A.tokens_q, f, n);
    bad |= !seq_range(A.start_k, s, A.tokens_k, f, n);
  }
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0) *A.status = any ? kStatusIndex : 0u;
}

// ---- row by row ----------------------------------------------------------------------------------------------------
//
// One wave works out one row (or key) in binary32, from the keys (or rows) that it sees and from no others.  Scores have a
// lane a key, sums over keys a lane for every two of the (up to 128) dimensions.  A sum that is NaN in all dimensions stays so, whatever
// follows: where a whole step has gone to NaN, 64 keys do for a row (two sequences of 4096, 28 heads over 4 of 128, bf16: 2.6 ms for 67
// forward, 4.1 for 197 backward; 0.26 and 0.9 where all is finite).

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Dot product of dim elements (a multiple of 8) from a and b on.
template <int DT>
__device__ __forceinline__ float dot_row(const void* a, int64_t ia, const void* b, int64_t ib, int dim) {
  float s = 0.0f;
  for (int d = 0; d < dim; d += 8) {
    float x[8], y[8];
    load_elems<DT, 8>(a, ia + d, x);
    load_elems<DT, 8>(b, ib + d, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[j], y[j], s);
  }
  return s;
}

template <int DT>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  if constexpr (DT == ISO_BF16) return f32_from_bits((uint32_t)gmem((const uint16_t*)p)[i] << 16);
  else return f32_from_bits(gmem((const uint32_t*)p)[i]);
}
template <int DT>
__device__ __forceinline__ void store_one(void* p, int64_t i, float v) {
  if constexpr (DT == ISO_BF16) gmem((uint16_t*)p)[i] = (uint16_t)pack_bf16(v, 0.0f);
  else gmem((uint32_t*)p)[i] = bits_from_f32(v);
}

// Elements of the two dimensions of a lane.
template <int DT>
struct Two {
  float v[2] = {0.0f, 0.0f};
  __device__ __forceinline__ void add(float w, const void* p, int64_t at, int lane, int dim) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (lane + 64 * h < dim) v[h] = fmaf(w, load_one<DT>(p, at + lane + 64 * h), v[h]);
  }
  __device__ __forceinline__ bool gone(int lane, int dim) const {   // all that the lane has is NaN
    return (lane >= dim || v[0] != v[0]) && (lane + 64 >= dim || v[1] != v[1]);
  }
  __device__ __forceinline__ void store(void* p, int64_t at, int lane, int dim, float scale) const {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (lane + 64 * h < dim) store_one<DT>(p, at + lane + 64 * h, v[h] * scale);
  }
};

// O and L of row r of kv head `head`.
template <int DT>
__device__ __forceinline__ void attend_row(const AttnArgs& A, const Seq& s, int head, int64_t r, int lane) {
  const int64_t i = r / A.group;
  const int h = head * A.group + (int)(r - i * A.group);
  int32_t lo, hi;
  keys_of(A, s, i, lo, hi);
  const int64_t q = (s.q0 + i) * A.ld_q + (int64_t)h * A.dim;
  Two<DT> o;
  float m = -INFINITY, l = 0.0f;
  for (int32_t j0 = lo; j0 < hi; j0 += 64) {
    const bool on = j0 + lane < hi;
    const int64_t j = s.k0 + (on ? j0 + lane : lo);
    const float x = dot_row<DT>(A.q, q, A.k, j * A.ld_k + (int64_t)head * A.dim, A.dim) * A.scale;
    const float top = fmaxf(m, wave_max(on ? x : -INFINITY));
    const float ref = top == -INFINITY ? 0.0f : top;
    const float f = exp2f((m - ref) * kLog2e), p = on ? exp2f((x - ref) * kLog2e) : 0.0f;
    m = top;
    l = l * f + wave_sum(p);
    o.v[0] *= f, o.v[1] *= f;
    const int n = min(64, hi - j0);
    for (int c = 0; c < n; ++c)
      o.add(__shfl(p, c), A.v, (s.k0 + j0 + c) * A.ld_v + (int64_t)head * A.dim, lane, A.dim);
    if (__all(l != l && o.gone(lane, A.dim))) break;
  }
  o.store(A.out, (s.q0 + i) * A.ld_out + (int64_t)h * A.dim, lane, A.dim, hi > lo ? 1.0f / l : 0.0f);
  if (lane == 0) gmem(A.lse)[(s.q0 + i) * A.heads + h] = hi > lo ? m + logf(l) : -INFINITY;
}

// P and dP - D of (row, key), the row given by its q, dout and L, D.
template <int DT>
__device__ __forceinline__ void pair(const AttnArgs& A, int64_t q, int64_t g, int64_t k, int64_t v, float lse, float delta, float& p,
                                     float& ds) {
  p = exp2f((dot_row<DT>(A.q, q, A.k, k, A.dim) * A.scale - lse) * kLog2e);
  ds = p * (dot_row<DT>(A.dout, g, A.v, v, A.dim) - delta);
}

// Where the list of a kv head's rows starts in stat, and D of row r of it.
__device__ __forceinline__ int64_t list_of(const AttnArgs& A, const Seq& s, int head) {
  return ((int64_t)head * A.tokens_q + s.q0) * A.group;
}
__device__ __forceinline__ float delta_of(const AttnArgs& A, const Seq& s, int head, int64_t r) {
  return gmem(A.stat)[A.tokens_q * A.heads + list_of(A, s, head) + r];
}

// dq of row r.
template <int DT>
__device__ __forceinline__ void dq_row(const AttnArgs& A, const Seq& s, int head, int64_t r, int lane) {
  const int64_t i = r / A.group, col = (int64_t)head * A.dim;
  const int h = head * A.group + (int)(r - i * A.group);
  int32_t lo, hi;
  keys_of(A, s, i, lo, hi);
  const int64_t q = (s.q0 + i) * A.ld_q + (int64_t)h * A.dim, g = (s.q0 + i) * A.ld_dout + (int64_t)h * A.dim;
  const float lse = gmem(A.lse)[(s.q0 + i) * A.heads + h], delta = delta_of(A, s, head, r);
  Two<DT> sum;
  for (int32_t j0 = lo; j0 < hi; j0 += 64) {
    const int64_t j = s.k0 + min(j0 + lane, hi - 1);
    float p, ds;
    pair<DT>(A, q, g, j * A.ld_k + col, j * A.ld_v + col, lse, delta, p, ds);
    const int n = min(64, hi - j0);
    for (int c = 0; c < n; ++c) sum.add(__shfl(ds, c), A.k, (s.k0 + j0 + c) * A.ld_k + col, lane, A.dim);
    if (__all(sum.gone(lane, A.dim))) break;
  }
  sum.store(A.dq, (s.q0 + i) * A.ld_dq + (int64_t)h * A.dim, lane, A.dim, A.scale);
}

// dk and dv of key j.
template <int DT>
__device__ __forceinline__ void dkv_row(const AttnArgs& A, const Seq& s, int head, int32_t j, int lane) {
  int32_t lo, hi;
  queries_of(A, s, j, lo, hi);
  const int64_t col = (int64_t)head * A.dim, k = (s.k0 + j) * A.ld_k + col, v = (s.k0 + j) * A.ld_v + col;
  const int64_t first = (int64_t)lo * A.group, last = (int64_t)hi * A.group;
  Two<DT> dk, dv;
  for (int64_t r0 = first; r0 < last; r0 += 64) {
    const int64_t r = min(r0 + lane, last - 1), i = s.q0 + r / A.group;
    const int h = head * A.group + (int)(r % A.group);
    const int64_t q = i * A.ld_q + (int64_t)h * A.dim, g = i * A.ld_dout + (int64_t)h * A.dim;
    float p, ds;
    pair<DT>(A, q, g, k, v, gmem(A.lse)[i * A.heads + h], delta_of(A, s, head, r), p, ds);
    const int n = (int)min((int64_t)64, last - r0);
    for (int c = 0; c < n; ++c) {
      dk.add(__shfl(ds, c), A.q, __shfl(q, c), lane, A.dim);
      dv.add(__shfl(p, c), A.dout, __shfl(g, c), lane, A.dim);
    }
    if (__all(dk.gone(lane, A.dim) && dv.gone(lane, A.dim))) break;
  }
  dk.store(A.dk, (s.k0 + j) * A.ld_dk + col, lane, A.dim, A.scale);
  dv.store(A.dv, (s.k0 + j) * A.ld_dv + col, lane, A.dim, 1.0f);
}

}  // namespace iso
