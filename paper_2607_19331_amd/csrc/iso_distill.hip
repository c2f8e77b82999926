// Distillation from a teacher's top entries: with t = softmax(y / T) over a token's list and L = logsumexp(z / T) over the
// vocabulary, loss = w T^2 sum t (log t - z_id / T + L) and grad_v = w T (exp(z_v / T - L) - sum of t at id v).
//
// Bound by memory: 2 (or 4) bytes of a logit read, as many written for a gradient, against one exponential each.  The list
// (up to 256 entries, one a thread) is a few microseconds of latency a row, hidden under other rows.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "iso.h"
#include "iso_device.h"
#include "iso_grad.h"
#include "iso_grad_device.h"

namespace iso {

namespace {

constexpr float kLog2e = 1.44269504088896341f;

struct DistillArgs {
  const void* z;
  const void* ids;
  const float *y, *w;
  float *loss, *lse;
  void* grad;
  int64_t tokens, vocab, ld, ld_grad, pad_id;
  int32_t top, id_type, pieces;   // pieces: workgroups a row
  float inv_t;                    // 1 / T
  double t;
  float* part;                    // maximum and sum of a piece (scaled by 1 / T), tokens x pieces
  uint32_t* status;
};

// Maximum of x and sum of 2^((x - maximum) log2 e), for values and for pairs of these.
struct Lse {
  float m = -INFINITY, s = 0.0f;
};
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ Lse join(Lse a, Lse b) {
  const float m = fmaxf(a.m, b.m), ref = m == -INFINITY ? 0.0f : m;
  // a NaN sum stays one; so does infinity, whose own term is exp(inf - inf)
  return Lse{m, a.s * exp_of(a.m - ref) + b.s * exp_of(b.m - ref)};
}

template <int N>
__device__ __forceinline__ Lse block_lse(Lse v, float (*lds)[2]) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = join(v, Lse{__shfl_xor(v.m, d), __shfl_xor(v.s, d)});
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6][0] = v.m, lds[threadIdx.x >> 6][1] = v.s;
  __syncthreads();
  v = Lse{lds[0][0], lds[0][1]};
#pragma unroll
  for (int i = 1; i < N / 64; ++i) v = join(v, Lse{lds[i][0], lds[i][1]});
  return v;
}

__device__ __forceinline__ int64_t id_at(const DistillArgs& A, int64_t i) {
  return A.id_type == ISO_I64 ? gmem((const int64_t*)A.ids)[i] : (int64_t)gmem((const int32_t*)A.ids)[i];
}
__device__ __forceinline__ bool outside(const DistillArgs& A, int64_t id) {
  return id != A.pad_id && (id < 0 || id >= A.vocab);
}

// Lists of up to this many entries in all are looked at by one workgroup, which then writes the status word by itself; where
// there are more, a launch before clears it and every row looks at its own.
constexpr int64_t kFewEntries = 8192;

__device__ __forceinline__ void check_ids(const DistillArgs& A) {
  bool bad = false;
  for (int64_t i = threadIdx.x; i < A.tokens * A.top; i += blockDim.x) bad |= outside(A, id_at(A, i));
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0) *A.status = any ? kStatusIndex : 0u;
}

__global__ void k_distill_clear(uint32_t* status) { *status = 0; }

// A token's list: thread e (of at least 256) has entry e.
struct Entry {
  int32_t id = -1;     // -1: none
  float t = 0.0f;      // its share; that of all entries with the same id where `sum` was called
  float log_t = 0.0f;
  bool first = false;  // the first of the entries with its id
};

struct ListSpace {
  int32_t id[ISO_DISTILL_MAX_TOP];
  float t[ISO_DISTILL_MAX_TOP];
  float red[16][2];
};

// Every thread of the workgroup calls; `any` is whether the token has entries.
template <int N>
__device__ __forceinline__ Entry list_of(const DistillArgs& A, int64_t row, ListSpace& S, bool& any) {
  const int e = threadIdx.x;
  Entry r;
  float y = -INFINITY;
  if (e < A.top) {
    const int64_t id = id_at(A, row * A.top + e);
    const float v = gmem(A.y)[row * A.top + e];
    if (outside(A, id)) {
      if (A.tokens * A.top > kFewEntries) atomicOr(A.status, kStatusIndex);
    } else if (id != A.pad_id && v != -INFINITY) {
      r.id = (int32_t)id;
      y = v * A.inv_t;
    }
  }
  // the first four waves hold the entries
  Lse l{y, r.id >= 0 ? 1.0f : 0.0f};
  if (r.id >= 0 && !(fabsf(y) < INFINITY)) l.s = NAN;   // an infinite or NaN logit of the teacher
  l = block_lse<256>(l, S.red);
  any = l.s != 0.0f;
  if (r.id >= 0) {
    r.log_t = (y - l.m) - logf(l.s);
    r.t = exp_of(r.log_t);
  }
  if (e < ISO_DISTILL_MAX_TOP) S.id[e] = r.id, S.t[e] = r.t;
  __syncthreads();
  return r;
}

// Entries with the same id as one: their first has the sum.
__device__ __forceinline__ void merge(const DistillArgs& A, const ListSpace& S, Entry& r) {
  if (r.id < 0) return;
  r.first = true;
  float t = 0.0f;
  for (int i = 0; i < A.top; ++i)
    if (S.id[i] == r.id) {
      if (i < (int)threadIdx.x) r.first = false;
      t += S.t[i];
    }
  r.t = t;
}

// The row's loss from its entries, in binary64: the sum of t (log t - z + L) cancels where the student has learnt.
template <int DT>
__device__ __forceinline__ void store_loss(const DistillArgs& A, int64_t row, const Entry& r, float z, double lse, bool any, double* lds) {
  double v = 0.0;
  if (r.id >= 0 && r.t != 0.0f) v = (double)r.t * ((double)r.log_t - (double)z / A.t + lse);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0 && threadIdx.x < 256) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    const float w = A.w != nullptr ? gmem(A.w)[row] : 1.0f;
    v = lds[0] + lds[1] + lds[2] + lds[3];
    gmem(A.loss)[row] = any && w != 0.0f ? (float)(w * A.t * A.t * v) : 0.0f;
    gmem(A.lse)[row] = (float)lse;
  }
}

template <int DT>
__device__ __forceinline__ float load_z(const DistillArgs& A, int64_t i) {
  if constexpr (DT == ISO_BF16) return f32_from_bits((uint32_t)gmem((const uint16_t*)A.z)[i] << 16);
  else return f32_from_bits(gmem((const uint32_t*)A.z)[i]);
}

// Maximum and sum over columns [lo, hi) of a row, a workgroup of 256.
template <int DT>
__device__ __forceinline__ Lse row_lse(const DistillArgs& A, int64_t row, int64_t lo, int64_t hi, float (*lds)[2]) {
  constexpr int V = kVec<DT>, U = 4;
  const int64_t base = row * A.ld;
  Lse l;
  auto add = [&](const float* v, int n) {
    float top = l.m;
#pragma unroll
    for (int j = 0; j < U * V; ++j)
      if (j < n) top = fmaxf(top, v[j] * A.inv_t);
    const float ref = top == -INFINITY ? 0.0f : top;
    float s = l.s * exp_of(l.m - ref);
#pragma unroll
    for (int j = 0; j < U * V; ++j)
      if (j < n) s += exp_of(fmaf(v[j], A.inv_t, -ref));
    l = Lse{top, s};
  };
  int64_t c = lo + (int64_t)threadIdx.x * V;
  for (; c + (U - 1) * 256 * V + V <= hi; c += U * 256 * V) {
    u32x4_t w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = load_raw<DT>(A.z, base + c + u * 256 * V);
    float v[U * V];
#pragma unroll
    for (int u = 0; u < U; ++u) unpack_raw<DT>(w[u], v + u * V);
    add(v, U * V);
  }
  for (; c < hi; c += 256 * V) {
    float v[U * V];
    unpack_raw<DT>(load_raw<DT>(A.z, base + c, hi - c), v);
    add(v, (int)min((int64_t)V, hi - c));
  }
  return block_lse<256>(l, lds);
}

// The gradient over columns [lo, hi) of a row, a workgroup of N.  Entries' own values are written after the others'.
template <int DT, int N>
__device__ __forceinline__ void row_grad(const DistillArgs& A, int64_t row, int64_t lo, int64_t hi, const Entry& r, float z, float lse,
                                         bool any) {
  constexpr int V = kVec<DT>;
  const int64_t from = row * A.ld, to = row * A.ld_grad;
  const float w = A.w != nullptr ? gmem(A.w)[row] : 1.0f, f = w * (float)A.t;
  const bool zero = !any || w == 0.0f;
  // the gradient may lie over the logits: entries have theirs before anything is written
  asm volatile("s_waitcnt vmcnt(0)" ::"v"(z) : "memory");
  __syncthreads();
  for (int64_t c = lo + (int64_t)threadIdx.x * V; c < hi; c += N * V) {
    float v[V];
    load_elems<DT, V>(A.z, from + c, v, hi - c);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = zero ? 0.0f : f * exp_of(fmaf(v[j], A.inv_t, -lse));
    store_elems<DT, V>(A.grad, to + c, v, hi - c);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (!zero && r.first && r.id >= lo && r.id < hi) {
    const float v = f * (exp_of(fmaf(z, A.inv_t, -lse)) - r.t);
    if constexpr (DT == ISO_BF16) gmem((uint16_t*)A.grad)[to + r.id] = (uint16_t)pack_bf16(v, 0.0f);
    else gmem((uint32_t*)A.grad)[to + r.id] = bits_from_f32(v);
  }
}

// Loss (and gradient) of a row, one workgroup: two walks over the row where both are asked for.
template <int DT>
__global__ void __launch_bounds__(256) k_distill_row(DistillArgs A) {
  __shared__ ListSpace S;
  __shared__ double sums[4];
  const int64_t row = blockIdx.x;
  if (row == 0 && A.tokens * A.top <= kFewEntries) check_ids(A);
  const Lse l = row_lse<DT>(A, row, 0, A.vocab, S.red);
  __syncthreads();
  bool any;
  Entry r = list_of<256>(A, row, S, any);
  const float z = r.id >= 0 ? load_z<DT>(A, row * A.ld + r.id) : 0.0f;
  const double lse = (double)l.m + log((double)l.s);
  store_loss<DT>(A, row, r, z, lse, any, sums);
  if (A.grad == nullptr) return;
  merge(A, S, r);
  row_grad<DT, 256>(A, row, 0, A.vocab, r, z, (float)lse, any);
}

// A piece of a row: its share of the sum, and from these the loss.
template <int DT>
__global__ void __launch_bounds__(256) k_distill_part(DistillArgs A, int64_t each) {
  __shared__ ListSpace S;
  if (blockIdx.x == 0 && A.tokens * A.top <= kFewEntries) check_ids(A);
  const int64_t row = blockIdx.x / A.pieces, lo = (blockIdx.x - row * A.pieces) * each;
  const Lse l = row_lse<DT>(A, row, lo, min(lo + each, A.vocab), S.red);
  if (threadIdx.x == 0) gmem(A.part)[2 * blockIdx.x] = l.m, gmem(A.part)[2 * blockIdx.x + 1] = l.s;
}

template <int DT>
__global__ void __launch_bounds__(256) k_distill_join(DistillArgs A) {
  __shared__ ListSpace S;
  __shared__ double sums[4];
  const int64_t row = blockIdx.x;
  Lse l;
  for (int i = threadIdx.x; i < A.pieces; i += 256) {
    const auto p = gmem((const float*)A.part) + 2 * (row * A.pieces + i);
    l = join(l, Lse{p[0], p[1]});
  }
  l = block_lse<256>(l, S.red);
  __syncthreads();
  bool any;
  const Entry r = list_of<256>(A, row, S, any);
  const float z = r.id >= 0 ? load_z<DT>(A, row * A.ld + r.id) : 0.0f;
  store_loss<DT>(A, row, r, z, (double)l.m + log((double)l.s), any, sums);
}

// The gradient of a piece of a row from the row's L.
template <int DT>
__global__ void __launch_bounds__(256) k_distill_grad(DistillArgs A, int64_t each) {
  __shared__ ListSpace S;
  const int64_t row = blockIdx.x / A.pieces, lo = (blockIdx.x - row * A.pieces) * each;
  bool any;
  Entry r = list_of<256>(A, row, S, any);
  const float z = r.id >= 0 ? load_z<DT>(A, row * A.ld + r.id) : 0.0f;
  merge(A, S, r);
  row_grad<DT, 256>(A, row, lo, min(lo + each, A.vocab), r, z, gmem(A.lse)[row], any);
}

DistillArgs args_of(const iso_distill& d, uint8_t* ws) {
  DistillArgs A{};
  A.z = d.logits, A.ids = d.ids, A.y = d.teacher, A.w = d.weight, A.loss = d.loss, A.lse = d.lse, A.grad = d.grad;
  A.tokens = d.tokens, A.vocab = d.vocab, A.ld = d.ld, A.ld_grad = d.ld_grad, A.pad_id = d.pad_id;
  A.top = d.top, A.id_type = d.id_type;
  A.inv_t = (float)(1.0 / d.temperature), A.t = d.temperature;
  A.status = (uint32_t*)ws;
  A.part = (float*)(ws + kStatusBytes);
  return A;
}

template <int DT>
void loss(const DistillArgs& A, hipStream_t s) {
  k_distill_row<DT><<<(unsigned)A.tokens, 256, 0, s>>>(A);
}

template <int DT>
void gradient(DistillArgs A, hipStream_t s) {
  A.pieces = 1;
  k_distill_grad<DT><<<(unsigned)A.tokens, 256, 0, s>>>(A, A.vocab);
}

}  // namespace

hipError_t run_distill_loss(const iso_distill& d, int dt, uint8_t* ws, hipStream_t s) {
  const DistillArgs A = args_of(d, ws);
  if (A.tokens == 0 || A.tokens * A.top > kFewEntries) k_distill_clear<<<1, 1, 0, s>>>(A.status);
  if (A.tokens > 0) dt == ISO_BF16 ? loss<ISO_BF16>(A, s) : loss<ISO_F32>(A, s);
  return hipGetLastError();
}

hipError_t run_distill_grad(const iso_distill& d, int dt, uint8_t* ws, hipStream_t s) {
  const DistillArgs A = args_of(d, ws);
  if (A.tokens == 0 || A.tokens * A.top > kFewEntries) k_distill_clear<<<1, 1, 0, s>>>(A.status);
  if (A.tokens > 0) dt == ISO_BF16 ? gradient<ISO_BF16>(A, s) : gradient<ISO_F32>(A, s);
  return hipGetLastError();
}

}  // namespace iso
