// Distillation from a teacher's top entries: with t = softmax(y / T) over a token's list and L = logsumexp(z / T) over the
// vocabulary, loss = w T^2 sum t (log t - z_id / T + L) and grad_v = w T (exp(z_v / T - L) - sum of t at id v).
//
// Bound by memory: 2 (or 4) bytes of a logit read, as many written for a gradient, against one exponential each (two for both in
// one call).  The list (up to 256 entries, one a thread) is a few microseconds of latency a row, hidden under other rows.
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

constexpr float kLn2 = 0.693147180559945309f;

struct DistillArgs {
  const void* z;
  const void* ids;
  const float *y, *w;
  float *loss, *lse;
  void* grad;
  int64_t tokens, vocab, ld, ld_grad, pad_id;
  int32_t top, id_type, pieces;   // pieces: workgroups a row
  float c;                        // log2(e) / T
  double log2e_t;                 // the same, not rounded to binary32
  double t, tc, inv_tc;           // T, T c and its reciprocal
  float* part;                    // reference and sum of a piece, tokens x pieces
  uint32_t* status;
};

// The sum of 2^(z c - m) over some logits, m their largest z c rounded: as m is what is subtracted, its rounding is no error.  It is in the
// exponent, though, and reaches 2^6 at 2^31; so m is no less than -2^31 (logits behind that, a mask's, have no part in a sum, and a
// row of nothing else an L of minus infinity), and L is NaN where it is more than 2^31.
constexpr float kFar = 2147483648.0f;
struct Lse {
  float m = -kFar, s = 0.0f;
};
// A NaN sum stays one; so does infinity, whose own term is exp(inf - inf).
__device__ __forceinline__ Lse join(Lse a, Lse b) {
  const float m = fmaxf(a.m, b.m);
  return Lse{m, a.s * __builtin_amdgcn_exp2f(a.m - m) + b.s * __builtin_amdgcn_exp2f(b.m - m)};
}
// Of a list, m being its largest logit as it is (minus infinity: none): differences are taken before they are scaled.
__device__ __forceinline__ Lse join_list(Lse a, Lse b, float c) {
  const float m = fmaxf(a.m, b.m), ref = m == -INFINITY ? 0.0f : m;
  return Lse{m, a.s * __builtin_amdgcn_exp2f((a.m - ref) * c) + b.s * __builtin_amdgcn_exp2f((b.m - ref) * c)};
}

// Of a workgroup of N: every wave puts its own into LDS, and after a barrier all of them are joined.
template <class J>
__device__ __forceinline__ void put_lse(Lse v, float (*lds)[2], J join) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = join(v, Lse{__shfl_xor(v.m, d), __shfl_xor(v.s, d)});
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6][0] = v.m, lds[threadIdx.x >> 6][1] = v.s;
}
template <int N, class J>
__device__ __forceinline__ Lse get_lse(const float (*lds)[2], J join) {
  const int i = threadIdx.x & (N / 64 - 1);   // each N / 64 lanes for themselves, all alike
  Lse v{lds[i][0], lds[i][1]};
#pragma unroll
  for (int d = N / 128; d > 0; d >>= 1) v = join(v, Lse{__shfl_xor(v.m, d), __shfl_xor(v.s, d)});
  return v;
}
template <int N, class J>
__device__ __forceinline__ Lse block_lse(Lse v, float (*lds)[2], J join) {
  put_lse(v, lds, join);
  __syncthreads();
  return get_lse<N>(lds, join);
}
struct Join {
  __device__ __forceinline__ Lse operator()(Lse a, Lse b) const { return join(a, b); }
};
struct JoinList {
  float c;
  __device__ __forceinline__ Lse operator()(Lse a, Lse b) const { return join_list(a, b, c); }
};

// Adds values to a sum, which is scaled once for all of them.  They are added up by themselves first: where an entry's logit is in the
// sum, one by one the others would be lost in its rounding.
template <int N>
__device__ __forceinline__ void add_to(Lse& l, const float* v, float c) {
  float top = v[0];
#pragma unroll
  for (int j = 1; j < N; ++j) top = fmaxf(top, v[j]);
  top = fmaxf(l.m, top * c);
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < N; ++j) s += __builtin_amdgcn_exp2f(fmaf(v[j], c, -top));
  l = Lse{top, fmaf(l.s, __builtin_amdgcn_exp2f(l.m - top), s)};
}

// Of one entry of a teacher's list (or none): the lowest and the largest finite logits have their shares, an infinite or NaN logit makes
// all of the list's shares NaN.
__device__ __forceinline__ Lse one(bool has, float y) { return has ? Lse{y, fabsf(y) < INFINITY ? 1.0f : NAN} : Lse{-INFINITY, 0.0f}; }
// Its exponent of 2 (shares from 2^-1000 down are none), of a list with m; its share and the share's logarithm, l having the reciprocal of
// the sum.  What the exponent's rounding takes, up to 5 2^-24 of a share of 10^-4, goes into a factor.
__device__ __forceinline__ double below(const DistillArgs& A, float y, Lse l) { return fmax(((double)y - (double)l.m) * A.log2e_t, -1000.0); }
__device__ __forceinline__ float share_of(const DistillArgs& A, float y, Lse l) {
  const double x = below(A, y, l);
  return __builtin_amdgcn_exp2f((float)x) * fmaf((float)(x - (float)x), kLn2, 1.0f) * l.s;
}
__device__ __forceinline__ float log_share_of(const DistillArgs& A, float y, Lse l) { return (float)below(A, y, l) * kLn2 + logf(l.s); }

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
  float t = 0.0f;      // its share; that of all entries with the same id after merge()
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
      y = v;
    }
  }
  // the first four waves hold the entries
  Lse l = block_lse<256>(one(r.id >= 0, y), S.red, JoinList{A.c});
  any = l.s != 0.0f;
  l.s = 1.0f / l.s;
  if (r.id >= 0) r.log_t = log_share_of(A, y, l), r.t = share_of(A, y, l);
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

__device__ __forceinline__ float weight_of(const DistillArgs& A, int64_t row) { return A.w != nullptr ? gmem(A.w)[row] : 1.0f; }

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
    const float w = weight_of(A, row);
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

// One piece of 16 bytes at the end of a row: minus infinity behind it, which has no part in a maximum or a sum.
template <int DT>
__device__ __forceinline__ u32x4_t load_end(const void* p, int64_t i, int64_t left) {
  constexpr int V = kVec<DT>;
  constexpr uint32_t none = DT == ISO_BF16 ? 0xFF80FF80u : 0xFF800000u;
  u32x4_t w = {none, none, none, none};
  if (left >= V) return load_raw<DT>(p, i);
  if (left <= 0) return w;
  const u32x4_t x = load_raw<DT>(p, i, left);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t m = DT == ISO_BF16 ? 0xFFFFu << (16 * (j & 1)) : 0xFFFFFFFFu;
    if (j < left) w[j * 4 / V] = (w[j * 4 / V] & ~m) | (x[j * 4 / V] & m);
  }
  return w;
}

// Maximum and sum over columns [lo, hi) of a row, a workgroup of N.
template <int DT, int N>
__device__ __forceinline__ Lse row_lse(const DistillArgs& A, int64_t row, int64_t lo, int64_t hi, float (*lds)[2]) {
  constexpr int V = kVec<DT>, U = 4, kStride = N * V;
  const int64_t base = row * A.ld;
  Lse l;
  int64_t c = lo + (int64_t)threadIdx.x * V;
  for (; c + (U - 1) * kStride + V <= hi; c += U * kStride) {
    u32x4_t w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = load_raw<DT>(A.z, base + c + u * kStride);
    float v[U * V];
#pragma unroll
    for (int u = 0; u < U; ++u) unpack_raw<DT>(w[u], v + u * V);
    add_to<U * V>(l, v, A.c);
  }
  for (; c < hi; c += kStride) {
    float v[V];
    unpack_raw<DT>(load_end<DT>(A.z, base + c, hi - c), v);
    add_to<V>(l, v, A.c);
  }
  return block_lse<N>(l, lds, Join{});
}

// L of a row, in binary64: the loss takes differences of it.  m / c is a logit but for m's rounding, which s holds; the logarithm of s
// is that of a value from 1/2 to 1, which binary32 has to 2^-24, and a multiple of log 2.
__device__ __forceinline__ double lse_of(const DistillArgs& A, Lse l) {
  if (!(l.m < kFar)) return NAN;
  const float low = logf(__builtin_amdgcn_frexp_mantf(l.s));
  return fma((double)l.m, A.inv_tc, fma((double)__builtin_amdgcn_frexp_expf(l.s), 0.6931471805599453, (double)low));
}

// A row's factor w T, whether its gradient is zero, and its L: a probability is less 2^(z c - lse2), lse2 being T c L
// rounded and less the power of two of what that took (2^-21 for logits of 10, 1/2 for 10^7).
struct Factor {
  float f, less, lse2;
  bool zero;
  __device__ __forceinline__ Factor(const DistillArgs& A, float w, double lse, bool any) {
    f = w * (float)A.t;
    zero = !any || w == 0.0f;
    const double exact = lse * A.tc;
    lse2 = (float)exact;
    const double took = lse2 - exact;
    less = !(fabsf(lse2) < INFINITY) ? 1.0f : fabs(took) < 0x1p-12 ? (float)(1.0 + took * 0.6931471805599453) : exp2f((float)took);
  }
  __device__ __forceinline__ float probability(const DistillArgs& A, float z) const {
    return less * __builtin_amdgcn_exp2f(fmaf(z, A.c, -lse2));
  }
};
// The gradients of 16 bytes of logits.
template <int DT>
__device__ __forceinline__ void grads_of(const DistillArgs& A, const Factor& F, u32x4_t w, float* v) {
  unpack_raw<DT>(w, v);
  const float f = F.f * F.less;
#pragma unroll
  for (int j = 0; j < kVec<DT>; ++j) v[j] = f * __builtin_amdgcn_exp2f(fmaf(v[j], A.c, -F.lse2));
}

// Entries' own gradients, written after all of the row's: columns [lo, hi).
template <int DT>
__device__ __forceinline__ void put_entry(const DistillArgs& A, int64_t row, int64_t lo, int64_t hi, const Factor& F, const Entry& r, float z) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (F.zero || !r.first || r.id < lo || r.id >= hi) return;
  const float v = F.f * (F.probability(A, z) - r.t);
  const int64_t to = row * A.ld_grad + r.id;
  if constexpr (DT == ISO_BF16) gmem((uint16_t*)A.grad)[to] = (uint16_t)pack_bf16(v, 0.0f);
  else gmem((uint32_t*)A.grad)[to] = bits_from_f32(v);
}

// The gradient of 16 bytes a lane from column c on, U of them 256 lanes apart, of a row of A.vocab columns.
template <int DT, int U, bool STREAM>
__device__ __forceinline__ void put_grads(const DistillArgs& A, int64_t row, int64_t c, const Factor& F, const u32x4_t* w) {
  constexpr int V = kVec<DT>, kStride = 256 * V;
  const int64_t to = row * A.ld_grad;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = c + u * kStride;
    if (at >= A.vocab) continue;
    float v[V] = {};
    if (!F.zero) grads_of<DT>(A, F, w[u], v);
    store_elems<DT, V, STREAM>(A.grad, to + at, v, A.vocab - at);
  }
}

// Every entry of the row has its logit before anything is written: the gradient may lie over the logits.
__device__ __forceinline__ void before_writes(float z) {
  asm volatile("s_waitcnt vmcnt(0)" ::"v"(z) : "memory");
  __syncthreads();
}

// Loss of a row, one workgroup: the row's maximum and sum, then its list.  Bound by memory where there are many (4096 x 152064 bf16:
// 217 us, 5.7 TB/s), else by its own walk, four loads a lane under way.
template <int DT, int N>
__global__ void __launch_bounds__(N) k_distill_row(DistillArgs A) {
  __shared__ ListSpace S;
  __shared__ double sums[4];
  const int64_t row = blockIdx.x;
  if (row == 0 && A.tokens * A.top <= kFewEntries) check_ids(A);
  const Lse l = row_lse<DT, N>(A, row, 0, A.vocab, S.red);
  __syncthreads();
  bool any;
  const Entry r = list_of<256>(A, row, S, any);
  const float z = r.id >= 0 ? load_z<DT>(A, row * A.ld + r.id) : 0.0f;
  store_loss<DT>(A, row, r, z, lse_of(A, l), any, sums);
}

// A list before it is looked at: thread e has entry e.
struct RawEntry {
  int64_t id = 0;
  float y = 0.0f;
  __device__ __forceinline__ void load(const DistillArgs& A, int64_t row) {
    if ((int)threadIdx.x >= A.top) return;
    id = id_at(A, row * A.top + threadIdx.x);
    y = gmem(A.y)[row * A.top + threadIdx.x];
  }
};

template <int N>
struct HeldSpace {
  ListSpace list;
  float red[16][2], value[ISO_DISTILL_MAX_TOP];
  double sums[4];
  int16_t next[ISO_DISTILL_MAX_TOP];
  u32x4_t rest;      // what is left of a row behind its pieces
  int32_t head[N];   // the first of the entries that lie in a lane's columns; -1: none
};

// Loss and gradient of a row that a workgroup of N holds in registers, PER pieces of 16 bytes a lane: read once, written once
// (4096 x 152064 bf16: 486 us, 5.1 TB/s, the rate of a plain copy).
// All of a row is under way at once; what a CU does between its loads and its stores, other CUs' loads and stores fill.  Entries
// change the pieces they lie in before these are stored (a lane has a list of its own): written after them they would have to
// wait for the stores.  Workgroups that walk over rows and load a piece of the next row where one of this is stored were tried:
// the registers for it cost more than it gave (4096 x 152064 bf16: 577 us).
template <int DT, int N, int PER, bool STREAM>
__global__ void __launch_bounds__(N) k_distill_held(DistillArgs A) {
  constexpr int V = kVec<DT>;
  using bits = typename Fmt<DT>::bits_t;
  __shared__ HeldSpace<N> S;
  const int32_t vocab = (int32_t)A.vocab;
  const int e = threadIdx.x;
  uint32_t mine = threadIdx.x * V;
  const int64_t row = blockIdx.x;
  if (row == 0 && A.tokens * A.top <= kFewEntries) check_ids(A);
  // Every lane makes the same loads: the compiler counts them, and the row is summed as it comes in.  What lies behind the row's end is
  // taken from its last 16 bytes and replaced below, by minus infinity or by what is left of a piece.
  const bits* const z_row = (const bits*)A.z + row * A.ld;
  u32x4_t w[PER];
  const int32_t whole = vocab % V != 0 ? vocab / V * V : -1;
  if (whole >= 0 && e == whole / V % N) S.rest = load_end<DT>(z_row, whole, vocab - whole);   // and reads it
  RawEntry raw;
  raw.load(A, row);
  const uint32_t last = (uint32_t)(vocab - V) * sizeof(bits);
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const uint32_t at = min((uint32_t)(p * N * 16 + e * 16), last);   // bytes from a base that is the same in all lanes
    w[p] = *(global_ptr<const u32x4_any>)(gmem((const uint8_t*)z_row) + at);
  }
  // the list, and the logits of its entries behind the row's own
  Entry r;
  float y = -INFINITY;
  if (e < A.top) {
    if (outside(A, raw.id)) {
      if (A.tokens * A.top > kFewEntries) atomicOr(A.status, kStatusIndex);
    } else if (raw.id != A.pad_id && raw.y != -INFINITY) {
      r.id = (int32_t)raw.id;
      y = raw.y;
    }
  }
  bits z_bits = 0;   // as they are: made a value here, they would be waited for, and the row with them
  if (r.id >= 0) z_bits = gmem((const bits*)A.z)[row * A.ld + r.id];
  float weight = weight_of(A, row);
  // the row, as it comes in, one piece after the other
  constexpr uint32_t kNone = DT == ISO_BF16 ? 0xFF80FF80u : 0xFF800000u;
  const u32x4_t none = {kNone, kNone, kNone, kNone};
  Lse l;
#pragma unroll
  for (int p = 0; p < PER; p += 2) {
    asm volatile("" : "+v"(w[p]), "+v"(w[p + 1]), "+v"(l.s), "+v"(l.m), "+v"(mine));
    float v[2 * V];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int32_t c = (p + u) * N * V + (int32_t)mine;
      if ((p + u + 1) * N * V > vocab && c > vocab - V) w[p + u] = c == whole ? S.rest : none;
      unpack_raw<DT>(w[p + u], v + u * V);
    }
    add_to<2 * V>(l, v, A.c);
  }
  asm volatile("" : "+v"(z_bits), "+v"(weight));
  const float z = f32_from_bits(DT == ISO_BF16 ? (uint32_t)z_bits << 16 : (uint32_t)z_bits);
  put_lse(l, S.red, Join{});
  put_lse(one(r.id >= 0, y), S.list.red, JoinList{A.c});
  if (e < ISO_DISTILL_MAX_TOP) S.list.id[e] = r.id, S.list.t[e] = y;
  S.head[e] = -1;
  __syncthreads();
  l = get_lse<N>(S.red, Join{});
  Lse t = get_lse<256>(S.list.red, JoinList{A.c});   // the first four waves hold the entries
  const bool any = t.s != 0.0f;
  t.s = 1.0f / t.s;
  if (r.id >= 0) r.log_t = log_share_of(A, y, t), r.t = share_of(A, y, t);
  const double lse = lse_of(A, l);
  const Factor F(A, weight, lse, any);
  double part = r.id >= 0 && r.t != 0.0f ? (double)r.t * ((double)r.log_t - (double)z / A.t + lse) : 0.0;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) part += __shfl_xor(part, d);
  if ((e & 63) == 0 && e < 256) S.sums[e >> 6] = part;
  if (!F.zero && r.id >= 0) {   // as merge(), but for the logits in LDS; the first of the entries adds in their order
    r.first = true;
    for (int i = 0; i < A.top; ++i)
      if (S.list.id[i] == r.id && i != e) {
        if (i < e) r.first = false;
        r.t += share_of(A, S.list.t[i], t);
      }
  }
  if (r.first) {
    S.value[e] = F.f * (F.probability(A, z) - r.t);
    S.next[e] = (int16_t)atomicExch(&S.head[r.id / V % N], e);
  }
  // every entry has its logit: the gradient may lie over the logits
  asm volatile("s_waitcnt vmcnt(0)" ::"v"(z) : "memory");
  __syncthreads();
  if (e == 0) {
    part = S.sums[0] + S.sums[1] + S.sums[2] + S.sums[3];
    gmem(A.loss)[row] = F.zero ? 0.0f : (float)(weight * A.t * A.t * part);
    gmem(A.lse)[row] = (float)lse;
  }
  const int head = S.head[e];
  uint32_t has = 0;
  for (int i = head; i >= 0; i = S.next[i]) has |= 1u << (S.list.id[i] / (N * V));
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    asm volatile("" : "+v"(w[p]), "+v"(mine));   // unpacked again: there are registers for the row, not for its values twice over
    bits* const at = (bits*)A.grad + row * A.ld_grad + p * N * V;
    const int32_t left = vocab - p * N * V - (int32_t)mine;
    if (left <= 0) continue;
    float v[V] = {};
    if (!F.zero) grads_of<DT>(A, F, w[p], v);
    if (has >> p & 1u)
      for (int i = head; i >= 0; i = S.next[i]) {
        const int32_t id = S.list.id[i];
        if (id / (N * V) != p) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = id % V == j ? S.value[i] : v[j];
      }
    if ((p + 1) * N * V <= vocab) store_elems<DT, V, STREAM>(at, mine, v);
    else store_elems<DT, V, STREAM>(at, mine, v, left);
  }
}

// A piece of a row: its share of the sum, and from these the loss.  Both are latency: 3.4 and 3.5 us for one token of 151936.
template <int DT>
__global__ void __launch_bounds__(256) k_distill_part(DistillArgs A, int64_t each) {
  __shared__ ListSpace S;
  if (blockIdx.x == 0 && A.tokens * A.top <= kFewEntries) check_ids(A);
  const int64_t row = blockIdx.x / A.pieces, lo = (blockIdx.x - row * A.pieces) * each;
  const Lse l = row_lse<DT, 256>(A, row, lo, min(lo + each, A.vocab), S.red);
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
  l = block_lse<256>(l, S.red, Join{});
  __syncthreads();
  bool any;
  const Entry r = list_of<256>(A, row, S, any);
  const float z = r.id >= 0 ? load_z<DT>(A, row * A.ld + r.id) : 0.0f;
  store_loss<DT>(A, row, r, z, lse_of(A, l), any, sums);
}

// The gradient of a piece of a row from the row's L: kGradPiece columns a workgroup, four loads a lane, which are under way
// while the list is looked at (4096 x 152064 bf16: 473 us, 5.3 TB/s).
template <int DT>
constexpr int kGradPiece = 4 * 256 * kVec<DT>;

template <int DT, bool STREAM>
__global__ void __launch_bounds__(256) k_distill_grad(DistillArgs A, uint32_t pieces, bool check) {
  constexpr int V = kVec<DT>;
  __shared__ ListSpace S;
  if (blockIdx.x == 0 && check) check_ids(A);
  const int64_t row = blockIdx.x / pieces, lo = (int64_t)(blockIdx.x - (uint32_t)row * pieces) * kGradPiece<DT>;
  const int64_t c = lo + (int64_t)threadIdx.x * V;
  u32x4_t w[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) w[u] = load_end<DT>(A.z, row * A.ld + c + u * 256 * V, A.vocab - (c + u * 256 * V));
  bool any;
  Entry r = list_of<256>(A, row, S, any);
  const bool here = r.id >= lo && r.id < lo + kGradPiece<DT>;
  const float z = here ? load_z<DT>(A, row * A.ld + r.id) : 0.0f;
  if (here) merge(A, S, r);
  const Factor F(A, weight_of(A, row), gmem(A.lse)[row], any);
  before_writes(z);
  put_grads<DT, 4, STREAM>(A, row, c, F, w);
  put_entry<DT>(A, row, lo, lo + kGradPiece<DT>, F, r, z);
}

DistillArgs args_of(const iso_distill& d, uint8_t* ws) {
  DistillArgs A{};
  A.z = d.logits, A.ids = d.ids, A.y = d.teacher, A.w = d.weight, A.loss = d.loss, A.lse = d.lse, A.grad = d.grad;
  A.tokens = d.tokens, A.vocab = d.vocab, A.ld = d.ld, A.ld_grad = d.ld_grad, A.pad_id = d.pad_id;
  A.top = d.top, A.id_type = d.id_type;
  A.log2e_t = 1.4426950408889634 / d.temperature, A.c = (float)A.log2e_t, A.t = d.temperature, A.tc = A.t * A.c, A.inv_tc = 1.0 / A.tc;
  A.status = (uint32_t*)ws;
  A.part = (float*)(ws + kStatusBytes);
  return A;
}

// Workgroups that a row is shared out to where there are few, a piece 8 KiB at least; and columns of a piece.
int64_t share_out(DistillArgs& A, int dt) {
  const int64_t least = 8192 / (dt == ISO_BF16 ? 2 : 4), most = std::max<int64_t>(1, kMostPieces / 2 / A.tokens);
  A.pieces = (int32_t)std::min((A.vocab + least - 1) / least, most);
  const int64_t each = (A.vocab + A.pieces - 1) / A.pieces;
  return (each + 7) / 8 * 8;
}

template <int DT, bool STREAM>
void gradient(const DistillArgs& A, bool check, hipStream_t s) {
  const uint32_t pieces = (uint32_t)((A.vocab + kGradPiece<DT> - 1) / kGradPiece<DT>);
  k_distill_grad<DT, STREAM><<<(unsigned)(A.tokens * pieces), 256, 0, s>>>(A, pieces, check);
}

// Rows with a gradient that fit into a workgroup's registers are read once (k_distill_held), others' loss is formed before their
// gradient: both in one kernel, with two walks over a row, took 7 to 17% longer (2048 x 152064 fp32: 737 us for 665).  Few long rows
// are shared out, loss and join and gradient in a launch each; microseconds for rows of 304 KB, shared out and whole, with the
// gradient 1 token 17, 25; 64 27, 28; 128 39, 29; the loss alone 1 token 13.1, 13.7; 64 13.4, 14.6; 128 20.6, 17.2; rows of 200 KB with
// the gradient 1 token 17, 22; 64 23, 25; the loss alone 13.5, 10; rows of 100 KB with the gradient 18, 17.  Where there is no more than a row a CU, 1024 threads have it (608 KB, 128 rows: 20 us, with 256
// threads 33; 512 rows: 59 and 52).
template <int DT, bool STREAM>
void loss(DistillArgs A, hipStream_t s) {
  constexpr int V = kVec<DT>;
  const unsigned n = (unsigned)A.tokens;
  const bool held = A.grad != nullptr && A.vocab >= V && A.vocab <= 1024 * 20 * V;
  const bool shared = A.vocab > ((A.grad != nullptr ? 128 : 256) << 10) * V / 16 && A.tokens <= 64;
  if (held && !shared) {
    if (A.vocab <= 256 * 4 * V) k_distill_held<DT, 256, 4, STREAM><<<n, 256, 0, s>>>(A);
    else if (A.vocab <= 256 * 20 * V) k_distill_held<DT, 256, 20, STREAM><<<n, 256, 0, s>>>(A);
    else if (A.vocab <= 512 * 20 * V) k_distill_held<DT, 512, 20, STREAM><<<n, 512, 0, s>>>(A);
    else k_distill_held<DT, 1024, 20, STREAM><<<n, 1024, 0, s>>>(A);
    return;
  }
  if (shared) {
    const int64_t each = share_out(A, DT);
    k_distill_part<DT><<<n * A.pieces, 256, 0, s>>>(A, each);
    k_distill_join<DT><<<n, 256, 0, s>>>(A);
  } else if (n <= 256) {
    k_distill_row<DT, 1024><<<n, 1024, 0, s>>>(A);
  } else {
    k_distill_row<DT, 256><<<n, 256, 0, s>>>(A);
  }
  if (A.grad != nullptr) gradient<DT, STREAM>(A, false, s);
}

bool streams(const DistillArgs& A, int dt) { return A.grad != nullptr && streamed(A.tokens * A.vocab * (dt == ISO_BF16 ? 2 : 4)); }

}  // namespace

hipError_t run_distill_loss(const iso_distill& d, int dt, uint8_t* ws, hipStream_t s) {
  const DistillArgs A = args_of(d, ws);
  if (A.tokens == 0 || A.tokens * A.top > kFewEntries) k_distill_clear<<<1, 1, 0, s>>>(A.status);
  if (A.tokens > 0) streams(A, dt) ? (dt == ISO_BF16 ? loss<ISO_BF16, true>(A, s) : loss<ISO_F32, true>(A, s))
                                  : (dt == ISO_BF16 ? loss<ISO_BF16, false>(A, s) : loss<ISO_F32, false>(A, s));
  return hipGetLastError();
}

hipError_t run_distill_grad(const iso_distill& d, int dt, uint8_t* ws, hipStream_t s) {
  const DistillArgs A = args_of(d, ws);
  const bool few = A.tokens * A.top <= kFewEntries;
  if (A.tokens == 0 || !few) k_distill_clear<<<1, 1, 0, s>>>(A.status);
  if (A.tokens > 0) streams(A, dt) ? (dt == ISO_BF16 ? gradient<ISO_BF16, true>(A, few, s) : gradient<ISO_F32, true>(A, few, s))
                                  : (dt == ISO_BF16 ? gradient<ISO_BF16, false>(A, few, s) : gradient<ISO_F32, false>(A, few, s));
  return hipGetLastError();
}

}  // namespace iso
