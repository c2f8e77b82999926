// Attention over packed sequences, forward: O = softmax(scale Q K^T) V and the log-sum-exp of its rows.
#include <algorithm>

#include "iso_attend.h"
#include "iso_grad.h"

namespace iso {

namespace {

// The sequence whose range holds row t; a sequence without rows where there is none.
__device__ __forceinline__ Seq seq_at(const AttnArgs& A, const int32_t* start, int64_t t) {
  if (A.sequences == 0) return Seq{};
  int32_t lo = 0, hi = A.sequences - 1;
  while (lo < hi) {   // the first sequence that ends behind t
    const int32_t m = (lo + hi) / 2;
    if (gmem(start)[m + 1] > t) hi = m;
    else lo = m + 1;
  }
  return seq_of(A, lo);
}

// One wave a row.
template <int DT>
__global__ void __launch_bounds__(256) k_attend_rows(AttnArgs A) {
  if (blockIdx.x == 0) check_starts(A);
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = at / A.heads;
  if (t >= A.tokens_q) return;
  const Seq s = seq_at(A, A.start_q, t);
  if (t < s.q0 || t >= s.q0 + s.nq) return;
  const int h = (int)(at - t * A.heads), head = h / A.group;
  attend_row<DT>(A, s, head, (t - s.q0) * A.group + h % A.group, threadIdx.x & 63);
}

// D of a row, one wave a row.
template <int DT>
__global__ void __launch_bounds__(256) k_attend_delta(AttnArgs A) {
  if (blockIdx.x == 0) check_starts(A);
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = at / A.heads;
  if (t >= A.tokens_q) return;
  const int h = (int)(at - t * A.heads), lane = threadIdx.x & 63;
  float sum = 0.0f;
  for (int d = lane; d < A.dim; d += 64)
    sum = fmaf(load_one<DT>(A.out, t * A.ld_out + (int64_t)h * A.dim + d), load_one<DT>(A.dout, t * A.ld_dout + (int64_t)h * A.dim + d), sum);
  sum = wave_sum(sum);
  if (lane == 0) gmem(A.delta)[at] = sum;
}

template <int DT>
__global__ void __launch_bounds__(256) k_attend_dq_rows(AttnArgs A) {
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = at / A.heads;
  if (t >= A.tokens_q) return;
  const Seq s = seq_at(A, A.start_q, t);
  if (t < s.q0 || t >= s.q0 + s.nq) return;
  const int h = (int)(at - t * A.heads), head = h / A.group;
  dq_row<DT>(A, s, head, (t - s.q0) * A.group + h % A.group, threadIdx.x & 63);
}

template <int DT>
__global__ void __launch_bounds__(256) k_attend_dkv_rows(AttnArgs A) {
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = at / A.heads_kv;
  if (t >= A.tokens_k) return;
  const Seq s = seq_at(A, A.start_k, t);
  if (t < s.k0 || t >= s.k0 + s.nk) return;
  dkv_row<DT>(A, s, (int)(at - t * A.heads_kv), (int32_t)(t - s.k0), threadIdx.x & 63);
}

AttnArgs args_of(const iso_attn& a, uint8_t* ws) {
  AttnArgs A{};
  A.q = a.q, A.k = a.k, A.v = a.v, A.ld_q = a.ld_q, A.ld_k = a.ld_k, A.ld_v = a.ld_v;
  A.start_q = a.start_q, A.start_k = a.start_k, A.tokens_q = a.tokens_q, A.tokens_k = a.tokens_k;
  A.sequences = (int32_t)a.sequences, A.heads = a.heads, A.heads_kv = a.heads_kv, A.group = a.heads / a.heads_kv, A.dim = a.dim;
  A.causal = a.causal, A.window = a.window;
  A.scale = (float)a.scale, A.scale2 = (float)(a.scale * 1.4426950408889634);
  A.out = a.out, A.ld_out = a.ld_out, A.lse = a.lse, A.dout = a.dout, A.ld_dout = a.ld_dout;
  A.dq = a.dq, A.dk = a.dk, A.dv = a.dv, A.ld_dq = a.ld_dq, A.ld_dk = a.ld_dk, A.ld_dv = a.ld_dv;
  A.status = (uint32_t*)ws;
  A.delta = (float*)(ws + kStatusBytes);
  return A;
}

template <int DT>
hipError_t forward(const AttnArgs& A, hipStream_t s) {
  k_attend_rows<DT><<<(unsigned)std::max<int64_t>(1, (A.tokens_q * A.heads + 3) / 4), 256, 0, s>>>(A);
  return hipGetLastError();
}

template <int DT>
hipError_t backward(const AttnArgs& A, hipStream_t s) {
  const unsigned rows = (unsigned)((A.tokens_q * A.heads + 3) / 4), keys = (unsigned)((A.tokens_k * A.heads_kv + 3) / 4);
  k_attend_delta<DT><<<std::max(rows, 1u), 256, 0, s>>>(A);
  if (rows > 0) k_attend_dq_rows<DT><<<rows, 256, 0, s>>>(A);
  if (keys > 0) k_attend_dkv_rows<DT><<<keys, 256, 0, s>>>(A);
  return hipGetLastError();
}

}  // namespace

hipError_t run_attend(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s) {
  const AttnArgs A = args_of(a, ws);
  return dt == ISO_BF16 ? forward<ISO_BF16>(A, s) : forward<ISO_F32>(A, s);
}

hipError_t run_attend_grad(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s) {
  const AttnArgs A = args_of(a, ws);
  return dt == ISO_BF16 ? backward<ISO_BF16>(A, s) : backward<ISO_F32>(A, s);
}

}  // namespace iso
