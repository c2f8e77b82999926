// Attention over packed sequences, forward: O = softmax(scale Q K^T) V and the log-sum-exp of its rows.
#include <algorithm>

#include "iso_attend_tiles.h"
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

// Keys that the rows of a tile (or of a wave of it) see between them, and those that all of them see.
struct Span {
  int32_t lo, hi, lo_all, hi_all;
};
// Bounds grow with the query, so those of the first and last row do for all.
__device__ __forceinline__ Span span_of(const AttnArgs& A, const Seq& s, int64_t first, int64_t last) {
  Span x;
  keys_of(A, s, first / A.group, x.lo, x.hi_all);
  keys_of(A, s, last / A.group, x.lo_all, x.hi);
  return x;
}

// Pieces that the keys [lo, hi) of a tile are shared out to: of kPieceKeys at least, `most` at most.
__device__ __forceinline__ int pieces_of(int32_t lo, int32_t hi, int most) {
  return min(most, max(1, (hi - lo + kPieceKeys - 1) / kPieceKeys));
}

template <int DT, int D>
__global__ void __launch_bounds__(256, 2) k_attend(AttnArgs A, Deal deal) {
  using P = Panel<DT, D>;
  constexpr int kRows = 32 * kAttnWaves, KT = P::kTiles;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  if (blockIdx.x == 0) check_starts(A);
  int head;
  uint32_t tile, at;
  Seq s;
  if (!dealt(deal, A.heads_kv, blockIdx.x, head, tile)) return;
  const int piece = (int)(tile % (uint32_t)A.pieces);
  if (!find_tile<false, kRows>(A, tile / (uint32_t)A.pieces, s, at)) return;

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int32_t rows = s.nq * A.group, row0 = (int32_t)at * kRows, end = min(row0 + kRows, rows);
  const Span all = span_of(A, s, row0, end - 1);
  const int pieces = pieces_of(all.lo, all.hi, A.pieces);
  if (piece >= pieces) return;
  const int tiles = (all.hi - all.lo + P::kRows - 1) / P::kRows;
  const int first = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * piece / pieces));
  const int last = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * (piece + 1) / pieces));

  // a lane has one row of its wave's 32, the halves of a wave different keys
  const int32_t r = row0 + 32 * w + (lane & 31), i = r / A.group;
  const int h = head * A.group + r - i * A.group;
  const bool on = r < end, busy = row0 + 32 * w < end;
  int32_t lo = 0, hi = 0;
  if (on) keys_of(A, s, i, lo, hi);
  Span mine{0, 0, 0, 0};
  if (busy) mine = span_of(A, s, row0 + 32 * w, min(row0 + 32 * w + 32, end) - 1);
  if (row0 + 32 * w + 32 > end) mine.lo_all = INT32_MAX;   // rows past the end see nothing

  const int64_t col = (int64_t)head * A.dim;
  const Rows<DT, D> kr(A.k, s.k0 + all.lo, A.ld_k, col, s.nk - all.lo, A.dim, w, lane);
  const Rows<DT, D> vr(A.v, s.k0 + all.lo, A.ld_v, col, s.nk - all.lo, A.dim, w, lane);
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_u8*)smem);
  auto k_panel = [&](int t) { return lds + (t & 1) * P::kBytes; };
  auto v_panel = [&](int t) { return lds + (2 + (t & 1)) * P::kBytes; };
  const Reader<DT, D> rd(lane);

  if (first < last) {
    kr.load(first, k_panel(first), w);
    vr.load(first, v_panel(first), w);
    kr.load(first + 1, k_panel(first + 1), w);
  }
  OwnRow<DT, D> q;
  q.load(A.q, (s.q0 + i) * A.ld_q + (int64_t)h * A.dim, A.dim, half, on);

  f32x16_t o[D / 32], x0[KT], x1[KT];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) o[d] = 0.0f;
  float m = -INFINITY, l = 0.0f;   // running maximum (times log2 e) and sum of a lane's row, the sum of its half's keys

  auto scores = [&](f32x16_t (&x)[KT], int t) {
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      x[j] = 0.0f;
#pragma unroll
      for (int g = 0; g < P::kGroups; ++g) multiply<DT>(rd.row(k_panel(t), j, g), q.g[g], x[j]);
    }
  };
  auto needed = [&](int t) {   // keys of the tile that a row of the wave sees
    const int32_t k0 = all.lo + t * P::kRows;
    return busy && k0 < mine.hi && k0 + P::kRows > mine.lo;
  };
  auto step = [&](f32x16_t (&x)[KT], f32x16_t (&next)[KT], int t) {
    landed();   // K of t + 1 and V of t, loaded a step ago; K of t and V of t - 1 are free
    kr.load(t + 2, k_panel(t), w);
    vr.load(t + 1, v_panel(t + 1), w);
    if (needed(t + 1)) scores(next, t + 1);
    if (!needed(t)) return;
    const int32_t k0 = all.lo + t * P::kRows;
    if (k0 < mine.lo_all || k0 + P::kRows > mine.hi_all) {
#pragma unroll
      for (int j = 0; j < KT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int32_t key = k0 + 32 * j + 8 * (e / 4) + 4 * half + e % 4;
          x[j][e] = (uint32_t)(key - lo) < (uint32_t)(hi - lo) ? x[j][e] : -INFINITY;
        }
    }
    float top = x[0][0];
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, x[j][e]);
    top = fmaxf(top, other_half(top)) * A.scale2;
    if (__any(top > m + kSlack)) {   // the sums so far are scaled to a new reference
      const float up = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - (up == -INFINITY ? 0.0f : up));
      m = up;
      l *= f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] *= f;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      Packed<DT> p;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float a = __builtin_amdgcn_exp2f(fmaf(x[j][e], A.scale2, -ref)), b = __builtin_amdgcn_exp2f(fmaf(x[j][e + 1], A.scale2, -ref));
        l += a;
        l += b;
        p.set(e / 2, a, b);
      }
      multiply_columns<DT, D>(rd, v_panel(t), j, p, o);
    }
  };

  if (first < last) {
    landed();
    if (needed(first)) scores(x0, first);
    for (int t = first; t < last; t += 2) {
      step(x0, x1, t);
      if (t + 1 < last) step(x1, x0, t + 1);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may reach LDS after the workgroup's end
  l += other_half(l);

  const int64_t to = s.q0 + i;
  if (pieces > 1) {   // k_attend_join adds the pieces up
    if (!on) return;
    float* const part = A.part + (((int64_t)piece * A.tokens_q + to) * A.heads + h) * kPartLd;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int c = 32 * d + 2 * e + 4 * half;
        if (c < A.dim) store_elems<ISO_F32, 4>(part, c, (const float*)&o[d] + e);
      }
    if (half == 0) gmem(part)[128] = m, gmem(part)[129] = l;
    return;
  }
  const bool sees = hi > lo;
  const float f = sees ? 1.0f / l : 0.0f;
  // a row that is not finite may have met such a value at a key that it does not see
  const bool bad = on && trouble(o, f) != 0.0f;
  if (on && !bad) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int c = 32 * d + 2 * e + 4 * half;
        const float v[4] = {o[d][e] * f, o[d][e + 1] * f, o[d][e + 2] * f, o[d][e + 3] * f};
        if (c < A.dim) store_elems<DT, 4>(A.out, to * A.ld_out + (int64_t)h * A.dim + c, v);
      }
    if (half == 0) gmem(A.lse)[to * A.heads + h] = sees ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
  for (uint64_t rest = __ballot(bad); rest != 0;) {
    const int n = __builtin_ctzll(rest) & 31;
    rest &= ~(0x100000001ull << n);
    attend_row<DT>(A, s, head, row0 + 32 * w + n, lane);
  }
}

// Adds up the pieces of a row, one wave a row.
template <int DT>
__global__ void __launch_bounds__(256) k_attend_join(AttnArgs A) {
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), t = at / A.heads;
  if (t >= A.tokens_q) return;
  const Seq s = seq_at(A, A.start_q, t);
  if (t < s.q0 || t >= s.q0 + s.nq) return;
  constexpr int kRows = 32 * kAttnWaves;
  const int h = (int)(at - t * A.heads), head = h / A.group, lane = threadIdx.x & 63;
  const int32_t r = (int32_t)(t - s.q0) * A.group + h % A.group, row0 = r / kRows * kRows;
  const Span all = span_of(A, s, row0, min(row0 + kRows, s.nq * A.group) - 1);
  const int pieces = pieces_of(all.lo, all.hi, A.pieces);
  if (pieces == 1) return;
  const auto part = gmem((const float*)A.part) + at * kPartLd;
  const int64_t next = A.tokens_q * A.heads * kPartLd;
  const float mine = lane < pieces ? part[lane * next + 128] : -INFINITY;
  const float m = wave_max(mine), f = __builtin_amdgcn_exp2f(mine - (m == -INFINITY ? 0.0f : m));
  const float l = wave_sum(lane < pieces ? part[lane * next + 129] * f : 0.0f);
  int32_t lo, hi;
  keys_of(A, s, r / A.group, lo, hi);
  float o[2] = {0.0f, 0.0f};
  for (int p = 0; p < pieces; ++p) {
    const float g = __shfl(f, p);
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (lane + 64 * c < A.dim) o[c] = fmaf(part[p * next + lane + 64 * c], g, o[c]);
  }
  const float inv = hi > lo ? 1.0f / l : 0.0f;
  if (__any(fmaf(o[0] * inv, 0.0f, o[1] * inv * 0.0f) != 0.0f)) return attend_row<DT>(A, s, head, r, lane);
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + 64 * c < A.dim) store_one<DT>(A.out, t * A.ld_out + (int64_t)h * A.dim + lane + 64 * c, o[c] * inv);
  if (lane == 0) gmem(A.lse)[at] = hi > lo ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
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

template <int DT, int D>
hipError_t forward(const AttnArgs& A, hipStream_t s) {
  const Deal deal = deal_of(A.heads_kv, (uint32_t)(attend_tiles(A.tokens_q * A.group, A.sequences) * A.pieces));
  k_attend<DT, D><<<std::max(1u, deal_grid(deal, A.heads_kv)), 256, 4 * Panel<DT, D>::kBytes, s>>>(A, deal);
  if (A.pieces > 1) k_attend_join<DT><<<(unsigned)((A.tokens_q * A.heads + 3) / 4), 256, 0, s>>>(A);
  return hipGetLastError();
}

template <int DT>
hipError_t forward(const AttnArgs& A, hipStream_t s) {
  return A.dim > 64 ? forward<DT, 128>(A, s) : forward<DT, 64>(A, s);
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
  AttnArgs A = args_of(a, ws);
  A.pieces = attend_pieces(a);
  A.part = (float*)(ws + kStatusBytes);
  return dt == ISO_BF16 ? forward<ISO_BF16>(A, s) : forward<ISO_F32>(A, s);
}

hipError_t run_attend_grad(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s) {
  const AttnArgs A = args_of(a, ws);
  return dt == ISO_BF16 ? backward<ISO_BF16>(A, s) : backward<ISO_F32>(A, s);
}

}  // namespace iso
