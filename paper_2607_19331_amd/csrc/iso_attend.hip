// Attention over packed sequences, forward: O = softmax(scale Q K^T) V and the log-sum-exp of its rows.
#include "iso_attend_tiles.h"
#include "iso_grad.h"

namespace iso {

namespace {

// One pass over the keys that a tile sees, with the running maximum m and sum l of the softmax: a panel's scores X, P = 2^(X c - m),
// l += sum of P, O += P V, and O and l scaled where m has grown.
//
// A workgroup has 128 rows of a kv head's list (queries times the group, so that one token a sequence fills tiles too), a wave 32 of
// them; panels of 64 keys (32 in fp32) and their values lie in LDS twice over, loaded there by the memory unit while the one before
// is worked on.  X is formed as K Q^T, a row a lane: maximum and sum are a lane's own (and its other half's), and P is the second
// operand of the product with V where it is.  Q and O stay in registers.  With bf16, P is rounded to bf16 for that product, whose operands
// are of one type (P in two parts would be half as many products again); l is the sum of what was not rounded.  Of 2.1 thousandths by
// which O is off then, 1.6 are its own rounding.
//
// What bounds it: D = 128 the matrix instructions, 55% of the cycles at the 1.75 GHz that the card holds under them: four sequences
// of 4096 tokens, 28 heads over 4, causal, 500 us, 960 TFLOP/s (16 heads, all keys seen, 1035; a large product of the library 1200).
// D = 64 the exponentials and what goes with them, twice the matrix instructions' cycles (32 heads over 8: 325 us, 850 TFLOP/s).
// fp32 the matrix rate of its type (154 TFLOP/s, a sixteenth of bf16's): 8 heads of 128, one sequence of 8192, all keys seen, 122
// TFLOP/s with one wave a SIMD; causal, four of 2048, 314 us, 110.  Few rows: keys are shared out to pieces, see share_out; one token
// over 77 to 8192 keys for 16 sequences, 28 heads, 30 us with the join, 3.5 TB/s, of which 5 are a workgroup's start and 6 the join's
// launch.  One wave of four has rows there; in fp32 (139 us, 1.5 TB/s) its matrix instructions bound it.
template <int DT, int D>
__global__ void __launch_bounds__(256, (DT == ISO_F32 && D == 128 ? 1 : 2)) k_attend(AttnArgs A, Deal deal) {
  using P = Panel<DT, D>;
  constexpr int kRows = 32 * kAttnWaves, KT = P::kTiles;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  if (blockIdx.x == gridDim.x - 1) return check_starts(A);
  int head;
  uint32_t item;
  Item it;
  if (!dealt(deal, A.heads_kv, blockIdx.x, head, item) || !find_item<false, kRows>(A, A.pieces, item, it)) return;
  const Seq s = it.s;
  const int piece = it.piece;

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int32_t rows = s.nq * A.group, row0 = (int32_t)it.tile * kRows, end = min(row0 + kRows, rows);
  const Span all = span_of(A, s, row0, end - 1);
  const int pieces = pieces_of(all, A.pieces);
  if (piece >= pieces) return;
  const int tiles = (all.hi - all.lo + P::kRows - 1) / P::kRows;
  const int first = __builtin_amdgcn_readfirstlane((int)((uint32_t)tiles * (uint32_t)piece / (uint32_t)pieces));
  const int last = __builtin_amdgcn_readfirstlane((int)((uint32_t)tiles * (uint32_t)(piece + 1) / (uint32_t)pieces));

  // a lane has one row of its wave's 32, the halves of a wave different keys
  const int32_t r = row0 + 32 * w + (lane & 31), i = (int32_t)((uint32_t)r / (uint32_t)A.group);
  const int h = head * A.group + r - i * A.group;
  const bool on = r < end, busy = row0 + 32 * w < end;
  int32_t lo = 0, hi = 0;
  if (on) keys_of(A, s, i, lo, hi);
  Span mine{0, 0, 0, 0};
  if (busy) mine = span_of(A, s, row0 + 32 * w, min(row0 + 32 * w + 32, end) - 1);
  if (row0 + 32 * w + 32 > end) mine.lo_all = INT32_MAX;   // rows past the end see nothing

  const int64_t col = (int64_t)head * A.dim;
  Rows<DT, D> kr(A.k, s.k0 + all.lo, A.ld_k, col, s.nk - all.lo, A.dim, w, lane);
  Rows<DT, D> vr(A.v, s.k0 + all.lo, A.ld_v, col, s.nk - all.lo, A.dim, w, lane);
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_u8*)smem);
  constexpr uint32_t kV = 2 * P::kBytes;   // two panels of keys, then two of values
  const Reader<DT, D> rd(lds, lane);

  kr.skip(first), vr.skip(first);
  if (first < last) {
    kr.load(lds, w);
    vr.load(lds + kV, w);
    kr.load(lds + P::kBytes, w);
  }
  OwnRow<DT, D> q;
  q.load(A.q, (s.q0 + i) * A.ld_q + (int64_t)h * A.dim, A.dim, half, on);

  f32x16_t o[D / 32], x0[KT], x1[KT];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) o[d] = 0.0f;
  float m = -INFINITY, l = 0.0f;   // running maximum (times log2 e) and sum of a lane's row, the sum of its half's keys
  float top = -INFINITY;           // of the scores at hand, times log2 e

  auto scores = [&](f32x16_t (&x)[KT], int b) {
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      x[j] = 0.0f;
#pragma unroll
      for (int g = 0; g < P::kGroups; ++g) multiply<DT>(rd.row(b * P::kBytes, j, g), q.g[g], x[j]);
    }
  };
  auto most = [&](const f32x16_t (&x)[KT]) {
    float v = x[0][0];
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) v = fmaxf(v, x[j][e]);
    return both_halves(v) * A.scale2;
  };
  auto follow = [&] {   // the sums so far are scaled to a new reference where the maximum has grown by much
    if (__any(top > m + kSlack)) {
      const float up = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - (up == -INFINITY ? 0.0f : up));
      m = up;
      l *= f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] *= f;
    }
    return m == -INFINITY ? 0.0f : m;
  };
  // Probabilities of a tile and their product with V, and the next tile's scores, under whose products the exponentials run; the
  // next maximum is taken under the products with V.  Laid out by hand, one fragment read and a share of the rest a product.  One
  // way through for all tiles (those that the wave sees nothing of as well): sums that meet from two ways cost registers.
  auto step = [&](f32x16_t (&x)[KT], f32x16_t (&next)[KT], int t, int b) {   // b: the tile's panels
    landed();   // K of t + 1 and V of t, loaded a step ago; K of t and V of t - 1 are free
    kr.load(lds + b * P::kBytes, w);
    vr.load(lds + kV + (b ^ 1) * P::kBytes, w);
    const int32_t k0 = all.lo + t * P::kRows;
    if (k0 < mine.lo_all || k0 + P::kRows > mine.hi_all) {
#pragma unroll
      for (int j = 0; j < KT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int32_t key = k0 + 32 * j + 8 * (e / 4) + 4 * half + e % 4;
          x[j][e] = (uint32_t)(key - lo) < (uint32_t)(hi - lo) ? x[j][e] : -INFINITY;
        }
      top = most(x);
    }
    const float ref = follow();
    if constexpr (DT == ISO_BF16) {
      constexpr int G = P::kGroups, N = D / 32, kS = KT * G, kO = 2 * KT * N, kAhead = 3;
      u32x4_t ring[kAhead];
      auto read = [&](int n) {
        if (n < kS) ring[n % kAhead] = rd.row((b ^ 1) * P::kBytes, n / G, n % G);
        else if (n < kS + kO) ring[n % kAhead] = __builtin_bit_cast(u32x4_t, rd.col(kV + b * P::kBytes, (n - kS) / (2 * N), (n - kS) / N % 2, (n - kS) % N));
      };
#pragma unroll
      for (int n = 0; n < kAhead; ++n) read(n);
      Packed<DT> p[KT];
#pragma unroll
      for (int j = 0; j < KT; ++j) next[j] = 0.0f;
#pragma unroll
      for (int n = 0; n < kS; ++n) {
        multiply<DT>(ring[n % kAhead], q.g[n % G], next[n / G]);
        read(n + kAhead);
        constexpr int E = KT * 16 / kS;
#pragma unroll
        for (int e = E * n; e < E * (n + 1); e += 2) {
          const float u = __builtin_amdgcn_exp2f(fmaf(x[e / 16][e % 16], A.scale2, -ref));
          const float v = __builtin_amdgcn_exp2f(fmaf(x[e / 16][e % 16 + 1], A.scale2, -ref));
          l += u;
          l += v;
          p[e / 16].set(e % 16 / 2, u, v);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      float v = next[0][0];
#pragma unroll
      for (int n = 0; n < kO; ++n) {
        multiply<DT>(ring[(kS + n) % kAhead], p[n / (2 * N)].s[n / N % 2], o[n % N]);
        read(kS + n + kAhead);
        constexpr int E = KT * 16 / kO;
#pragma unroll
        for (int e = E * n; e < E * (n + 1); ++e) v = fmaxf(v, next[e / 16][e % 16]);
        __builtin_amdgcn_sched_barrier(0);
      }
      top = both_halves(v) * A.scale2;
    } else {
      if (t + 1 < last) scores(next, b ^ 1);   // bf16 has its own after the last tile too: a sixteenth of this time
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        Packed<DT> p;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float u = __builtin_amdgcn_exp2f(fmaf(x[j][e], A.scale2, -ref)), v = __builtin_amdgcn_exp2f(fmaf(x[j][e + 1], A.scale2, -ref));
          l += u;
          l += v;
          p.set(e / 2, u, v);
        }
        multiply_columns<DT, D>(rd, kV + b * P::kBytes, j, p, o);
      }
      top = most(next);
    }
  };

  if (first < last) {
    landed();
    if (busy) {
      scores(x0, 0);
      top = most(x0);
      for (int t = first; t < last; t += 2) {
        step(x0, x1, t, 0);
        if (t + 1 == last) break;
        step(x1, x0, t + 1, 1);
      }
    } else {   // a wave without rows has its share of the loads
      for (int t = first; t < last; ++t) {
        const int b = (t - first) & 1;
        landed();
        kr.load(lds + b * P::kBytes, w);
        vr.load(lds + kV + (b ^ 1) * P::kBytes, w);
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may reach LDS after the workgroup's end
  l = sum_of_halves(l);

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

// O = sum of 2^(m_p - m) O_p / sum of 2^(m_p - m) l_p over a row's pieces p, m the largest m_p; half a wave a row, four dimensions a
// lane.  Its time is latency (the row's sequence, then the pieces, U at once): 6 us for 16 tokens of 28 heads in up to 13 pieces.
template <int DT, int U>
__global__ void __launch_bounds__(256) k_attend_join(AttnArgs A) {
  constexpr int kRows = 32 * kAttnWaves;
  const int lane = threadIdx.x & 63, l32 = lane & 31, c = 4 * l32;
  const JoinRow j(A, (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5));
  const Span all = j.on ? span_of(A, j.s, j.r / kRows * kRows, min(j.r / kRows * kRows + kRows, j.s.nq * A.group) - 1) : Span{0, 0, 0, 0};
  const int pieces = pieces_of(all, A.pieces);
  const bool on = j.on && pieces > 1;
  const int64_t next = A.tokens_q * A.heads * kPartLd;
  Parts<U> parts(A.part + j.at * kPartLd, next, c, on && c < A.dim ? pieces : 0);
  const auto part = gmem((const float*)A.part) + j.at * kPartLd;
  float m[2], l[2], f[2];   // of pieces l32 and l32 + 32
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool has = on && l32 + 32 * i < pieces;
    m[i] = has ? part[(l32 + 32 * i) * next + 128] : -INFINITY;
    l[i] = has ? part[(l32 + 32 * i) * next + 129] : 0.0f;
  }
  float top = fmaxf(m[0], m[1]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[i] = __builtin_amdgcn_exp2f(m[i] - (top == -INFINITY ? 0.0f : top));
    sum += l[i] * f[i];
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  float o[4] = {};
  parts.add([&](int p) { return __shfl(p < 32 ? f[0] : f[1], (lane & 32) | (p & 31)); }, o);
  int32_t lo = 0, hi = 0;
  if (on) keys_of(A, j.s, j.r / A.group, lo, hi);
  const float inv = hi > lo ? 1.0f / sum : 0.0f;
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] *= inv, t = fmaf(o[i], 0.0f, t);
  const uint64_t bad = __ballot(t != 0.0f);
  if (on && (uint32_t)(bad >> (lane & 32)) == 0) {
    if (c < A.dim) store_elems<DT, 4>(A.out, j.t * A.ld_out + (int64_t)j.h * A.dim + c, o);
    if (l32 == 0) gmem(A.lse)[j.at] = hi > lo ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
  }
#pragma unroll 1
  for (int i = 0; i < 2; ++i)
    if ((uint32_t)(bad >> (32 * i)) != 0) {
      const JoinRow row = j.of(32 * i);
      attend_row<DT>(A, row.s, row.h / A.group, row.r, lane);
    }
}

template <int DT, int D>
hipError_t forward(const AttnArgs& A, hipStream_t s) {
  Deal deal = deal_of(A.heads_kv, attend_items(A.tokens_q * A.group, A.tokens_k, A.sequences, A.pieces));
  if (A.pieces.most == 1 && !(DT == ISO_F32 && D == 128)) deal = folded(deal, A.heads_kv, A.tokens_q * A.heads / kAttnTileRows);
  k_attend<DT, D><<<deal_grid(deal, A.heads_kv) + 1, 256, 4 * Panel<DT, D>::kBytes, s>>>(A, deal);   // one looks at the offsets
  const unsigned rows = (unsigned)((A.tokens_q * A.heads + 7) / 8);
  if (A.pieces.most > 4) k_attend_join<DT, 8><<<rows, 256, 0, s>>>(A);
  else if (A.pieces.most > 1) k_attend_join<DT, 4><<<rows, 256, 0, s>>>(A);
  return hipGetLastError();
}

template <int DT>
hipError_t forward(const AttnArgs& A, hipStream_t s) {
  return A.dim > 64 ? forward<DT, 128>(A, s) : forward<DT, 64>(A, s);
}

}  // namespace

hipError_t run_attend(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s) {
  AttnArgs A = args_of(a, ws);
  const AttendPlan plan = plan_attend(a, false);
  A.pieces = plan.rows;
  A.part = (float*)(ws + plan.part);
  return dt == ISO_BF16 ? forward<ISO_BF16>(A, s) : forward<ISO_F32>(A, s);
}

}  // namespace iso
