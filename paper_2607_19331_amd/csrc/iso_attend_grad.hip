// Attention over packed sequences, backward: with P = exp(scale Q K^T - L) worked out again, D = sum of dO O over a row and
// S = P (dO V^T - D),  dV = P^T dO,  dK = scale S^T Q,  dQ = scale S K.
//
// Two kinds of workgroups form P and S each for themselves: those of dkv have keys and walk over the rows that see them, those of
// dq have rows and walk over the keys that they see.  That is seven products of rows x keys x dim where one kernel would need five, but each
// result has one owner who adds in a fixed order: no atomics, the same bits every time.
//
// Both are bound by the matrix instructions (bf16, D = 128: busy 64% of the cycles, at the 1.5 to 1.6 GHz that the card holds
// under them): two sequences of 8192 tokens, 28 heads over 4, causal, 3.09 ms, 779 TFLOP/s of five products, 1090 of seven, where
// a large product of the library reaches 1200.  D = 64 (32 heads over 8, 4 x 4096): 1.08 ms, 634.  fp32 (8 heads of 128, 4 x 2048): 1.10
// ms, 78, 109 of seven, of its matrix rate's 154.
//
// With bf16, P and S are rounded to bf16 for the products with dO, Q and K, whose operands are of one type; P and S themselves and all sums
// are binary32.  Of 2.3 to 2.4 thousandths by which dQ, dK and dV are off then, 1.7 are their own rounding.
#include <algorithm>

#include "iso_attend_tiles.h"
#include "iso_grad.h"

namespace iso {

namespace {

// L log2(e) and D of every row, 16 lanes a row, in the order of the groups' lists: a panel's come into LDS with one load.  A row's place
// there does not depend on its sequence, so that none is looked up; those of rows without one are not used.  Bound by memory: O and dO
// read once (16384 tokens, 28 heads of 128: 51 us, 4.6 TB/s; 13379 tokens, 12 heads: 17 us, 4.8).
template <int DT>
__global__ void __launch_bounds__(256) k_attend_stat(AttnArgs A) {
  if (blockIdx.x == gridDim.x - 1) return check_starts(A);
  const int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), t = at / A.heads;
  if (t >= A.tokens_q || A.sequences == 0) return;   // without sequences, pointers may be null
  const int h = (int)(at - t * A.heads), head = h / A.group, c = (threadIdx.x & 15) * 8;
  float o[8] = {}, g[8] = {}, sum = 0.0f;
  if (c < A.dim) {
    load_elems<DT, 8>(A.out, t * A.ld_out + (int64_t)h * A.dim + c, o);
    load_elems<DT, 8>(A.dout, t * A.ld_dout + (int64_t)h * A.dim + c, g);
  }
  const float lse = gmem(A.lse)[at];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum = fmaf(o[j], g[j], sum);
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (c == 0) {
    const int64_t to = (head * A.tokens_q + t) * A.group + h - head * A.group;
    gmem(A.stat)[to] = lse * kLog2e;
    gmem(A.stat)[A.tokens_q * A.heads + to] = sum;
  }
}

// ---- dQ ------------------------------------------------------------------------------------------------------------

// Keys have much in common (a projection's bias) and a row's S next to no sum, so that the common part of S K cancels but for the
// sum of what the rounding of S to bf16 took.  That sum is kept, and the common part, for which the mean c of a few keys stands that
// the row sees, is added with it at the end: sum S k = sum round(S) k + sum (S - round(S)) (k - c) + c sum (S - round(S)),
// of which the middle is left out.  With a bias of twice the keys' own width the error of dQ is 2.4 thousandths instead of 4.2, of
// which 1.7 are its own rounding.
template <int DT, int D>
struct Common {
  static constexpr int kKeys = 16;
  static constexpr uint32_t kBytes = 512;   // of LDS, a wave
  // Where all rows of the wave see fewer keys than kOwn (narrow windows, the first rows of a sequence) a row has the first kOwn of its
  // own: what is left of the error is sqrt(1 + 1 / n) times the least for n keys, 3% more with 16 and 12% with 4.
  static constexpr int kOwn = 4;
  uint32_t lds;

  // Of keys [from, to) the first kKeys.  Before the loop and from memory, not from the panels as they come by: branches in the loop
  // cost registers that it has not got.
  __device__ __forceinline__ Common(const AttnArgs& A, uint32_t lds_, int64_t first, int32_t from, int32_t to, int64_t col, int lane)
      : lds(lds_) {
    const int32_t keys = min(to - from, kKeys);
    uint32_t w[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      w[i] = 0;
      if (i < keys && 2 * lane < A.dim) w[i] = pair(A, first + from + i, col, lane);
    }
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) a += f32_from_bits(w[i] << 16), b += f32_from_bits(w[i] & 0xFFFF0000u);
    const float f = 1.0f / (float)max(keys, 1);
    *(lds_word)(uintptr_t)(lds + 8 * lane) = bits_from_f32(a * f);
    *(lds_word)(uintptr_t)(lds + 8 * lane + 4) = bits_from_f32(b * f);
  }
  __device__ static __forceinline__ uint32_t pair(const AttnArgs& A, int64_t key, int64_t col, int lane) {
    return *(global_ptr<const uint32_t>)(gmem((const uint16_t*)A.k) + key * A.ld_k + col + 2 * lane);
  }

  // lost: of the lane's row, which sees keys [lo, hi) from row `first` of k on.  panel: LDS that the wave has to itself.
  __device__ __forceinline__ void add(const AttnArgs& A, uint32_t panel, int64_t first, bool on, int32_t lo, int32_t hi, int64_t col,
                                      f32x16_t (&acc)[D / 32], float lost, int lane) const {
    // what all rows see, worked out again: between the last one's first key and the first one's last
    const uint32_t rows = (uint32_t)__ballot(on), seeing = (uint32_t)__ballot(hi > lo);
    const bool own = seeing != 0 && __builtin_amdgcn_readlane(hi, 0) - __builtin_amdgcn_readlane(lo, 31 - __builtin_clz(rows)) < kOwn;
    const int half = lane >> 5;
    uint32_t at[kOwn], x[kOwn];
    float f[kOwn];
    if (own) {   // the keys as they are, in LDS
      const int end = 31 - __builtin_clz(seeing);
      const int32_t from = __builtin_amdgcn_readlane(lo, __builtin_ctz(seeing));
      const int32_t count = min(__builtin_amdgcn_readlane(lo, end) + kOwn, __builtin_amdgcn_readlane(hi, end)) - from;
      constexpr int kChunk = 12;
#pragma unroll 1
      for (int j0 = 0; j0 < count; j0 += kChunk) {
        uint32_t w[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
          w[j] = 0;
          if (2 * lane < A.dim) w[j] = pair(A, first + from + min(j0 + j, count - 1), col, lane);
        }
        if (4 * lane < 2 * D)
#pragma unroll
          for (int j = 0; j < kChunk; ++j)
            *(lds_word)(uintptr_t)(panel + (j0 + j) * 2 * D + (4 * lane ^ place(j0 + j))) = w[j];
      }
      const int32_t keys = min(hi - lo, kOwn);
#pragma unroll
      for (int k = 0; k < kOwn; ++k) {
        const int32_t key = max(lo - from + min(k, keys - 1), 0);
        at[k] = panel + key * 2 * D, x[k] = place(key) ^ 8 * half;
        f[k] = k < keys ? lost / (float)keys : 0.0f;
      }
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        f32x4_t c = 0.0f;
        if (own) {
#pragma unroll
          for (int k = 0; k < kOwn; ++k) {
            const lds_u32x2_t w = *(lds_pair)(uintptr_t)(at[k] + (x[k] ^ (64 * d + 4 * e)));
            c[0] = fmaf(f32_from_bits(w[0] << 16), f[k], c[0]), c[1] = fmaf(f32_from_bits(w[0] & 0xFFFF0000u), f[k], c[1]);
            c[2] = fmaf(f32_from_bits(w[1] << 16), f[k], c[2]), c[3] = fmaf(f32_from_bits(w[1] & 0xFFFF0000u), f[k], c[3]);
          }
        } else {
          c = *(lds_f32x4)(uintptr_t)(lds + (32 * d + 2 * e + 4 * half) * 4) * lost;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[d][e + i] += c[i];
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  // Keys' 8-byte pieces in different banks.
  __device__ static __forceinline__ uint32_t place(int key) { return D == 128 ? 8 * (key % 32) : 8 * (key / 2 % 16); }
};
// fp32 rounds no S: no sum, and no LDS.
template <int D>
struct Common<ISO_F32, D> {
  static constexpr uint32_t kBytes = 0;
  __device__ __forceinline__ Common(const AttnArgs&, uint32_t, int64_t, int32_t, int32_t, int64_t, int) {}
  __device__ __forceinline__ void add(const AttnArgs&, uint32_t, int64_t, bool, int32_t, int32_t, int64_t, f32x16_t (&)[D / 32], float, int) const {}
};

// Workgroup layout of dq_tile: two panels of keys, two of values, and what a wave keeps for Common.
template <int DT, int D>
struct Dq {
  using P = Panel<DT, D>;
  static constexpr uint32_t kV = 2 * P::kBytes, kCommon = 4 * P::kBytes;
  static constexpr uint32_t kLds = kCommon + kAttnWaves * Common<DT, D>::kBytes;
  static_assert(P::kBytes >= 36 * 2 * D, "a panel holds a wave's own keys, in whole chunks");
};

// dQ of a tile: as the forward kernel, 128 rows of a group's list a workgroup and panels of 64 keys and values in LDS twice over; Q and
// dO of a lane's row stay in registers (64 of bf16, as many as dQ has), S goes from result to operand where it is.
template <int DT, int D>
__device__ __forceinline__ void dq_tile(const AttnArgs& A, const Deal& deal, uint32_t block, uint8_t* smem) {
  using P = Panel<DT, D>;
  constexpr int kRows = 32 * kAttnWaves, KT = P::kTiles;
  int head;
  uint32_t item;
  Item it;
  if (!dealt(deal, A.heads_kv, block, head, item) || !find_item<false, kRows>(A, A.pieces, item, it)) return;
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

  const int32_t r = row0 + 32 * w + (lane & 31), i = (int32_t)((uint32_t)r / (uint32_t)A.group);
  const int h = head * A.group + r - i * A.group;
  const bool on = r < end, busy = row0 + 32 * w < end;
  int32_t lo = 0, hi = 0;
  if (on) keys_of(A, s, i, lo, hi);
  Span mine{0, 0, 0, 0};
  if (busy) mine = span_of(A, s, row0 + 32 * w, min(row0 + 32 * w + 32, end) - 1);
  const int32_t lo_all = mine.lo_all;
  if (row0 + 32 * w + 32 > end) mine.lo_all = INT32_MAX;

  const int64_t col = (int64_t)head * A.dim, to = s.q0 + i;
  Rows<DT, D> kr(A.k, s.k0 + all.lo, A.ld_k, col, s.nk - all.lo, A.dim, w, lane);
  Rows<DT, D> vr(A.v, s.k0 + all.lo, A.ld_v, col, s.nk - all.lo, A.dim, w, lane);
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_u8*)smem);
  using S = Dq<DT, D>;
  constexpr uint32_t kV = S::kV;
  Reader<DT, D> rd(lds, lane);
  kr.skip(first), vr.skip(first);
  if (first < last) {
    kr.load(lds, w);
    vr.load(lds + kV, w);
  }
  const Common<DT, D> common(A, lds + S::kCommon + w * Common<DT, D>::kBytes, s.k0, lo_all, mine.hi_all, col, lane);
  OwnRow<DT, D> q, g;
  q.load(A.q, to * A.ld_q + (int64_t)h * A.dim, A.dim, half, on);
  g.load(A.dout, to * A.ld_dout + (int64_t)h * A.dim, A.dim, half, on);
  const float lse = on ? gmem(A.stat)[list_of(A, s, head) + r] : 0.0f, delta = on ? delta_of(A, s, head, r) : 0.0f;
  q.arrive(), g.arrive();
  asm volatile("" ::"v"(lse), "v"(delta));

  f32x16_t dq[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dq[d] = 0.0f;
  float lost = 0.0f;   // what rounding took from the row's S, of its half's keys
  auto step = [&](int t, int b) {   // b: the tile's panels
    landed();
    kr.load(lds + (b ^ 1) * P::kBytes, w);
    vr.load(lds + kV + (b ^ 1) * P::kBytes, w);
    const int32_t k0 = all.lo + t * P::kRows;
    if (!busy || k0 >= mine.hi || k0 + P::kRows <= mine.lo) return;
    const bool whole = k0 >= mine.lo_all && k0 + P::kRows <= mine.hi_all;
    auto sees = [&](int j, int e) { return (uint32_t)(k0 + 32 * j + 8 * (e / 4) + 4 * half + e % 4 - lo) < (uint32_t)(hi - lo); };
    if constexpr (DT == ISO_BF16) {
      rd.again();   // kept, addresses and what Common::add needs took 20 bytes of scratch in this loop (heads of 128)
      // as in dkv_tile: fragments three products ahead, S and dP by rows, dQ by columns, one tile of 32 keys after the other
      constexpr int G = P::kGroups, N = P::kDims, kAhead = 3;
      static_assert(G == 2 * N, "as many products each");
      u32x4_t ring[kAhead];
      auto read = [&](int n) {
        const int j = n / (3 * G), i = n % (3 * G);
        if (j >= KT) return;
        if (i < G) ring[n % kAhead] = rd.row(b * P::kBytes, j, i);
        else if (i < 2 * G) ring[n % kAhead] = rd.row(kV + b * P::kBytes, j, i - G);
        else ring[n % kAhead] = __builtin_bit_cast(u32x4_t, rd.col(b * P::kBytes, j, (i - 2 * G) / N, (i - 2 * G) % N));
      };
#pragma unroll
      for (int n = 0; n < kAhead; ++n) read(n);
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        const int n0 = 3 * G * j;
        f32x16_t x = 0.0f, y = -delta;
#pragma unroll
        for (int n = 0; n < G; ++n) {
          multiply<DT>(ring[(n0 + n) % kAhead], q.g[n], x);
          read(n0 + n + kAhead);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < G; ++n) {
          multiply<DT>(ring[(n0 + G + n) % kAhead], g.g[n], y);
          read(n0 + G + n + kAhead);
#pragma unroll
          for (int e = 16 / G * n; e < 16 / G * (n + 1); ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], A.scale2, -lse));
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= y[e];
        if (!whole) {   // 0 times what is not seen may be NaN
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = sees(j, e) ? x[e] : 0.0f;
        }
        Packed<DT> ds;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          ds.set(e / 2, x[e], x[e + 1]);
          lost += x[e];
          lost += x[e + 1];
          lost = minus_pair(ds.s[e / 8][e / 2 % 4], lost);
        }
        asm volatile("" : "+v"(lost));   // here, not behind the products: x would be kept until then
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < G; ++n) {
          multiply<DT>(ring[(n0 + 2 * G + n) % kAhead], ds.s[n / N], dq[n % N]);
          read(n0 + 2 * G + n + kAhead);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        f32x16_t x = 0.0f, y = -delta;
#pragma unroll
        for (int e = 0; e < P::kGroups; ++e) multiply<DT>(rd.row(b * P::kBytes, j, e), q.g[e], x);
#pragma unroll
        for (int e = 0; e < P::kGroups; ++e) multiply<DT>(rd.row(kV + b * P::kBytes, j, e), g.g[e], y);
        Packed<DT> ds;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], A.scale2, -lse)) * y[e];
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = sees(j, e) ? x[e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 16; e += 2) ds.set(e / 2, x[e], x[e + 1]);
        multiply_columns<DT, D>(rd, b * P::kBytes, j, ds, dq);
      }
    }
  };
  for (int t = first; t < last; t += 2) {
    step(t, 0);
    if (t + 1 < last) step(t + 1, 1);
  }
  landed();   // panels are free, and no load may reach LDS after the workgroup's end
  common.add(A, lds + w * P::kBytes, s.k0, on, lo, hi, col, dq, sum_of_halves(lost), lane);

  if (pieces > 1) {
    if (!on) return;
    float* const part = A.part + (((int64_t)piece * A.tokens_q + to) * A.heads + h) * kPartLd;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int c = 32 * d + 2 * e + 4 * half;
        if (c < A.dim) store_elems<ISO_F32, 4>(part, c, (const float*)&dq[d] + e);
      }
    return;
  }
  // what is not finite may have met such a value at a key that the row does not see
  const bool bad = on && trouble(dq, A.scale) != 0.0f;
  if (on && !bad) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int c = 32 * d + 2 * e + 4 * half;
        const float v[4] = {dq[d][e] * A.scale, dq[d][e + 1] * A.scale, dq[d][e + 2] * A.scale, dq[d][e + 3] * A.scale};
        if (c < A.dim) store_elems<DT, 4>(A.dq, to * A.ld_dq + (int64_t)h * A.dim + c, v);
      }
  }
  for (uint64_t rest = __ballot(bad); rest != 0;) {
    const int n = __builtin_ctzll(rest) & 31;
    rest &= ~(0x100000001ull << n);
    dq_row<DT>(A, s, head, row0 + 32 * w + n, lane);
  }
}

// dQ from a row's pieces, half a wave a row.
template <int DT>
__device__ __forceinline__ void dq_join(const AttnArgs& A, uint32_t block) {
  constexpr int kRows = 32 * kAttnWaves;
  const int lane = threadIdx.x & 63, c = 4 * (lane & 31);
  const JoinRow j(A, (int64_t)block * 8 + (threadIdx.x >> 5));
  const Span all = j.on ? span_of(A, j.s, j.r / kRows * kRows, min(j.r / kRows * kRows + kRows, j.s.nq * A.group) - 1) : Span{0, 0, 0, 0};
  const int pieces = pieces_of(all, A.pieces);
  const bool on = j.on && pieces > 1;
  float v[4] = {}, t = 0.0f;
  Parts<4> parts(A.part + j.at * kPartLd, A.tokens_q * A.heads * kPartLd, c, on && c < A.dim ? pieces : 0);
  parts.add([](int) { return 1.0f; }, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] *= A.scale, t = fmaf(v[i], 0.0f, t);
  const uint64_t bad = __ballot(t != 0.0f);
  if (on && (uint32_t)(bad >> (lane & 32)) == 0 && c < A.dim) store_elems<DT, 4>(A.dq, j.t * A.ld_dq + (int64_t)j.h * A.dim + c, v);
#pragma unroll 1
  for (int i = 0; i < 2; ++i)
    if ((uint32_t)(bad >> (32 * i)) != 0) {
      const JoinRow row = j.of(32 * i);
      dq_row<DT>(A, row.s, row.h / A.group, row.r, lane);
    }
}

// ---- dK and dV -----------------------------------------------------------------------------------------------------

// Panels of a group's list of rows, of q and of dO.  Offsets within a panel come from the row that it starts at, by its query and
// its place in the group: row / group and what is left.
template <class P>
struct ListRows {
  const uint8_t *q, *g;           // at the first query of the panel
  int64_t q_left, g_left;         // bytes from there on to the end of the last query's
  int32_t q_ld, g_ld, dim, group, rest;
  uint32_t byte[P::kLoads];
  int32_t row[P::kLoads];

  __device__ __forceinline__ ListRows(const AttnArgs& A, const Seq& s, int head, int32_t first, int wave, int lane) {
    const int32_t query = first / A.group;
    group = A.group, rest = first - query * group, dim = A.dim * P::kSize;
    q_ld = (int32_t)A.ld_q * P::kSize, g_ld = (int32_t)A.ld_dout * P::kSize;
    const int64_t col = (int64_t)head * group * dim, left = s.nq - query;
    q = (const uint8_t*)A.q + (s.q0 + query) * q_ld + col;
    g = (const uint8_t*)A.dout + (s.q0 + query) * g_ld + col;
    q_left = left > 0 ? (left - 1) * q_ld + group * dim : 0;
    g_left = left > 0 ? (left - 1) * g_ld + group * dim : 0;
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) {
      int b;
      P::source(j, wave, lane, row[j], b);
      byte[j] = b < dim ? b : kOutside;
    }
  }
  __device__ __forceinline__ void load(uint32_t q_lds, uint32_t g_lds, int wave) {
    const u32x4_t qb = scalar_buffer_of(q, q_left), gb = scalar_buffer_of(g, g_left);
    const uint32_t inverse = ((1u << 21) + group - 1) / group;   // x / group = x inverse / 2^21 for x < group + 32, group <= 1024
    q_lds = __builtin_amdgcn_readfirstlane(q_lds), g_lds = __builtin_amdgcn_readfirstlane(g_lds);
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) {
      const uint32_t x = rest + row[j], query = __umul24(x, inverse) >> 21;
      const uint32_t at = __umul24(x - __umul24(query, group), dim) + byte[j];
      load_lds(qb, q_lds + (j * kAttnWaves + wave) * 1024, at + __umul24(query, q_ld));
      load_lds(gb, g_lds + (j * kAttnWaves + wave) * 1024, at + __umul24(query, g_ld));
    }
    rest += P::kRows % group;
    int32_t queries = P::kRows / group;
    if (rest >= group) rest -= group, ++queries;
    const int64_t dq = (int64_t)queries * q_ld, dg = (int64_t)queries * g_ld;
    q += dq, q_left -= dq, g += dg, g_left -= dg;
  }
};

// Workgroup layout of dkv_tile.  Two waves a SIMD need 256 registers a lane to do: 128 hold the sums, so that bf16 values
// stay in LDS and only keys are kept in registers.  fp32 has one wave a SIMD and both in registers.
template <int DT, int D>
struct Dkv {
  using P = Panel<DT, D, 32>;
  static constexpr bool kValuesInLds = DT == ISO_BF16;
  static constexpr int kWaves = DT == ISO_F32 ? 1 : 2;
  static constexpr uint32_t kG = 2 * P::kBytes, kValues = 4 * P::kBytes, kStat = kValues + (kValuesInLds ? 4 * P::kBytes : 0);   // 32 values a wave
  static constexpr uint32_t kLds = kStat + 512;
};

// dK and dV of a tile of 128 keys, a wave 32 of them: panels of 32 rows of Q and dO in LDS twice over, with their L and D.  Heads of a
// group are rows of one list, so the sum over them is made here.
template <int DT, int D>
__device__ __forceinline__ void dkv_tile(const AttnArgs& A, const Deal& deal, uint32_t block, uint8_t* smem) {
  using S = Dkv<DT, D>;
  using P = typename S::P;
  constexpr int kKeys = 32 * kAttnWaves;
  int head;
  uint32_t item;
  Item it;
  if (!dealt(deal, A.heads_kv, block, head, item) || !find_item<true, kKeys>(A, A.key_pieces, item, it)) return;
  const Seq s = it.s;
  const int piece = it.piece;

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int32_t key0 = (int32_t)it.tile * kKeys, end = min(key0 + kKeys, s.nk);
  const Span all = list_span(A, s, key0, end - 1);
  const int pieces = pieces_of(all, A.key_pieces);
  if (piece >= pieces) return;
  const int tiles = (all.hi - all.lo + P::kRows - 1) / P::kRows;
  const int first = __builtin_amdgcn_readfirstlane((int)((uint32_t)tiles * (uint32_t)piece / (uint32_t)pieces));
  const int last = __builtin_amdgcn_readfirstlane((int)((uint32_t)tiles * (uint32_t)(piece + 1) / (uint32_t)pieces));

  // a lane has one key of its wave's 32, the halves of a wave different rows
  const int32_t key = key0 + 32 * w + (lane & 31);
  const bool on = key < end, busy = key0 + 32 * w < end;
  int32_t lo = 0, hi = 0;
  if (on) {
    queries_of(A, s, key, lo, hi);
    lo *= A.group, hi *= A.group;
  }
  Span mine{0, 0, 0, 0};
  if (busy) mine = list_span(A, s, key0 + 32 * w, min(key0 + 32 * w + 32, end) - 1);
  if (key0 + 32 * w + 32 > end) mine.lo_all = INT32_MAX;

  const int64_t col = (int64_t)head * A.dim, to = s.k0 + key;
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_u8*)smem);
  ListRows<P> list(A, s, head, all.lo + first * P::kRows, w, lane);
  const float* stat = A.stat + list_of(A, s, head) + all.lo + first * P::kRows;
  // of a panel's rows, L in eight lanes' pieces and D in the next eight
  const uint32_t stat_at = lane < 8 ? lane * 16 : lane < 16 ? (uint32_t)(A.tokens_q * A.heads * 4) + (lane - 8) * 16 : kOutside;
  auto load = [&](int b) {   // the next panel, into panels b
    list.load(lds + b * P::kBytes, lds + S::kG + b * P::kBytes, w);
    if (w == 0 && lane < 16) load_lds(scalar_buffer_of((const uint8_t*)stat, 0x80000000ll), lds + S::kStat + b * 256, stat_at);   // 256 bytes
    stat += P::kRows;
  };
  Reader<DT, D> rd(lds, lane);
  OwnRow<DT, D> k, v;
  if constexpr (S::kValuesInLds) {
    Rows<DT, D, P> vr(A.v, s.k0 + key0, A.ld_v, col, end - key0, A.dim, w, lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) vr.load(lds + S::kValues + j * P::kBytes, w);
  } else {
    v.load(A.v, to * A.ld_v + col, A.dim, half, on);
  }
  load(0);
  k.load(A.k, to * A.ld_k + col, A.dim, half, on);
  k.arrive();
  if constexpr (!S::kValuesInLds) v.arrive();
  const Reader<DT, D> own(lds + S::kValues + w * P::kBytes, lane);

  f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dk[d] = 0.0f, dv[d] = 0.0f;

  auto sees = [&](int32_t r0, int e) { return (uint32_t)(r0 + 8 * (e / 4) + 4 * half + e % 4 - lo) < (uint32_t)(hi - lo); };
  uint32_t of = lds + S::kStat + 16 * half;
  constexpr uint32_t qp = 0, gp = S::kG;
  for (int t = first; t < last; ++t) {
    landed();
    load((t - first + 1) & 1);
    const int32_t r0 = all.lo + t * P::kRows;
    if (!busy || r0 >= mine.hi || r0 + P::kRows <= mine.lo) {
      rd.swap(P::kBytes);
      of ^= 256;
      continue;
    }
    const bool whole = r0 >= mine.lo_all && r0 + P::kRows <= mine.hi_all;
    f32x16_t x = 0.0f, y = 0.0f;
    Packed<DT> p, ds;
    rd.again();
    if constexpr (DT == ISO_BF16) {
      // Fragments are read some products ahead, in the order laid out here: S and dP by rows, dV and dK by columns.  Left to
      // itself the compiler reads a whole product's ahead, for which there are no registers.
      constexpr int G = P::kGroups, N = 2 * P::kDims, kAhead = 3, kAll = 2 * G + 2 * N;
      u32x4_t ring[kAhead], vf[2];
      auto read = [&](int n) {
        if (n < G) ring[n % kAhead] = rd.row(qp, 0, n);
        else if (n < 2 * G) ring[n % kAhead] = rd.row(gp, 0, n - G);
        else if (n < 2 * G + N) ring[n % kAhead] = __builtin_bit_cast(u32x4_t, rd.col(gp, 0, (n - 2 * G) / (N / 2), (n - 2 * G) % (N / 2)));
        else if (n < kAll) ring[n % kAhead] = __builtin_bit_cast(u32x4_t, rd.col(qp, 0, (n - 2 * G - N) / (N / 2), (n - 2 * G - N) % (N / 2)));
      };
#pragma unroll
      for (int n = 0; n < kAhead; ++n) read(n);
#pragma unroll
      for (int n = 0; n < G; ++n) {
        multiply<DT>(ring[n % kAhead], k.g[n], x);
        read(n + kAhead);
        if (n >= G - 2) vf[n & 1] = own.row(0, 0, n - (G - 2));
        __builtin_amdgcn_sched_barrier(0);
      }
      f32x4_t lse = *(lds_f32x4)(uintptr_t)of;
#pragma unroll
      for (int n = 0; n < G; ++n) {
        multiply<DT>(ring[(G + n) % kAhead], vf[n & 1], y);
        read(G + n + kAhead);
        if (n + 2 < G) vf[n & 1] = own.row(0, 0, n + 2);
#pragma unroll
        for (int e = 16 / G * n; e < 16 / G * (n + 1); ++e) {
          x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], A.scale2, -lse[e % 4]));
          if (e % 4 == 3 && e < 15) lse = *(lds_f32x4)(uintptr_t)(of + 8 * (e + 1));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x4_t delta = *(lds_f32x4)(uintptr_t)(of + 128 + 8 * e);
#pragma unroll
        for (int c = 0; c < 4; ++c) y[e + c] = x[e + c] * (y[e + c] - delta[c]);
      }
      if (!whole) {   // of both: 0 times what is not seen may be NaN
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool on = sees(r0, e);
          x[e] = on ? x[e] : 0.0f, y[e] = on ? y[e] : 0.0f;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        p.set(e / 2, x[e], x[e + 1]), p.set(e / 2 + 1, x[e + 2], x[e + 3]);
        ds.set(e / 2, y[e], y[e + 1]), ds.set(e / 2 + 1, y[e + 2], y[e + 3]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        multiply<DT>(ring[(2 * G + n) % kAhead], p.s[n / (N / 2)], dv[n % (N / 2)]);
        read(2 * G + n + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
        multiply<DT>(ring[(2 * G + N + n) % kAhead], ds.s[n / (N / 2)], dk[n % (N / 2)]);
        read(2 * G + N + n + kAhead);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int e = 0; e < P::kGroups; ++e) multiply<DT>(rd.row(qp, 0, e), k.g[e], x);
#pragma unroll
      for (int e = 0; e < P::kGroups; ++e) multiply<DT>(rd.row(gp, 0, e), v.g[e], y);
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x4_t lse = *(lds_f32x4)(uintptr_t)(of + 8 * e), delta = *(lds_f32x4)(uintptr_t)(of + 128 + 8 * e);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          x[e + c] = __builtin_amdgcn_exp2f(fmaf(x[e + c], A.scale2, -lse[c]));
          y[e + c] = x[e + c] * (y[e + c] - delta[c]);
          if (!whole && !sees(r0, e + c)) x[e + c] = 0.0f, y[e + c] = 0.0f;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; e += 2) p.set(e / 2, x[e], x[e + 1]), ds.set(e / 2, y[e], y[e + 1]);
      multiply_columns<DT, D>(rd, gp, 0, p, dv);
      multiply_columns<DT, D>(rd, qp, 0, ds, dk);
    }
    rd.swap(P::kBytes);
    of ^= 256;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load may reach LDS after the workgroup's end

  if (pieces > 1) {
    if (!on) return;
    float* const part = A.key_part + (((int64_t)piece * A.tokens_k + to) * A.heads_kv + head) * (2 * kPartLd);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int c = 32 * d + 2 * e + 4 * half;
        if (c >= A.dim) continue;
        store_elems<ISO_F32, 4>(part, c, (const float*)&dk[d] + e);
        store_elems<ISO_F32, 4>(part, kPartLd + c, (const float*)&dv[d] + e);
      }
    return;
  }
  const bool bad = on && fmaf(trouble(dk, A.scale), 1.0f, trouble(dv, 1.0f)) != 0.0f;
  if (on && !bad) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int c = 32 * d + 2 * e + 4 * half;
        if (c >= A.dim) continue;
        const float x[4] = {dk[d][e] * A.scale, dk[d][e + 1] * A.scale, dk[d][e + 2] * A.scale, dk[d][e + 3] * A.scale};
        store_elems<DT, 4>(A.dk, to * A.ld_dk + col + c, x);
        store_elems<DT, 4>(A.dv, to * A.ld_dv + col + c, (const float*)&dv[d] + e);
      }
  }
  for (uint64_t rest = __ballot(bad); rest != 0;) {
    const int n = __builtin_ctzll(rest) & 31;
    rest &= ~(0x100000001ull << n);
    dkv_row<DT>(A, s, head, key0 + 32 * w + n, lane);
  }
}

// Adds up the pieces of a key, a wave a key and kv head: dK in its first half, dV in its second.
template <int DT>
__device__ __forceinline__ void dkv_join(const AttnArgs& A, uint32_t block) {
  constexpr int kKeys = 32 * kAttnWaves;
  const int64_t at = (int64_t)block * 4 + (threadIdx.x >> 6), t = at / A.heads_kv;
  if (t >= A.tokens_k) return;
  const Seq s = seq_at<true>(A, t);
  if (t < s.k0 || t >= s.k0 + s.nk) return;
  const int head = (int)(at - t * A.heads_kv), lane = threadIdx.x & 63, c = 4 * (lane & 31);
  const int32_t key = (int32_t)(t - s.k0), key0 = key / kKeys * kKeys;
  const int pieces = pieces_of(list_span(A, s, key0, min(key0 + kKeys, s.nk) - 1), A.key_pieces);
  if (pieces == 1) return;
  const bool values = lane >= 32;
  float v[4] = {}, bad = 0.0f;
  Parts<4> parts(A.key_part + at * (2 * kPartLd) + (values ? kPartLd : 0), A.tokens_k * A.heads_kv * (2 * kPartLd), c, c < A.dim ? pieces : 0);
  parts.add([](int) { return 1.0f; }, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!values) v[i] *= A.scale;
    bad = fmaf(v[i], 0.0f, bad);
  }
  if (__any(bad != 0.0f)) return dkv_row<DT>(A, s, head, key, lane);
  if (c >= A.dim) return;
  if (values) store_elems<DT, 4>(A.dv, t * A.ld_dv + (int64_t)head * A.dim + c, v);
  else store_elems<DT, 4>(A.dk, t * A.ld_dk + (int64_t)head * A.dim + c, v);
}

// ---- both ----------------------------------------------------------------------------------------------------------

// Workgroups up to `keys` have keys, the others rows: in one launch, where the ones' last round leaves room for the others.
template <int DT, int D>
__global__ void __launch_bounds__(256, (Dkv<DT, D>::kWaves)) k_attend_grad(AttnArgs A, Deal dkv, Deal dq, uint32_t keys) {
  extern __shared__ __attribute__((aligned(32768))) uint8_t smem[];   // panels in turn are one bit of an address apart
  if (blockIdx.x < keys) dkv_tile<DT, D>(A, dkv, blockIdx.x, smem);
  else dq_tile<DT, D>(A, dq, blockIdx.x - keys, smem);
}

template <int DT>
__global__ void __launch_bounds__(256) k_attend_grad_join(AttnArgs A, uint32_t keys) {
  if (blockIdx.x < keys) dkv_join<DT>(A, blockIdx.x);
  else dq_join<DT>(A, blockIdx.x - keys);
}

template <int DT, int D>
hipError_t backward(AttnArgs A, const AttendPlan& plan, uint8_t* ws, hipStream_t s) {
  const int64_t rows = A.tokens_q * A.heads, keys = A.tokens_k * A.heads_kv, list = A.tokens_q * A.group;
  A.stat = (float*)(ws + kStatusBytes);
  A.pieces = plan.rows, A.part = (float*)(ws + plan.part);
  A.key_pieces = plan.keys, A.key_part = (float*)(ws + plan.key_part);
  k_attend_stat<DT><<<(unsigned)((rows + 15) / 16) + 1, 256, 0, s>>>(A);   // one looks at the offsets
  const Deal dkv = deal_of(A.heads_kv, attend_items(A.tokens_k, list, A.sequences, A.key_pieces));
  const Deal dq = deal_of(A.heads_kv, attend_items(list, A.tokens_k, A.sequences, A.pieces));
  const uint32_t of_keys = keys > 0 ? deal_grid(dkv, A.heads_kv) : 0, of_rows = rows > 0 ? deal_grid(dq, A.heads_kv) : 0;
  constexpr uint32_t lds = std::max(Dq<DT, D>::kLds, Dkv<DT, D>::kLds);
  if (of_keys + of_rows > 0) k_attend_grad<DT, D><<<of_keys + of_rows, 256, lds, s>>>(A, dkv, dq, of_keys);
  const uint32_t join_keys = A.key_pieces.most > 1 ? (uint32_t)((keys + 3) / 4) : 0, join_rows = A.pieces.most > 1 ? (uint32_t)((rows + 7) / 8) : 0;
  if (join_keys + join_rows > 0) k_attend_grad_join<DT><<<join_keys + join_rows, 256, 0, s>>>(A, join_keys);
  return hipGetLastError();
}

template <int DT>
hipError_t backward(const AttnArgs& A, const AttendPlan& plan, uint8_t* ws, hipStream_t s) {
  return A.dim > 64 ? backward<DT, 128>(A, plan, ws, s) : backward<DT, 64>(A, plan, ws, s);
}

}  // namespace

hipError_t run_attend_grad(const iso_attn& a, int dt, uint8_t* ws, hipStream_t s) {
  const AttnArgs A = args_of(a, ws);
  const AttendPlan plan = plan_attend(a, true);
  return dt == ISO_BF16 ? backward<ISO_BF16>(A, plan, ws, s) : backward<ISO_F32>(A, plan, ws, s);
}

}  // namespace iso
