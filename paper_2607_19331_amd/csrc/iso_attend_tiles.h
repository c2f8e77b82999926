// Tiles of the attention kernels: panels of token rows in LDS, fragments of them for matrix instructions.
//
// All products have 32 x 32 results.  A result has one column a lane (lane % 32) and in register r row 8 (r / 4) + 4 half + r % 4,
// half = lane / 32.  Scores are formed with the summed-over index of the next product as rows: that product then takes them from
// the registers where they are.  Which 8 (bf16) values of the summed index a lane holds for one instruction is free as long as
// both operands agree, so the other operand is read from LDS in the order that the result has.
#pragma once

#include <algorithm>

#include "iso_attend.h"
#include "iso_mfma.h"

namespace iso {

constexpr int kAttnWaves = 4;

// Panels of kRows token rows of D dimensions (head dimensions up to D, the rest zero); a row's 16-byte pieces are
// permuted (piece p at p ^ mix(row)), so that 16 successive rows have the same piece in different banks, and so have four
// successive rows 64 bytes next to each other (bf16) or two rows four apart 128 bytes (fp32).
template <int DT, int D, int ROWS = DT == ISO_BF16 ? 64 : 32>
struct Panel {
  static constexpr int kSize = DT == ISO_BF16 ? 2 : 4;
  static constexpr int kRowBytes = D * kSize;
  static constexpr int kPieces = kRowBytes / 16;
  static constexpr int kRows = ROWS;
  static constexpr int kBytes = kRows * kRowBytes;
  static constexpr int kLoads = kBytes / (1024 * kAttnWaves);   // 16-byte loads a lane
  static constexpr int kTiles = kRows / 32;                     // 32-row tiles
  static constexpr int kGroups = kRowBytes / 32;                // 32-byte groups of a row: 16 bytes for either half of a wave
  static constexpr int kDims = D / 32;                          // 32-dimension tiles

  __device__ static __forceinline__ int mix(int row) {
    if constexpr (DT == ISO_F32) return (row & 3) | ((row >> 3) & 1) << 2 | ((row >> 2) & 1) << 3;
    else if constexpr (D == 128) return (row & 3) << 2 | ((row >> 2) & 3);
    else return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
  }

  // Of load j of a wave: the panel's row and the byte of the row that a lane takes from memory.
  __device__ static __forceinline__ void source(int j, int wave, int lane, int& row, int& byte) {
    const int at = (j * kAttnWaves + wave) * 64 + lane;
    row = at / kPieces;
    byte = ((at % kPieces) ^ mix(row)) * 16;
  }
};

constexpr uint32_t kOutside = 0xC0000000u;   // an offset behind the end of every buffer

// One operand's rows in memory, loaded panel by panel: a kv head's from some row on, `rows` of them.
template <int DT, int D, class PANEL = Panel<DT, D>>
struct Rows {
  using P = PANEL;
  const uint8_t* at;
  int64_t step, left;   // bytes of a panel's rows, and from `at` on to the end of the last row
  uint32_t offset[P::kLoads];

  __device__ __forceinline__ Rows(const void* p, int64_t first, int64_t ld, int64_t col, int64_t rows, int dim, int wave, int lane) {
    at = (const uint8_t*)p + (first * ld + col) * P::kSize;
    step = P::kRows * ld * P::kSize;
    left = rows > 0 ? ((rows - 1) * ld + dim) * P::kSize : 0;
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) {
      int row, byte;
      P::source(j, wave, lane, row, byte);
      offset[j] = byte < dim * P::kSize ? (uint32_t)(row * (int)ld * P::kSize + byte) : kOutside;
    }
  }
  __device__ __forceinline__ void skip(int64_t panels) { at += panels * step, left -= panels * step; }
  // The next panel into LDS; behind the last row, zeros.
  __device__ __forceinline__ void load(uint32_t lds, int wave) {
    const u32x4_t b = scalar_buffer_of(at, left);
    lds = __builtin_amdgcn_readfirstlane(lds);
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) load_lds(b, lds + (j * kAttnWaves + wave) * 1024, offset[j]);
    at += step, left -= step;
  }
};

typedef __attribute__((address_space(3))) const u32x4_t* lds_piece;
typedef __attribute__((address_space(3))) const float* lds_float;
typedef __attribute__((address_space(3))) uint32_t* lds_word;

// Where a lane reads fragments of panels: rows, 16 bytes a group, for products that sum over dimensions; and columns, for those
// that sum over rows.  Groups, 32-dimension tiles and rows are bits of the permuted piece, so one exclusive or makes each address
// from the lane's first, and which panel it is goes into the instruction.
template <int DT, int D>
struct Reader {
  using P = Panel<DT, D>;
  uint32_t row0, col0;

  __device__ __forceinline__ Reader(uint32_t lds, int lane) {
    const int r = lane & 31, half = lane >> 5, i = lane & 15, g = lane >> 4;
    row0 = lds + r * P::kRowBytes + (P::mix(r) ^ half) * 16;
    if constexpr (DT == ISO_BF16) {
      // 16 lanes read a block of four rows by 16 columns and get a column each
      const int row = 4 * (g >> 1) + (i >> 2), byte = (g & 1) * 32 + (i & 3) * 8;
      col0 = lds + row * P::kRowBytes + ((byte / 16) ^ P::mix(row)) * 16 + byte % 16;
    } else {
      const int row = 4 * half;
      col0 = lds + row * P::kRowBytes + ((r / 4) ^ P::mix(row)) * 16 + (r % 4) * 4;
    }
  }
  // Addresses are worked out where they are used: kept from one tile to the next they would take sixteen registers.
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(row0), "+v"(col0)); }
  // Over to the panel `bytes` (a power of two) on, or back.
  __device__ __forceinline__ void swap(uint32_t bytes) { row0 ^= bytes, col0 ^= bytes; }
  // 16 bytes of group g of the lane's row of tile t of the panel `panel` bytes on.
  __device__ __forceinline__ u32x4_t row(uint32_t panel, int t, int g) const {
    return *(lds_piece)(uintptr_t)((row0 ^ (32 * g)) + (panel + t * 32 * P::kRowBytes));
  }
  // bf16: dimensions 32 d + lane % 32 of rows 16 s + 4 half + {0..3, 8..11} of tile t.
  __device__ __forceinline__ bf16x8_t col(uint32_t panel, int t, int s, int d) const {
    struct {
      s16x4_t h[2];
    } f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t at = (col0 ^ (64 * d ^ (h ? P::mix(8) * 16 : 0))) + (panel + (t * 32 + 16 * s + 8 * h) * P::kRowBytes);
      f.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_frag)(uintptr_t)at);
    }
    return __builtin_bit_cast(bf16x8_t, f);
  }
  // fp32: dimension 32 d + lane % 32 of row 8 g + 4 half + e of tile t.
  __device__ __forceinline__ float one(uint32_t panel, int t, int g, int e, int d) const {
    const uint32_t x = (uint32_t)(P::mix((8 * g) & 15) ^ P::mix(e)) * 16 ^ 128 * d;
    return *(lds_float)(uintptr_t)((col0 ^ x) + (panel + (t * 32 + 8 * g + e) * P::kRowBytes));
  }
};

// acc += A B over one group of 16 (bf16) or 8 (fp32) dimensions; of these, half of a wave holds 8 or 4 in order.
template <int DT>
__device__ __forceinline__ void multiply(u32x4_t a, u32x4_t b, f32x16_t& acc) {
  if constexpr (DT == ISO_BF16) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(f32_from_bits(a[e]), f32_from_bits(b[e]), acc, 0, 0, 0);
  }
}

// A lane's row (a query's, say) as second operand: all groups, in registers.
template <int DT, int D>
struct OwnRow {
  u32x4_t g[Panel<DT, D>::kGroups];
  // From element `at` on, dim of them; zeros where !on.
  __device__ __forceinline__ void load(const void* p, int64_t at, int dim, int half, bool on) {
    constexpr int V = 16 / Panel<DT, D>::kSize;
#pragma unroll
    for (int i = 0; i < Panel<DT, D>::kGroups; ++i) {
      const int c = (2 * i + half) * V;
      g[i] = u32x4_t{0, 0, 0, 0};
      if (on && c < dim) g[i] = load_raw<DT>(p, at + c);
    }
  }
  // The loads have come back.  Before a loop that loads into LDS: the first use, if it were in there, would wait for those too,
  // each time round.
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int i = 0; i < Panel<DT, D>::kGroups; ++i) asm volatile("" : "+v"(g[i]));
  }
};

// Results as second operand of a product that sums over their rows, in the type of the call.
template <int DT>
struct Packed;
template <>
struct Packed<ISO_BF16> {
  u32x4_t s[2];
  __device__ __forceinline__ void set(int i, float lo, float hi) { s[i / 4][i % 4] = pack_bf16(lo, hi); }   // registers 2i, 2i + 1
};
template <>
struct Packed<ISO_F32> {
  float v[16];
  __device__ __forceinline__ void set(int i, float lo, float hi) { v[2 * i] = lo, v[2 * i + 1] = hi; }
};

// acc[d] += (columns 32 d ... of tile t of a panel)^T x, summed over the tile's 32 rows.
template <int DT, int D>
__device__ __forceinline__ void multiply_columns(const Reader<DT, D>& r, uint32_t panel, int t, const Packed<DT>& x,
                                                 f32x16_t (&acc)[D / 32]) {
  if constexpr (DT == ISO_BF16) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.col(panel, t, s, d), __builtin_bit_cast(bf16x8_t, x.s[s]), acc[d], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(r.one(panel, t, i / 4, i % 4, d), x.v[i], acc[d], 0, 0, 0);
  }
}

// All loads into LDS have landed and all LDS reads are done, of every wave.
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A value and that of the lane with the same column in the other half.
__device__ __forceinline__ float both_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(bits_from_f32(v), bits_from_f32(v), false, false);
  return fmaxf(f32_from_bits(r[0]), f32_from_bits(r[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(bits_from_f32(v), bits_from_f32(v), false, false);
  return f32_from_bits(r[0]) + f32_from_bits(r[1]);
}

// ---- which tile a workgroup has ------------------------------------------------------------------------------------

// Work is a list of items for every kv head: tiles of rows (or keys), the keys (rows) that a tile walks over shared out to the
// pieces of its sequence.  Workgroup b runs on XCD b % 8: heads are dealt to as many classes of XCDs as divide them evenly, so
// that a head's keys and values are read through few L2 caches, and a class takes the items of a head, its XCDs in turn.
struct Deal {
  int32_t classes, per;   // classes of XCDs, XCDs of a class
  uint32_t items;         // of a head, or an upper bound
  uint32_t fold, end;     // places [fold, end) of a class are taken from the end, and heads in turn; 0: neither
};

inline Deal deal_of(int heads, uint32_t items) {
  int c = 8;
  while (heads % c != 0) c /= 2;
  return Deal{c, 8 / c, items, 0, 0};
}
// Items of falling length that all start at once, counted as two a CU (bf16 heads up to 64 run three): the second half from its end on, so
// that the shortest go with the longest.  `tiles`: about how many there are.  Four sequences of 2048, causal, 8 heads of 64, fp32:
// 161 us for 206; 2048 tokens, 32 heads of 128, bf16: 53 for 63.
inline Deal folded(Deal d, int heads, int64_t tiles) {
  const uint32_t cus = 32 * d.per, all = (uint32_t)(heads / d.classes) * d.items;   // CUs of a class
  if (all > cus && tiles <= 2 * (int64_t)cus * d.classes) d.fold = cus, d.end = std::min(all, 2 * cus);
  return d;
}
inline uint32_t deal_grid(const Deal& d, int heads) {
  const uint64_t n = (uint64_t)(heads / d.classes) * d.items;
  return (uint32_t)((n + d.per - 1) / d.per * 8);
}
__device__ __forceinline__ bool dealt(const Deal& d, int heads, uint32_t b, int& head, uint32_t& item) {
  const uint32_t x = b & 7u, c = x % d.classes, each = (uint32_t)(heads / d.classes);
  uint32_t j = (b >> 3) * d.per + x / d.classes, h;
  if (j >= each * d.items) return false;
  if (d.fold > 0) {
    if (j >= d.fold && j < d.end) j = d.fold + d.end - 1 - j;
    item = j / each, h = j - item * each;
  } else {
    h = j / d.items, item = j - h * d.items;
  }
  head = (int)(c + d.classes * h);
  return true;
}

// A tile of a sequence and a piece of it.
struct Item {
  Seq s;
  uint32_t tile;
  int32_t piece;
};

// Sequences that a wave looks at, a lane each, where some offsets do not ascend: those that begin before the end of an earlier range get
// no rows.  `taken`: by the sequences before these, and then by these too.
__device__ __forceinline__ void only_free(Seq& mine, bool range, Taken& taken) {
  const int lane = threadIdx.x & 63;
  Taken up_to;   // this lane
  if (range) up_to.add(mine);
#pragma unroll 1
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t q = __shfl_up(up_to.q, d), k = __shfl_up(up_to.k, d);
    if (lane >= d) up_to.q = max(up_to.q, q), up_to.k = max(up_to.k, k);
  }
  Taken before{__shfl_up(up_to.q, 1), __shfl_up(up_to.k, 1)};
  if (lane == 0) before = Taken{};
  before.q = max(before.q, taken.q), before.k = max(before.k, taken.k);
  if (!range || !before.free(mine)) mine = Seq{0, 0, 0, 0};
  taken = Taken{max(taken.q, __shfl(up_to.q, 63)), max(taken.k, __shfl(up_to.k, 63))};
}

// Item `item` of the list of all sequences' items, tiles of TILE rows (queries times the group) or of keys, those that have most to do
// under a causal mask first.  Up to 64 sequences are taken level by level (tiles that have as many before them, or behind them for
// keys), so that the last workgroups to start are short whichever sequences are long; more are taken one after the other, a workgroup
// looking no further than its own.  Level by level and one after the other, four sequences of 2048, 8 heads, fp32: 314 and 497 us; 12
// heads over 2, bf16: 72 and 85, backward 231 and 245; 16 samples of 1 to 2048 tokens, backward 284 and 305; 64 sequences of one new
// token (whose levels are not searched) 121 and 120.  Every lane of a wave takes part, each with a sequence.
template <bool KEYS, int TILE>
__device__ __forceinline__ bool find_item(const AttnArgs& A, const Pieces& p, uint32_t item, Item& found) {
  const int lane = threadIdx.x & 63;
  Seq mine;
  uint32_t tiles, pieces;
  bool ascend = true;   // all offsets so far
  Taken taken;          // by the sequences so far, if not
  auto look = [&](int32_t s0) {
    mine = Seq{0, 0, 0, 0};
    bool range = true;
    if (s0 + lane < A.sequences) range = seq_of(A, s0 + lane, mine);
    if (__any(!range) || !ascend) {
      if (ascend && s0 > 0) taken = Taken{gmem(A.start_q)[s0], gmem(A.start_k)[s0]};
      ascend = false;
      only_free(mine, range && s0 + lane < A.sequences, taken);
    }
    const uint32_t rows = (uint32_t)mine.nq * (uint32_t)A.group, keys = (uint32_t)mine.nk;
    tiles = ((KEYS ? keys : rows) + TILE - 1) / TILE;
    pieces = min((uint32_t)p.most, max(1u, ((KEYS ? rows : keys) + p.keys - 1) / p.keys));
  };
  auto up_to = [&](uint32_t sum) {   // sum of the lanes up to one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    return sum;
  };
  // what is the same in every lane is said to be so: the code behind then branches for the whole wave
  auto of = [](auto v, int src) { return (decltype(v))__builtin_amdgcn_readlane((int32_t)v, src); };
  auto take = [&](int src) { found.s = Seq{of(mine.q0, src), of(mine.k0, src), of(mine.nq, src), of(mine.nk, src)}; };
  if (A.sequences <= 64) {
    look(0);
    // the last level that has the item on it or a level behind: a lane a level, in steps of 64 levels and then of one
    uint32_t level = 0, step = 1, items = 0;
    while (__any(tiles > 64 * step)) step *= 64;
    const bool one = !__any(tiles > 1);
    const uint32_t both = tiles * 64 + pieces - 1;   // up to 2^18 tiles, up to 64 pieces
    for (; !one; step /= 64) {
      const uint32_t at = level + step * (uint32_t)lane;
      uint32_t from = 0;   // items on the level and those behind it
      for (int32_t s = 0; s < A.sequences; ++s) {
        const uint32_t x = of(both, s);
        from += __umul24(__builtin_elementwise_sub_sat(x / 64, at), x % 64 + 1);
      }
      const uint64_t behind = __ballot(from > item);
      if (behind == 0) return false;
      const int k = 63 - __builtin_clzll(behind);
      level += step * (uint32_t)k;
      items = of(from, k);
      if (step == 1) break;
    }
    const uint32_t sum = up_to(tiles > level ? pieces : 0), in = one ? item : item - (items - of(sum, 63));
    if (in >= of(sum, 63)) return false;
    const int src = __builtin_ctzll(__ballot(sum > in));
    take(src);
    found.tile = KEYS ? of(tiles, src) - 1 - level : level;
    found.piece = (int32_t)(in - (of(sum, src) - of(pieces, src)));
    return true;
  }
  uint32_t before = 0;
  for (int32_t s0 = 0; s0 < A.sequences; s0 += 64) {
    look(s0);
    const uint32_t sum = up_to(tiles * pieces);
    const uint64_t behind = __ballot(before + sum > item);
    if (behind != 0) {
      const int src = __builtin_ctzll(behind);
      const uint32_t in = item - before - of(sum - tiles * pieces, src), tile = in / of(pieces, src);
      take(src);
      found.tile = KEYS ? tile : of(tiles, src) - 1 - tile;
      found.piece = (int32_t)(in - tile * of(pieces, src));
      return true;
    }
    before += of(sum, 63);
  }
  return false;
}

// The sequence that holds row t of q (of k: KEYS); one without rows where there is none.  For the joins, whose sequences are fewer than
// a thousand (there are no pieces where tiles are many) and whose call has looked at its offsets: where they do not ascend, the
// sequences are gone through as find_item does.
template <bool KEYS>
__device__ __forceinline__ Seq seq_among(const AttnArgs& A, int64_t t) {
  Taken taken;
  for (int32_t i = 0; i < A.sequences; ++i) {
    Seq s;
    if (!seq_of(A, i, s)) continue;
    const bool free = taken.free(s);
    taken.add(s);
    if (free && (KEYS ? t >= s.k0 && t < s.k0 + s.nk : t >= s.q0 && t < s.q0 + s.nq)) return s;
  }
  return Seq{};
}

template <bool KEYS>
__device__ __forceinline__ Seq seq_at(const AttnArgs& A, int64_t t) {
  if (A.sequences == 0) return Seq{};
  const auto start = gmem(KEYS ? A.start_k : A.start_q);
  const uint32_t status = *gmem((const uint32_t*)A.status);
  int32_t lo = 0, hi = A.sequences - 1;
  while (lo < hi) {   // the first sequence that ends behind t
    const int32_t m = (lo + hi) / 2;
    if (start[m + 1] > t) hi = m;
    else lo = m + 1;
  }
  return status == 0 ? seq_of(A, lo) : seq_among<KEYS>(A, t);
}

// The same where half a wave asks for one row of q: up to 64 sequences are looked at at once.
__device__ __forceinline__ Seq seq_at_half(const AttnArgs& A, int64_t t) {
  if (A.sequences > 64) return seq_at<false>(A, t);
  const int lane = threadIdx.x & 31, side = threadIdx.x & 32;
  const uint32_t status = *gmem((const uint32_t*)A.status);
  uint64_t ends = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool behind = lane + 32 * i < A.sequences && gmem(A.start_q)[lane + 32 * i + 1] > t;
    ends |= (__ballot(behind) >> side & 0xFFFFFFFFull) << (32 * i);
  }
  if (status != 0) return seq_among<false>(A, t);
  return ends != 0 ? seq_of(A, __builtin_ctzll(ends)) : Seq{};
}

// Keys that the rows of a tile (or of a wave of it) see between them, and those that all of them see.
struct Span {
  int32_t lo, hi, lo_all, hi_all;
};
// Bounds grow with the query, so those of the first and last row do for all.
__device__ __forceinline__ Span span_of(const AttnArgs& A, const Seq& s, int32_t first, int32_t last) {
  Span x;
  keys_of(A, s, (uint32_t)first / (uint32_t)A.group, x.lo, x.hi_all);
  keys_of(A, s, (uint32_t)last / (uint32_t)A.group, x.lo_all, x.hi);
  return x;
}

// The same of the rows of a group's list that see the keys of a tile.
__device__ __forceinline__ Span list_span(const AttnArgs& A, const Seq& s, int32_t first, int32_t last) {
  Span x;
  queries_of(A, s, first, x.lo, x.hi_all);
  queries_of(A, s, last, x.lo_all, x.hi);
  return Span{x.lo * A.group, x.hi * A.group, x.lo_all * A.group, x.hi_all * A.group};
}

// Pieces that the keys (or rows) [lo, hi) of a tile are shared out to.
__device__ __forceinline__ int pieces_of(const Span& x, const Pieces& p) {
  return min(p.most, max(1, (int32_t)((uint32_t)(x.hi - x.lo + p.keys - 1) / (uint32_t)p.keys)));
}

// A row (of tokens_q x heads) whose pieces half a wave adds up.
struct JoinRow {
  int64_t at, t;
  Seq s;
  int32_t h, r;   // head, and row of its group's list
  bool on;
  __device__ __forceinline__ JoinRow(const AttnArgs& A, int64_t at_) : at(at_), t(at_ / A.heads), s(), h(0), r(0), on(t < A.tokens_q) {
    if (on) s = seq_at_half(A, t);
    on = on && t >= s.q0 && t < s.q0 + s.nq;
    h = (int32_t)(at - t * A.heads);
    if (on) r = (int32_t)(t - s.q0) * A.group + h % A.group;
  }
  // That of the half with lane `src`, for the whole wave.
  __device__ __forceinline__ JoinRow of(int src) const {
    JoinRow x = *this;
    x.at = __shfl(at, src), x.t = __shfl(t, src), x.h = __shfl(h, src), x.r = __shfl(r, src);
    x.s.q0 = __shfl(s.q0, src), x.s.k0 = __shfl(s.k0, src), x.s.nq = __shfl(s.nq, src), x.s.nk = __shfl(s.nk, src);
    return x;
  }
};

// sum[0..3] += weight(p) part[p next + c + 0..3] over the pieces, U of them under way at once: the first from the start.
template <int U>
struct Parts {
  const __attribute__((address_space(1))) float* part;
  int64_t next;
  int pieces;
  f32x4_t v[U];

  __device__ __forceinline__ void load(int p0) {
#pragma unroll
    for (int p = 0; p < U; ++p) {
      v[p] = 0.0f;
      if (p0 + p < pieces) v[p] = *(global_ptr<const f32x4_t>)(part + (p0 + p) * next);
    }
  }
  __device__ __forceinline__ Parts(const float* at, int64_t next_, int c, int pieces_) : part(gmem(at) + c), next(next_), pieces(pieces_) { load(0); }
  template <class W>
  __device__ __forceinline__ void add(W weight, float* sum) {
    for (int p0 = 0; __any(p0 < pieces); p0 += U) {
      if (p0 > 0) load(p0);
#pragma unroll
      for (int p = 0; p < U; ++p) {
        const float w = weight(p0 + p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p0 + p < pieces) sum[i] = fmaf(v[p][i], w, sum[i]);
      }
    }
  }
};

// Whether the values of a wave hold a NaN or an infinity: 0 times such a value is NaN, and a sum with one stays one.
template <int N>
__device__ __forceinline__ float trouble(const f32x16_t (&v)[N], float f) {
  float t = 0.0f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(v[d][r] * f, 0.0f, t);
  return t;
}

}  // namespace iso
