// Embedding lookup with scaling and its gradient by sorted tokens.
//
//   x_i = round(scale W[id_i])          G[v] = round([G[v] +] scale sum_{i: id_i = v} dX_i)
//
// Both move rows of dim elements and compute almost nothing: their floor is the bytes of the rows.  The gradient's
// sum over a token's occurrences needs them gathered: the tokens are sorted by id (stable, so that a row's sum runs in
// token order and is the same in every run), and a wave sums one row's occurrences in registers and writes it once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "iso.h"
#include "iso_device.h"
#include "iso_grad.h"
#include "iso_grad_device.h"
#include "iso_kernels.h"

namespace iso {

namespace {

// Workgroups of a launch over `n` pieces of work, which the kernels walk in strides of the grid (a launch holds fewer
// than 2^32 threads).
unsigned grid_for(int64_t n) { return (unsigned)std::min<int64_t>(std::max<int64_t>(n, 1), 1 << 22); }

struct Ids {
  const void* p;
  int32_t wide;        // 64-bit ids
  int32_t pad_on;
  int64_t pad, vocab;
};

// id of token t as a row of the table; -1 at padding, -2 outside the vocabulary.
__device__ __forceinline__ int32_t row_of(const Ids& ids, int64_t t) {
  const int64_t v = ids.wide ? gmem((const int64_t*)ids.p)[t] : (int64_t)gmem((const int32_t*)ids.p)[t];
  if (ids.pad_on && v == ids.pad) return -1;
  return (v >= 0 && v < ids.vocab) ? (int32_t)v : -2;
}

// ---- lookup --------------------------------------------------------------------------------------------------------

constexpr int kLookupItems = 2;   // 16-byte vectors a thread (28 us; one, four and eight: 30 for 16384 tokens of 3584)
constexpr int kLookupBlock = 256 * kLookupItems;

// With `alone` (lookup_checks_alone) workgroup 0 looks at every id and writes the status word, so that the call is one launch:
// nothing has to be cleared before the others find a bad id.  Else a launch before clears the word and it does nothing.  The
// others copy 512 vectors each, numbered through tokens and columns: a thread's ids, and then its vectors, are in flight together.
template <int DT, bool STREAM>
__global__ void __launch_bounds__(256) k_embed_lookup(Ids ids, const void* __restrict__ table, void* __restrict__ x,
                                                      int64_t tokens, int64_t dim, int64_t ld_x, float scale,
                                                      bool alone, uint32_t* status) {
  if (blockIdx.x == 0) {
    if (!alone) return;
    __shared__ int any;
    if (threadIdx.x == 0) any = 0;
    __syncthreads();
    bool bad = false;
    for (int64_t t = threadIdx.x; t < tokens; t += 256) bad |= row_of(ids, t) == -2;
    if (bad) any = 1;
    __syncthreads();
    if (threadIdx.x == 0) *status = any ? kStatusIndex : 0u;
    return;
  }
  constexpr int V = kVec<DT>;
  const uint32_t per_row = (uint32_t)((dim + V - 1) / V);
  const int64_t items = tokens * per_row, step = (int64_t)(gridDim.x - 1) * kLookupBlock;
  for (int64_t base = (int64_t)(blockIdx.x - 1) * kLookupBlock; base < items; base += step) {
    const int64_t t0 = base / per_row;
    const uint32_t c0 = (uint32_t)(base - t0 * per_row);
    int64_t tok[kLookupItems], col[kLookupItems];
    int32_t row[kLookupItems];
#pragma unroll
    for (int q = 0; q < kLookupItems; ++q) {
      const uint32_t r = c0 + q * 256 + threadIdx.x, d = r / per_row;
      tok[q] = t0 + d;
      col[q] = (int64_t)(r - d * per_row) * V;
      row[q] = tok[q] < tokens ? row_of(ids, tok[q]) : -1;
      if (row[q] == -2 && !alone) flag_status(status, kStatusIndex);
    }
    u32x4_t w[kLookupItems];
#pragma unroll
    for (int q = 0; q < kLookupItems; ++q) {
      w[q] = u32x4_t{0, 0, 0, 0};
      if (row[q] >= 0) w[q] = load_raw<DT>(table, row[q] * dim + col[q], dim - col[q]);
    }
#pragma unroll
    for (int q = 0; q < kLookupItems; ++q) {
      if (tok[q] >= tokens) continue;
      float v[V];
      unpack_raw<DT>(w[q], v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = row[q] >= 0 ? v[j] * scale : 0.0f;
      store_elems<DT, V, STREAM>(x, tok[q] * ld_x + col[q], v, dim - col[q]);
    }
  }
}

// ---- gradient: shared pieces ---------------------------------------------------------------------------------------

// Lanes of the wave whose key equals this lane's (of those with `on`), by one ballot per key bit.
__device__ __forceinline__ uint64_t peers(uint32_t key, int bits, bool on) {
  uint64_t m = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t s = __ballot((key >> b) & 1u);
    m &= ((key >> b) & 1u) ? s : ~s;
  }
  return m;
}

// Where the tokens of the wave's lanes go, each with the counter `key` of its next place (one counter per key and wave):
// equal keys take successive places in lane order, and their counter moves past them.  Every lane calls it.
__device__ __forceinline__ uint32_t take_places(uint32_t* counters, uint32_t key, int bits, bool on) {
  const uint64_t m = peers(key, bits, on);
  const int lane = threadIdx.x & 63, lead = on ? __ffsll((unsigned long long)m) - 1 : lane;
  uint32_t at = 0;
  if (on && lane == lead) at = atomicAdd(&counters[key], (uint32_t)__popcll(m));
  return (uint32_t)__shfl((int)at, lead) + __popcll(m & ((1ull << lane) - 1));
}

// Sum of `value` over the threads before this one, and the workgroup's total; WAVES waves, scratch of as many words.
template <int WAVES>
__device__ __forceinline__ uint32_t scan_block(uint32_t value, uint32_t* scratch, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = value;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t v = (uint32_t)__shfl_up((int)sum, d);
    if (lane >= d) sum += v;
  }
  if (lane == 63) scratch[wave] = sum;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const uint32_t v = scratch[w];
    if (w < wave) before += v;
    total += v;
  }
  __syncthreads();
  return before + sum - value;
}

struct Rows {
  const void* x;
  void* grad;
  int64_t dim, ld_x;
  float scale;
};

// acc += the rows of dX of up to 64 tokens (lane l holds the l-th) for this lane's columns, in order; eight rows' loads are
// in flight together (32 in k_embed_parts took no less time).
constexpr int kFlight = 8;
template <int DT>
__device__ __forceinline__ void add_rows(const Rows& a, uint32_t mine, uint32_t count, int64_t col, float* acc) {
  const int64_t left = a.dim - col;
  const uint32_t m = __builtin_amdgcn_readfirstlane(count);
  for (uint32_t q = 0; q < m; q += kFlight) {
    u32x4_t w[kFlight];
#pragma unroll
    for (int h = 0; h < kFlight; ++h)
      if (q + h < m) {
        const int64_t row = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)mine, (int)(q + h)) * a.ld_x;
        if (left > 0) w[h] = load_raw<DT>(a.x, row + col, left);
      }
#pragma unroll
    for (int h = 0; h < kFlight; ++h)
      if (q + h < m) {
        float v[kVec<DT>];
        unpack_raw<DT>(w[h], v);
#pragma unroll
        for (int j = 0; j < kVec<DT>; ++j) acc[j] += v[j];
      }
  }
}

template <int DT, int DTG, bool ADD>
__device__ __forceinline__ void finish_row(const Rows& a, int64_t v, int64_t col, const float* acc) {
  constexpr int V = kVec<DT>;
  if (col >= a.dim) return;
  float g[V];
  if constexpr (ADD) load_elems<DTG, V>(a.grad, v * a.dim + col, g, a.dim - col);
#pragma unroll
  for (int j = 0; j < V; ++j) g[j] = ADD ? g[j] + a.scale * acc[j] : a.scale * acc[j];
  store_elems<DTG, V>(a.grad, v * a.dim + col, g, a.dim - col);
}

// Ids are dealt to 1 << log2 buckets by their low bits, which spreads the frequent ones (low ids, in most vocabularies);
// id v is local id v >> log2 of bucket v & mask.
struct Buckets {
  int log2;
  int32_t width;     // local ids of a bucket
  int bits;          // of a local id
};

// Zeros over the gradient, one vector a thread in memory order: written so, memory takes 6.9 TB/s on a 1.1 GB
// gradient, against 5 to 6 where threads write several vectors or waves follow the rows.
struct Fill {
  void* p;
  int64_t vectors;     // of 16 bytes
  int32_t tail;        // 2-byte words after the last vector
};

__device__ __forceinline__ void fill_zeros(const Fill& f, uint32_t block, uint32_t blocks) {
  for (int64_t v = (int64_t)block * 256 + threadIdx.x; v < f.vectors; v += (int64_t)blocks * 256)
    gmem((u32x4_t*)f.p)[v] = u32x4_t{0, 0, 0, 0};
  if (block == 0 && (int)threadIdx.x < f.tail) gmem((uint16_t*)f.p)[f.vectors * 8 + threadIdx.x] = 0;
}

// ---- gradient: few tokens, one launch ------------------------------------------------------------------------------

constexpr int kFewWaves = 8;
constexpr int kFewWidth = 512;   // local ids of a bucket, at most

// A workgroup per bucket and column block: it reads all ids (eight a thread at most), keeps its own, sorts them in LDS and
// writes its rows that have tokens, with `zeros` the others too.  Ids with more than kRun tokens are done last, a run a wave.
template <int DT, int DTG, bool ADD>
__global__ void __launch_bounds__(64 * kFewWaves) k_embed_few(Ids ids, int tokens, Buckets B, int64_t blocks, Rows a,
                                                              bool zeros, uint32_t* status) {
  constexpr int V = kVec<DT>, kThreads = 64 * kFewWaves, kIds = kFewTokens / kThreads, kCols = 64 * V;
  constexpr int kEach = kFewWidth / kThreads;
  __shared__ union {
    uint32_t cnt[kFewWaves][kFewWidth];   // per wave and local id: the next place in perm
    float part[kFewWaves][kCols];
  } u;
  __shared__ uint16_t perm[kFewTokens];
  __shared__ uint16_t start[kFewWidth], count[kFewWidth];
  __shared__ uint16_t some[kFewWidth], many[kFewTokens / kRun];   // local ids with up to kRun tokens, and with more
  __shared__ uint32_t scratch[kFewWaves], n_some, n_many;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const uint32_t bucket = (uint32_t)(blockIdx.x / blocks);
  const int64_t col = (int64_t)(blockIdx.x - bucket * blocks) * kCols + lane * V;
  const uint32_t mask = (1u << B.log2) - 1;
  if (tid == 0) n_some = n_many = 0;
  for (int q = tid; q < kFewWaves * kFewWidth; q += kThreads) (&u.cnt[0][0])[q] = 0;
  // each wave takes successive tokens
  const int per = (tokens + kThreads - 1) / kThreads * 64, t0 = wave * per + lane;
  int32_t row[kIds];
#pragma unroll
  for (int k = 0; k < kIds; ++k) {
    row[k] = -1;
    if (64 * k < per && t0 + 64 * k < tokens) row[k] = row_of(ids, t0 + 64 * k);
  }
  bool bad = false;
  int mine = 0;
#pragma unroll
  for (int k = 0; k < kIds; ++k) {
    bad |= row[k] == -2;
    row[k] = row[k] >= 0 && ((uint32_t)row[k] & mask) == bucket ? row[k] >> B.log2 : -1;
    mine += row[k] >= 0;
  }
  const bool any = __syncthreads_or(mine);
  if (blockIdx.x == 0) {
    const bool wrong = __syncthreads_or(bad);
    if (tid == 0) *status = wrong ? kStatusIndex : 0u;
  }
  if (any) {
#pragma unroll
    for (int k = 0; k < kIds; ++k)
      if (row[k] >= 0) atomicAdd(&u.cnt[wave][row[k]], 1u);
    __syncthreads();
    uint32_t c[kEach][kFewWaves], n[kEach], sum = 0, total;
#pragma unroll
    for (int h = 0; h < kEach; ++h) {
      n[h] = 0;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) n[h] += c[h][w] = u.cnt[w][tid * kEach + h];
      sum += n[h];
    }
    uint32_t at = scan_block<kFewWaves>(sum, scratch, total);
#pragma unroll
    for (int h = 0; h < kEach; ++h) {
      const int q = tid * kEach + h;
      start[q] = (uint16_t)at;
      count[q] = (uint16_t)n[h];
      // in any order: each is done by itself
      if (n[h] > kRun) many[atomicAdd(&n_many, 1u)] = (uint16_t)q;
      else if (n[h] > 0) some[atomicAdd(&n_some, 1u)] = (uint16_t)q;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        u.cnt[w][q] = at;
        at += c[h][w];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kIds; ++k) {
      if (__ballot(row[k] >= 0) == 0) continue;
      const uint32_t to = take_places(u.cnt[wave], row[k] >= 0 ? row[k] : 0, B.bits, row[k] >= 0);
      if (row[k] >= 0) perm[to] = (uint16_t)(t0 + 64 * k);
    }
    __syncthreads();
  }
  if (zeros) {
    const float zero[V] = {};
    for (int q = wave; q < B.width; q += kFewWaves) {
      const int64_t v = ((int64_t)q << B.log2) + bucket;
      if (v < ids.vocab && (!any || count[q] == 0)) finish_row<DT, DTG, false>(a, v, col, zero);
    }
  }
  if (!any) return;
  const uint32_t few = n_some, hot = n_many;
  for (uint32_t h = wave; h < few; h += kFewWaves) {
    const uint32_t q = some[h], m = count[q];
    float acc[V] = {};
    add_rows<DT>(a, (uint32_t)lane < m ? perm[start[q] + lane] : 0u, m, col, acc);
    finish_row<DT, DTG, ADD>(a, ((int64_t)q << B.log2) + bucket, col, acc);
  }
  for (uint32_t h = 0; h < hot; ++h) {
    const uint32_t q = many[h], s = start[q], e = s + count[q];
    float out[V] = {};
    for (uint32_t r0 = s; r0 < e; r0 += kRun * kFewWaves) {
      __syncthreads();
      const uint32_t r = r0 + wave * kRun, m = r < e ? min(e - r, (uint32_t)kRun) : 0u;
      if (m > 0) {
        float acc[V] = {};
        add_rows<DT>(a, (uint32_t)lane < m ? perm[r + lane] : 0u, m, col, acc);
#pragma unroll
        for (int j = 0; j < V; ++j) u.part[wave][j * 64 + lane] = acc[j];
      }
      __syncthreads();
      if (wave == 0)
        for (int w = 0; w < kFewWaves && r0 + w * kRun < e; ++w)
#pragma unroll
          for (int j = 0; j < V; ++j) out[j] += u.part[w][j * 64 + lane];
    }
    if (wave == 0) finish_row<DT, DTG, ADD>(a, ((int64_t)q << B.log2) + bucket, col, out);
  }
}

__global__ void __launch_bounds__(256) k_embed_fill(Fill f) { fill_zeros(f, blockIdx.x, gridDim.x); }

// ---- gradient: many tokens -----------------------------------------------------------------------------------------
//
// Count (with further workgroups that write the gradient's zeros), scatter into buckets, sort each bucket, partial sums of
// frequent ids, rows.  32768 tokens into 152064 x 3584 in bf16: 266 us, of which the zeros take 150 (1.09 GB), the sort's
// latencies 20, the reads of dX and the rows that have tokens the rest; their bytes alone would take 209.  Spreading the zeros
// over the first four launches, under whose latencies they would hide, gained nothing (270 to 280 us).

constexpr int kMaxWidth = ISO_EMBED_MAX_VOCAB / kMaxBuckets;

// Distinct ids and the runs of frequent ones, appended bucket by bucket in any order (each is worked on by itself).  Ids of
// 1/16 of the buckets share a counter, on a line of its own, and the part of the list that their tokens take in sorted order:
// with one counter for all, 512 additions to one address took 7 of the sort's 12 us.
struct Lists {
  uint32_t* n;               // runs, frequent ids; from kLine on the groups' ids, kLine apart
  uint4* ids;                // id, first sorted position, tokens (at most kRun)
  uint2* runs;               // first sorted position, tokens
  uint4* many;               // id with more than kRun tokens, its first run, its runs
  const uint32_t* bucket0;   // first sorted position of each bucket
  int shift;                 // group of a bucket: bucket >> shift
  int groups;
};

// Tokens per (tile, bucket); tokens outside the vocabulary are noted per tile, the lists are empty yet.
__global__ void __launch_bounds__(256) k_embed_count(Ids ids, int64_t tokens, int64_t tile, int tiles, Buckets B,
                                                     uint32_t* __restrict__ hist, uint32_t* __restrict__ bad,
                                                     uint32_t* __restrict__ listed, Fill f) {
  if (blockIdx.x >= tiles) return fill_zeros(f, blockIdx.x - tiles, gridDim.x - tiles);
  __shared__ uint32_t h[kMaxBuckets];
  __shared__ uint32_t any;
  const int buckets = 1 << B.log2;
  for (int b = threadIdx.x; b < buckets; b += 256) h[b] = 0;
  if (threadIdx.x == 0) any = 0;
  if (blockIdx.x == 0 && threadIdx.x <= kGroups) listed[threadIdx.x * kLine] = listed[threadIdx.x * kLine + 1] = 0;
  __syncthreads();
  const int64_t t0 = blockIdx.x * tile, t1 = min(tokens, t0 + tile);
  for (int64_t t = t0 + threadIdx.x; t < t1; t += 256) {
    const int32_t r = row_of(ids, t);
    if (r >= 0) atomicAdd(&h[r & (buckets - 1)], 1u);
    if (r == -2) any = 1;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < buckets; b += 256) hist[(int64_t)blockIdx.x * buckets + b] = h[b];
  if (threadIdx.x == 0) bad[blockIdx.x] = any;
}

// Stable scatter of (local id, token) into buckets.  Each workgroup adds up the counts before its tile itself (at most
// 64 x 512 of them), each wave owns a contiguous part of the tile.
__global__ void __launch_bounds__(512) k_embed_scatter(Ids ids, int64_t tokens, int64_t tile, int tiles, Buckets B,
                                                       const uint32_t* __restrict__ hist,
                                                       const uint32_t* __restrict__ bad, uint32_t* __restrict__ bucket0,
                                                       uint2* __restrict__ pairs, uint32_t* status) {
  __shared__ uint32_t cnt[8][kMaxBuckets];
  __shared__ uint32_t scratch[8];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, buckets = 1 << B.log2;
  for (int b = tid; b < 8 * kMaxBuckets; b += 512) (&cnt[0][0])[b] = 0;
  uint32_t total = 0, before = 0, all;
  if (tid < buckets) {
#pragma unroll 8
    for (int w = 0; w < tiles; ++w) {
      const uint32_t c = hist[w * buckets + tid];
      before += w < (int)blockIdx.x ? c : 0u;
      total += c;
    }
  }
  __syncthreads();
  const int64_t t0 = blockIdx.x * tile, t1 = min(tokens, t0 + tile), per = (tile + 511) / 512 * 64;
  const int64_t w0 = min(t1, t0 + wave * per), w1 = min(t1, w0 + per);
  for (int64_t t = w0 + lane; t < w1; t += 64) {
    const int32_t r = row_of(ids, t);
    if (r >= 0) atomicAdd(&cnt[wave][r & (buckets - 1)], 1u);
  }
  const uint32_t first = scan_block<8>(total, scratch, all);
  if (tid < buckets) {
    if (blockIdx.x == 0) bucket0[tid] = first;
    uint32_t at = first + before;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const uint32_t c = cnt[w][tid];
      cnt[w][tid] = at;
      at += c;
    }
  }
  if (blockIdx.x == 0) {
    if (tid == 0) bucket0[buckets] = all;
    const bool any = __syncthreads_or(tid < tiles && bad[tid] != 0);
    if (tid == 0) *status = any ? kStatusIndex : 0u;
  }
  __syncthreads();
  for (int64_t t = w0; t < w1; t += 64) {
    const int32_t r = t + lane < w1 ? row_of(ids, t + lane) : -1;
    const uint32_t at = take_places(cnt[wave], r >= 0 ? r & (buckets - 1) : 0, B.log2, r >= 0);
    if (r >= 0) pairs[at] = make_uint2((uint32_t)r >> B.log2, (uint32_t)(t + lane));
  }
}

// One workgroup per bucket: stable counting sort by local id.  Writes the sorted tokens and appends to the lists.
// Dynamic LDS: 8 waves x width counters.
__global__ void __launch_bounds__(512) k_embed_bucket(Buckets B, const uint2* __restrict__ pairs,
                                                      uint32_t* __restrict__ perm, Lists l) {
  extern __shared__ uint32_t cnt[];
  __shared__ uint32_t scratch[8], n_ids, n_runs, n_many;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, width = B.width;
  const uint32_t s = l.bucket0[blockIdx.x], n = l.bucket0[blockIdx.x + 1] - s, group = blockIdx.x >> l.shift;
  if (n == 0) return;
  for (int q = tid; q < 8 * width; q += 512) cnt[q] = 0;
  if (tid == 0) n_ids = n_runs = n_many = 0;
  __syncthreads();
  const uint32_t per = (n + 511) / 512 * 64;
  const uint32_t w0 = min(n, wave * per), w1 = min(n, w0 + per);
  for (uint32_t q = w0 + lane; q < w1; q += 64) atomicAdd(&cnt[wave * width + pairs[s + q].x], 1u);
  __syncthreads();
  constexpr int kChunks = kMaxWidth / 512;
  uint32_t base = s, first[kChunks], many[kChunks], id_at[kChunks], run_at[kChunks];
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    many[k] = 0;
    if (k * 512 >= width) continue;
    const int q = k * 512 + tid;
    uint32_t c[8], all;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      c[w] = q < width ? cnt[w * width + q] : 0;
      many[k] += c[w];
    }
    uint32_t at = first[k] = base + scan_block<8>(many[k], scratch, all);
    if (many[k] > 0) id_at[k] = atomicAdd(many[k] > kRun ? &n_many : &n_ids, 1u);
    if (many[k] > kRun) run_at[k] = atomicAdd(&n_runs, (many[k] + kRun - 1) / kRun);
    if (q < width) {
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        cnt[w * width + q] = at;
        at += c[w];
      }
    }
    base += all;
  }
  __syncthreads();
  if (tid == 0) {
    if (n_ids > 0) n_ids = l.bucket0[group << l.shift] + atomicAdd(&l.n[kLine * (group + 1)], n_ids);
    if (n_many > 0) {
      n_runs = atomicAdd(&l.n[0], n_runs);
      n_many = atomicAdd(&l.n[1], n_many);
    }
  }
  for (uint32_t q = w0; q < w1; q += 64) {
    const bool on = q + lane < w1;
    const uint2 p = on ? pairs[s + q + lane] : make_uint2(0, 0);
    const uint32_t to = take_places(cnt + wave * width, p.x, B.bits, on);
    if (on) perm[to] = p.y;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    if (many[k] == 0) continue;
    const uint32_t v = ((uint32_t)(k * 512 + tid) << B.log2) + blockIdx.x;
    if (many[k] > kRun) {
      const uint32_t run0 = n_runs + run_at[k], runs = (many[k] + kRun - 1) / kRun;
      for (uint32_t p = 0; p < runs; ++p)
        l.runs[run0 + p] = make_uint2(first[k] + p * kRun, min((uint32_t)kRun, many[k] - p * kRun));
      l.many[n_many + id_at[k]] = make_uint4(v, run0, runs, 0);
    } else {
      l.ids[n_ids + id_at[k]] = make_uint4(v, first[k], many[k], 0);
    }
  }
}

// Partial sums of ids with more than kRun tokens, a wave per run and column block.
template <int DT>
__global__ void __launch_bounds__(256) k_embed_parts(const uint32_t* __restrict__ perm, Lists l, Rows a, int64_t blocks,
                                                     float* __restrict__ part) {
  constexpr int V = kVec<DT>;
  const int lane = threadIdx.x & 63;
  const int64_t items = (int64_t)l.n[0] * blocks;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
    const int64_t run = item / blocks;
    const uint2 r = l.runs[run];
    const int64_t col = (item - run * blocks) * (64 * V) + lane * V;
    float acc[V] = {};
    add_rows<DT>(a, (uint32_t)lane < r.y ? perm[r.x + lane] : 0u, r.y, col, acc);
    if (col < a.dim) store_elems<ISO_F32, V>(part, run * a.dim + col, acc, a.dim - col);
  }
}

// The gradient's rows that have tokens.  Frequent ids take a workgroup a column block: its waves add up a quarter of the id's
// runs each, in order, and then the quarters.  The others take a wave a column block; a wave has the list's entry after
// next and the next one's tokens under way while it adds the current rows, so that it waits for one memory access a row
// block instead of three.
template <int DT, int DTG, bool ADD>
__global__ void __launch_bounds__(256) k_embed_rows(const uint32_t* __restrict__ perm, Lists l, Rows a, int64_t blocks,
                                                    const float* __restrict__ part) {
  constexpr int V = kVec<DT>, kSums = 4;
  __shared__ float quarter[4][V][64];
  __shared__ uint32_t before[kGroups + 1], place[kGroups];   // ids of the groups before a group, and where its own lie
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t many = (int64_t)l.n[1] * blocks;
  const uint32_t own = (uint32_t)min(many, (int64_t)(gridDim.x / 2));   // workgroups of the frequent ids
  for (int64_t b = blockIdx.x; b < many && blockIdx.x < own; b += own) {
    const int64_t unit = b / blocks;
    const uint4 id = l.many[unit];
    const int64_t col = (b - unit * blocks) * (64 * V) + lane * V;
    const uint32_t each = (id.z + 3) / 4, r0 = min(id.z, wave * each), r1 = min(id.z, r0 + each);
    float acc[V] = {};
    for (uint32_t r = r0; r < r1; r += kSums) {
      float p[kSums][V];
#pragma unroll
      for (int h = 0; h < kSums; ++h)
        if (r + h < r1) load_elems<ISO_F32, V>(part, (int64_t)(id.y + r + h) * a.dim + col, p[h], a.dim - col);
#pragma unroll
      for (int h = 0; h < kSums; ++h)
        if (r + h < r1) {
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] += p[h][j];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) quarter[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] = ((quarter[0][j][lane] + quarter[1][j][lane]) + quarter[2][j][lane]) + quarter[3][j][lane];
      finish_row<DT, DTG, ADD>(a, id.x, col, acc);
    }
    __syncthreads();
  }
  if (blockIdx.x < own) return;
  if (wave == 0) {
    uint32_t sum = lane < l.groups ? l.n[kLine * (lane + 1)] : 0;
    if (lane < l.groups) place[lane] = l.bucket0[lane << l.shift];
#pragma unroll
    for (int d = 1; d < kGroups; d <<= 1) {
      const uint32_t v = (uint32_t)__shfl_up((int)sum, d);
      if (lane >= d) sum += v;
    }
    if (lane < kGroups) before[lane + 1] = sum;
    if (lane == 0) before[0] = 0;
  }
  __syncthreads();
  const int64_t stride = (int64_t)(gridDim.x - own) * 4, items = (int64_t)before[kGroups] * blocks;
  int64_t item = (int64_t)(blockIdx.x - own) * 4 + wave;
  auto entry = [&](int64_t at) {
    if (at >= items) return make_uint4(0, 0, 0, 0);
    const uint32_t unit = (uint32_t)(at / blocks);
    int g = 0;
#pragma unroll
    for (int half = kGroups / 2; half > 0; half /= 2)
      if (before[g + half] <= unit) g += half;
    return l.ids[place[g] + (unit - before[g])];
  };
  auto tokens = [&](const uint4& id) { return (uint32_t)lane < id.z ? perm[id.y + lane] : 0u; };
  uint4 now = entry(item), next = entry(item + stride);
  uint32_t mine = tokens(now);
  for (; item < items; item += stride) {
    const uint4 after = entry(item + 2 * stride);
    const uint32_t theirs = tokens(next);
    const int64_t col = (item - item / blocks * blocks) * (64 * V) + lane * V;
    float acc[V] = {};
    add_rows<DT>(a, mine, now.z, col, acc);
    finish_row<DT, DTG, ADD>(a, now.x, col, acc);
    now = next, next = after, mine = theirs;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------

Buckets buckets_of(int64_t vocab, int log2) {
  Buckets B;
  B.log2 = log2;
  B.width = (int32_t)((vocab + (1ll << log2) - 1) >> log2);
  B.bits = log2_up(B.width);
  return B;
}

Ids ids_of(const iso_embed& e) {
  return Ids{e.ids, e.id_type == ISO_I64, e.pad_id != ISO_NO_PAD, e.pad_id, e.vocab};
}

Fill zeros_of(const iso_embed& e, int dt_grad) {
  const int64_t words = e.vocab * e.dim * (dt_grad == ISO_BF16 ? 1 : 2);
  return Fill{e.grad, words / 8, (int32_t)(words % 8)};
}
unsigned grid_of(const Fill& f) { return grid_for((f.vectors + 255) / 256); }

// Gradients from 64 MiB on are cleared by a launch of their own at the rate of fill_zeros, smaller ones by the workgroups
// that hold the ids, whose writes are slower (5.0 against 6.9 TB/s) but need no second launch (4 us).
constexpr int64_t kOwnFill = 64ll << 20;

template <int DT, int DTG, bool ADD>
hipError_t grad_few(const iso_embed& e, const Rows& a, uint8_t* ws, hipStream_t s) {
  // 512 buckets, or as many as the vocabulary takes to leave at most 512 ids in each
  const Buckets B = buckets_of(e.vocab, std::max(std::min(9, log2_up(e.vocab)), log2_up((e.vocab + kFewWidth - 1) / kFewWidth)));
  const int64_t blocks = (e.dim + 64 * kVec<DT> - 1) / (64 * kVec<DT>);   // at most 1024: 2^21 workgroups, 2^30 threads
  const bool fill = !ADD && e.vocab * e.dim * (DTG == ISO_BF16 ? 2 : 4) >= kOwnFill;
  if (fill) {
    const Fill f = zeros_of(e, DTG);
    k_embed_fill<<<grid_of(f), 256, 0, s>>>(f);
  }
  k_embed_few<DT, DTG, ADD><<<(unsigned)(blocks << B.log2), 64 * kFewWaves, 0, s>>>(ids_of(e), (int)e.tokens, B, blocks, a,
                                                                                    !ADD && !fill, (uint32_t*)ws);
  return hipGetLastError();
}

template <int DT, int DTG, bool ADD>
hipError_t grad_many(const iso_embed& e, const Rows& a, uint8_t* ws, hipStream_t s) {
  const EmbedPlan P = embed_plan(e.tokens, e.vocab, e.dim);
  const Ids ids = ids_of(e);
  const Buckets B = buckets_of(e.vocab, std::min(9, log2_up(e.vocab)));
  const unsigned tiles = (unsigned)P.tiles, buckets = 1u << B.log2;
  const Lists l{(uint32_t*)(ws + P.listed), (uint4*)(ws + P.ids), (uint2*)(ws + P.runs), (uint4*)(ws + P.many),
                (const uint32_t*)(ws + P.bucket0), std::max(0, B.log2 - 4), std::min(kGroups, 1 << B.log2)};
  uint32_t* const perm = (uint32_t*)(ws + P.perm);
  uint2* const pairs = (uint2*)(ws + P.pairs);
  float* const part = (float*)(ws + P.part);
  const Fill f = zeros_of(e, DTG);
  k_embed_count<<<tiles + (ADD ? 0 : grid_of(f)), 256, 0, s>>>(ids, e.tokens, P.tile, tiles, B, (uint32_t*)(ws + P.hist),
                                                               (uint32_t*)(ws + P.bad), l.n, f);
  k_embed_scatter<<<tiles, 512, 0, s>>>(ids, e.tokens, P.tile, tiles, B, (const uint32_t*)(ws + P.hist),
                                        (const uint32_t*)(ws + P.bad), (uint32_t*)(ws + P.bucket0), pairs, (uint32_t*)ws);
  k_embed_bucket<<<buckets, 512, sizeof(uint32_t) * 8 * (size_t)B.width, s>>>(B, pairs, perm, l);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int64_t blocks = (e.dim + 64 * kVec<DT> - 1) / (64 * kVec<DT>);
  k_embed_parts<DT><<<(unsigned)std::min<int64_t>((P.most_runs * blocks + 3) / 4, 2048), 256, 0, s>>>(perm, l, a, blocks, part);
  const int64_t most = (std::min(e.tokens, e.vocab) * blocks + 3) / 4;
  k_embed_rows<DT, DTG, ADD><<<(unsigned)std::min<int64_t>(most + 1, 2048), 256, 0, s>>>(perm, l, a, blocks, part);
  return hipGetLastError();
}

template <int DT, int DTG, bool ADD>
hipError_t grad(const iso_embed& e, uint8_t* ws, hipStream_t s) {
  const Rows a{e.x, e.grad, e.dim, e.ld_x, (float)e.scale};
  return e.tokens <= kFewTokens ? grad_few<DT, DTG, ADD>(e, a, ws, s) : grad_many<DT, DTG, ADD>(e, a, ws, s);
}

}  // namespace

hipError_t run_embed_lookup(const iso_embed& e, int dt, uint8_t* ws, hipStream_t s) {
  const int v = dt == ISO_BF16 ? kVec<ISO_BF16> : kVec<ISO_F32>;
  const int64_t items = e.tokens * ((e.dim + v - 1) / v), row_bytes = e.dim * (dt == ISO_BF16 ? 2 : 4);
  const bool alone = lookup_checks_alone(e.tokens, row_bytes);
  const unsigned grid = 1 + grid_for((items + kLookupBlock - 1) / kLookupBlock);
  auto go = [&](auto k) {
    k<<<grid, 256, 0, s>>>(ids_of(e), e.table, e.x, e.tokens, e.dim, e.ld_x, (float)e.scale, alone, (uint32_t*)ws);
  };
  if (!alone) {
    const hipError_t err = fill_u32((uint32_t*)ws, 1, 0u, s);
    if (err != hipSuccess) return err;
  }
  const bool stream = streamed(e.tokens * row_bytes);
  if (dt == ISO_BF16) stream ? go(k_embed_lookup<ISO_BF16, true>) : go(k_embed_lookup<ISO_BF16, false>);
  else stream ? go(k_embed_lookup<ISO_F32, true>) : go(k_embed_lookup<ISO_F32, false>);
  return hipGetLastError();
}

hipError_t run_embed_grad(const iso_embed& e, int dt, int dt_grad, bool accumulate, uint8_t* ws, hipStream_t s) {
  auto go = [&](auto f) { return f(e, ws, s); };
  if (dt == ISO_BF16 && dt_grad == ISO_BF16)
    return go(accumulate ? grad<ISO_BF16, ISO_BF16, true> : grad<ISO_BF16, ISO_BF16, false>);
  if (dt == ISO_BF16) return go(accumulate ? grad<ISO_BF16, ISO_F32, true> : grad<ISO_BF16, ISO_F32, false>);
  if (dt_grad == ISO_BF16) return go(accumulate ? grad<ISO_F32, ISO_BF16, true> : grad<ISO_F32, ISO_BF16, false>);
  return go(accumulate ? grad<ISO_F32, ISO_F32, true> : grad<ISO_F32, ISO_F32, false>);
}

}  // namespace iso
