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

namespace iso {

namespace {

// Workgroups of a launch over `n` pieces of work, which the kernels walk in strides of the grid (a launch holds fewer
// than 2^32 threads).
unsigned grid_for(int64_t n) { return (unsigned)std::min<int64_t>(std::max<int64_t>(n, 1), 1 << 23); }

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

constexpr int kLookupItems = 4;   // 16-byte vectors (or elements) a thread
constexpr int kLookupBlock = 256 * kLookupItems;

// Workgroup 0 looks at every id and writes the status word, so that the call is one launch: nothing has to be
// cleared before the others find a bad id.  The others copy 1024 vectors each, numbered through tokens and columns:
// a thread's four ids, and then its four vectors, are in flight together.
template <int DT, bool VEC>
__global__ void __launch_bounds__(256) k_embed_lookup(Ids ids, const void* __restrict__ table, void* __restrict__ x,
                                                      int64_t tokens, int64_t dim, int64_t ld_x, float scale,
                                                      uint32_t* status) {
  if (blockIdx.x == 0) {
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
  constexpr int V = VEC ? Fmt<DT>::kPerVec : 1;
  const uint32_t per_row = (uint32_t)(dim / V);
  const int64_t items = tokens * per_row, step = (int64_t)(gridDim.x - 1) * kLookupBlock;
  for (int64_t base = (int64_t)(blockIdx.x - 1) * kLookupBlock; base < items; base += step) {
    const int64_t t0 = base / per_row;
    const uint32_t c0 = (uint32_t)(base - t0 * per_row);
    int64_t tok[kLookupItems];
    uint32_t col[kLookupItems];
    int32_t row[kLookupItems];
#pragma unroll
    for (int q = 0; q < kLookupItems; ++q) {
      const uint32_t r = c0 + q * 256 + threadIdx.x, d = r / per_row;
      tok[q] = t0 + d;
      col[q] = r - d * per_row;
      row[q] = tok[q] < tokens ? row_of(ids, tok[q]) : -1;
    }
    float v[kLookupItems][V];
#pragma unroll
    for (int q = 0; q < kLookupItems; ++q) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[q][j] = 0.0f;
      if (row[q] >= 0) load_elems<DT, V>(table, (int64_t)row[q] * dim + (int64_t)col[q] * V, v[q]);
    }
#pragma unroll
    for (int q = 0; q < kLookupItems; ++q) {
      if (tok[q] >= tokens) continue;
      if (row[q] >= 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[q][j] *= scale;
      }
      store_elems<DT, V>(x, tok[q] * ld_x + (int64_t)col[q] * V, v[q]);
    }
  }
}

// ---- gradient: the sort --------------------------------------------------------------------------------------------

constexpr int kMaxBuckets = 512;
constexpr int kMaxTiles = 64;
constexpr int kMinTile = 1024;
constexpr int kRun = 32;          // tokens of one partial sum
constexpr int kSlotSpan = 16;     // an id with m > kRun tokens from sorted position p on owns slots p/16 ...:
                                  // ceil(m/32) <= floor(m/16) of them, so no two ids share one

// Lanes of the wave whose key equals this lane's (of those with `on`), by one ballot per key bit.
__device__ __forceinline__ uint64_t peers(uint32_t key, int bits, bool on) {
  uint64_t m = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t s = __ballot((key >> b) & 1u);
    m &= ((key >> b) & 1u) ? s : ~s;
  }
  return m;
}

// Counts per (tile, bucket); tokens outside the vocabulary are noted per tile, no slot is taken yet.
__global__ void __launch_bounds__(256) k_embed_count(Ids ids, int64_t tokens, int64_t tile, int shift, int buckets,
                                                     uint32_t* __restrict__ hist, uint32_t* __restrict__ bad,
                                                     int32_t* __restrict__ task, int64_t slots) {
  __shared__ uint32_t h[kMaxBuckets];
  __shared__ uint32_t any;
  for (int b = threadIdx.x; b < buckets; b += 256) h[b] = 0;
  if (threadIdx.x == 0) any = 0;
  __syncthreads();
  const int64_t t0 = blockIdx.x * tile, t1 = min(tokens, t0 + tile);
  for (int64_t t = t0 + threadIdx.x; t < t1; t += 256) {
    const int32_t r = row_of(ids, t);
    if (r >= 0) atomicAdd(&h[r >> shift], 1u);
    if (r == -2) any = 1;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < buckets; b += 256) hist[(int64_t)blockIdx.x * buckets + b] = h[b];
  if (threadIdx.x == 0) bad[blockIdx.x] = any;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < slots; q += (int64_t)gridDim.x * 256) task[q] = -1;
}

// Stable scatter of (id, token) into buckets.  Each workgroup adds up the counts before its tile itself (at most
// 64 x 512 of them), each wave owns a contiguous part of the tile and ranks equal buckets by ballots.
__global__ void __launch_bounds__(256) k_embed_scatter(Ids ids, int64_t tokens, int64_t tile, int shift, int buckets,
                                                       int bits, const uint32_t* __restrict__ hist,
                                                       const uint32_t* __restrict__ bad, uint32_t* __restrict__ bucket0,
                                                       uint2* __restrict__ pairs, uint32_t* status) {
  __shared__ uint32_t cnt[4][kMaxBuckets];
  __shared__ uint32_t scan[256];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, tiles = gridDim.x;
  uint32_t total[2], before[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int b = 2 * tid + h;
    total[h] = before[h] = 0;
    if (b < buckets) {
      for (int w = 0; w < tiles; ++w) {
        const uint32_t c = hist[(int64_t)w * buckets + b];
        if (w < (int)blockIdx.x) before[h] += c;
        total[h] += c;
      }
    }
  }
  scan[tid] = total[0] + total[1];
  for (int b = tid; b < 4 * kMaxBuckets; b += 256) (&cnt[0][0])[b] = 0;
  __syncthreads();
  for (int d = 1; d < 256; d <<= 1) {
    const uint32_t v = tid >= d ? scan[tid - d] : 0;
    __syncthreads();
    scan[tid] += v;
    __syncthreads();
  }
  const int64_t t0 = blockIdx.x * tile, per = (tile + 3) / 4;
  const int64_t w0 = min(min(tokens, t0 + tile), t0 + wave * per), w1 = min(min(tokens, t0 + tile), w0 + per);
  for (int64_t t = w0 + lane; t < w1; t += 64) {
    const int32_t r = row_of(ids, t);
    if (r >= 0) atomicAdd(&cnt[wave][r >> shift], 1u);
  }
  __syncthreads();
  const uint32_t first = scan[tid] - total[0] - total[1];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int b = 2 * tid + h;
    const uint32_t s = first + (h ? total[0] : 0);
    if (b < buckets) {
      if (blockIdx.x == 0) bucket0[b] = s;
      uint32_t at = s + before[h];
      for (int w = 0; w < 4; ++w) {
        const uint32_t c = cnt[w][b];
        cnt[w][b] = at;
        at += c;
      }
    }
  }
  if (blockIdx.x == 0 && tid == 255) bucket0[buckets] = scan[255];
  if (blockIdx.x == 0 && tid == 0) {
    uint32_t any = 0;
    for (int w = 0; w < tiles; ++w) any |= bad[w];
    *status = any ? kStatusIndex : 0u;
  }
  __syncthreads();
  for (int64_t t = w0; t < w1; t += 64) {
    const int32_t r = t + lane < w1 ? row_of(ids, t + lane) : -1;
    const uint32_t b = r >= 0 ? (uint32_t)r >> shift : 0u;
    const uint64_t m = peers(b, bits, r >= 0);
    if (r >= 0) {
      const int lead = __ffsll((unsigned long long)m) - 1;
      uint32_t at = 0;
      if (lane == lead) at = atomicAdd(&cnt[wave][b], (uint32_t)__popcll(m));
      at = (uint32_t)__shfl((int)at, lead) + __popcll(m & ((1ull << lane) - 1));
      pairs[at] = make_uint2((uint32_t)r, (uint32_t)(t + lane));
    }
  }
}

// One workgroup per bucket: stable counting sort by the id's low bits.  Writes the sorted tokens and their ids, the
// first sorted position of every id of the bucket's range, and the slots of ids with more than kRun tokens.
// Dynamic LDS: 8 waves x (1 << shift) counters.
__global__ void __launch_bounds__(512) k_embed_bucket(int64_t vocab, int shift, int buckets,
                                                      const uint32_t* __restrict__ bucket0,
                                                      const uint2* __restrict__ pairs, uint32_t* __restrict__ perm,
                                                      uint32_t* __restrict__ sid, uint32_t* __restrict__ start,
                                                      int32_t* __restrict__ task) {
  extern __shared__ uint32_t cnt[];
  __shared__ uint32_t scan[512];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int width = 1 << shift;
  const uint32_t s = bucket0[blockIdx.x], e = bucket0[blockIdx.x + 1], n = e - s;
  for (int q = tid; q < 8 * width; q += 512) cnt[q] = 0;
  __syncthreads();
  const uint32_t per = (n + 7) / 8;
  const uint32_t w0 = min(n, wave * per), w1 = min(n, w0 + per);
  for (uint32_t q = w0 + lane; q < w1; q += 64) atomicAdd(&cnt[wave * width + (pairs[s + q].x & (width - 1))], 1u);
  __syncthreads();
  // ids of this thread: `each` in a row (width <= 2048: at most four)
  const int each = (width + 511) / 512, id0 = tid * each;
  uint32_t own[4], sum = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    own[q] = 0;
    if (q < each && id0 + q < width) {
      for (int w = 0; w < 8; ++w) own[q] += cnt[w * width + id0 + q];
      sum += own[q];
    }
  }
  scan[tid] = sum;
  __syncthreads();
  for (int d = 1; d < 512; d <<= 1) {
    const uint32_t v = tid >= d ? scan[tid - d] : 0;
    __syncthreads();
    scan[tid] += v;
    __syncthreads();
  }
  uint32_t at = s + scan[tid] - sum;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q < each && id0 + q < width) {
      const int64_t v = ((int64_t)blockIdx.x << shift) + id0 + q;
      if (v < vocab) start[v] = at;
      if (own[q] > kRun)
        for (uint32_t c = 0; c * kRun < own[q]; ++c) task[at / kSlotSpan + c] = (int32_t)v;
      for (int w = 0; w < 8; ++w) {
        const uint32_t c = cnt[w * width + id0 + q];
        cnt[w * width + id0 + q] = at;
        at += c;
      }
    }
  }
  if (blockIdx.x == buckets - 1 && tid == 0) start[vocab] = e;
  __syncthreads();
  for (uint32_t q = w0; q < w1; q += 64) {
    const bool on = q + lane < w1;
    const uint2 p = on ? pairs[s + q + lane] : make_uint2(0, 0);
    const uint32_t b = p.x & (width - 1);
    const uint64_t m = peers(b, shift, on);
    if (on) {
      const int lead = __ffsll((unsigned long long)m) - 1;
      uint32_t to = 0;
      if (lane == lead) to = atomicAdd(&cnt[wave * width + b], (uint32_t)__popcll(m));
      to = (uint32_t)__shfl((int)to, lead) + __popcll(m & ((1ull << lane) - 1));
      perm[to] = p.y;
      sid[to] = p.x;
    }
  }
}

// ---- gradient: the sums --------------------------------------------------------------------------------------------

constexpr int kRowVecs = 4;   // vectors a lane holds of its wave's columns

struct RowArgs {
  const uint32_t* perm;
  const uint32_t* sid;
  const uint32_t* start;
  const int32_t* task;
  const void* x;
  float* part;
  void* grad;
  int64_t rows, dim, ld_x;   // rows: vocab, sorted positions or slots, whichever the launch walks
  int64_t blocks;            // column blocks of a row
  int64_t vocab;
  float scale;
};

// Sum of dX over the sorted positions [s, e), at most 64 of them, for this lane's columns: in order, four rows' loads
// in flight.
template <int DT, int V>
__device__ __forceinline__ void sum_rows(const RowArgs& a, uint32_t s, uint32_t e, int64_t col, float acc[kRowVecs][V]) {
  const int lane = threadIdx.x & 63;
  const uint32_t m = e - s;
  const uint32_t mine = (uint32_t)lane < m ? a.perm[s + lane] : 0u;
  uint32_t q = 0;
  for (; q + 4 <= m; q += 4) {
    float v[4][kRowVecs][V];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int64_t row = (int64_t)(uint32_t)__builtin_amdgcn_readlane(mine, q + h) * a.ld_x;
#pragma unroll
      for (int u = 0; u < kRowVecs; ++u)
        if (col + u * 64 * V < a.dim) load_elems<DT, V>(a.x, row + col + u * 64 * V, v[h][u]);
    }
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int u = 0; u < kRowVecs; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[u][j] += v[h][u][j];
  }
  for (; q < m; ++q) {
    const int64_t row = (int64_t)(uint32_t)__builtin_amdgcn_readlane(mine, q) * a.ld_x;
#pragma unroll
    for (int u = 0; u < kRowVecs; ++u) {
      if (col + u * 64 * V >= a.dim) continue;
      float v[V];
      load_elems<DT, V>(a.x, row + col + u * 64 * V, v);
#pragma unroll
      for (int j = 0; j < V; ++j) acc[u][j] += v[j];
    }
  }
}

// Partial sums of ids with more than kRun tokens, a wave per slot and column block.
template <int DT, int V>
__global__ void __launch_bounds__(256) k_embed_parts(RowArgs a) {
  const int64_t items = a.rows * a.blocks;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
    const int64_t slot = item / a.blocks;
    const int32_t v = a.task[slot];
    if (v < 0) continue;
    const uint32_t s = a.start[v], e = a.start[v + 1];
    const uint32_t p = s + (uint32_t)(slot - s / kSlotSpan) * kRun;
    const int64_t col = (item - slot * a.blocks) * (64 * kRowVecs * V) + (threadIdx.x & 63) * V;
    float acc[kRowVecs][V] = {};
    sum_rows<DT, V>(a, p, min(e, p + kRun), col, acc);
#pragma unroll
    for (int u = 0; u < kRowVecs; ++u)
      if (col + u * 64 * V < a.dim) store_elems<ISO_F32, V>(a.part, slot * a.dim + col + u * 64 * V, acc[u]);
  }
}

// One row of the gradient a wave and column block.  ADD = false walks the whole vocabulary (a row without tokens is
// zeros), ADD = true the sorted positions, of which the first of each id does the id's row.
template <int DT, int DTG, int V, bool ADD>
__global__ void __launch_bounds__(256) k_embed_rows(RowArgs a) {
  const int64_t units = ADD ? a.start[a.vocab] : a.rows;   // padding is not sorted
  const int64_t items = units * a.blocks;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
    const int64_t unit = item / a.blocks;
    const int64_t col = (item - unit * a.blocks) * (64 * kRowVecs * V) + (threadIdx.x & 63) * V;
    const int64_t v = ADD ? a.sid[unit] : unit;
    const uint32_t s = a.start[v], e = a.start[v + 1];
    if (ADD && s != (uint32_t)unit) continue;
    float acc[kRowVecs][V] = {};
    if (e - s <= kRun) {
      sum_rows<DT, V>(a, s, e, col, acc);
    } else {
      const int64_t slot0 = s / kSlotSpan, parts = (e - s + kRun - 1) / kRun;
      for (int64_t c = 0; c < parts; ++c)
#pragma unroll
        for (int u = 0; u < kRowVecs; ++u) {
          if (col + u * 64 * V >= a.dim) continue;
          float p[V];
          load_elems<ISO_F32, V>(a.part, (slot0 + c) * a.dim + col + u * 64 * V, p);
#pragma unroll
          for (int j = 0; j < V; ++j) acc[u][j] += p[j];
        }
    }
#pragma unroll
    for (int u = 0; u < kRowVecs; ++u) {
      if (col + u * 64 * V >= a.dim) continue;
      const int64_t at = v * a.dim + col + u * 64 * V;
      float g[V];
      if constexpr (ADD) load_elems<DTG, V>(a.grad, at, g);
#pragma unroll
      for (int j = 0; j < V; ++j) g[j] = ADD ? g[j] + a.scale * acc[u][j] : a.scale * acc[u][j];
      store_elems<DTG, V, !ADD>(a.grad, at, g);
    }
  }
}

template <int DT, int DTG, int V>
hipError_t launch_rows(RowArgs a, int64_t vocab, int64_t tokens, int64_t slots, bool accumulate, hipStream_t s) {
  a.blocks = (a.dim + 64 * kRowVecs * V - 1) / (64 * kRowVecs * V);
  a.vocab = vocab;
  if (slots > 0) {
    a.rows = slots;
    k_embed_parts<DT, V><<<grid_for((slots * a.blocks + 3) / 4), 256, 0, s>>>(a);
  }
  a.rows = accumulate ? tokens : vocab;
  const unsigned grid = grid_for((a.rows * a.blocks + 3) / 4);
  if (accumulate) k_embed_rows<DT, DTG, V, true><<<grid, 256, 0, s>>>(a);
  else k_embed_rows<DT, DTG, V, false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

Ids ids_of(const iso_embed& e) {
  return Ids{e.ids, e.id_type == ISO_I64, e.pad_id != ISO_NO_PAD, e.pad_id, e.vocab};
}

template <int DT, bool VEC>
void launch_lookup(const iso_embed& e, uint8_t* ws, hipStream_t s) {
  constexpr int V = VEC ? Fmt<DT>::kPerVec : 1;
  const int64_t items = e.tokens * (e.dim / V);
  const unsigned grid = 1 + grid_for((items + kLookupBlock - 1) / kLookupBlock);
  k_embed_lookup<DT, VEC><<<grid, 256, 0, s>>>(ids_of(e), e.table, e.x, e.tokens, e.dim, e.ld_x, (float)e.scale,
                                               (uint32_t*)ws);
}

}  // namespace

EmbedPlan embed_plan(int64_t tokens, int64_t vocab, int64_t dim) {
  EmbedPlan P;
  while (((vocab - 1) >> P.shift) >= kMaxBuckets) ++P.shift;
  P.buckets = (int)((vocab - 1) >> P.shift) + 1;
  P.tile = std::max<int64_t>(kMinTile, (tokens + kMaxTiles - 1) / kMaxTiles);
  P.tiles = std::max<int64_t>(1, (tokens + P.tile - 1) / P.tile);
  P.slots = tokens > kRun ? tokens / kSlotSpan + 1 : 0;
  size_t at = kStatusBytes;
  auto region = [&](size_t bytes) {
    const size_t o = at;
    at = align_up(at + bytes, 256);
    return o;
  };
  P.bad = region(sizeof(uint32_t) * P.tiles);
  P.hist = region(sizeof(uint32_t) * P.tiles * P.buckets);
  P.bucket0 = region(sizeof(uint32_t) * (P.buckets + 1));
  P.pairs = region(sizeof(uint2) * tokens);
  P.perm = region(sizeof(uint32_t) * tokens);
  P.sid = region(sizeof(uint32_t) * tokens);
  P.start = region(sizeof(uint32_t) * (vocab + 1));
  P.task = region(sizeof(int32_t) * P.slots);
  P.part = region(sizeof(float) * P.slots * dim);
  P.total = at;
  return P;
}

hipError_t run_embed_lookup(const iso_embed& e, int dt, uint8_t* ws, hipStream_t s) {
  const bool vec = vector_rows(e.dim, e.ld_x, dt == ISO_BF16 ? 8 : 4);
  if (dt == ISO_BF16) vec ? launch_lookup<ISO_BF16, true>(e, ws, s) : launch_lookup<ISO_BF16, false>(e, ws, s);
  else vec ? launch_lookup<ISO_F32, true>(e, ws, s) : launch_lookup<ISO_F32, false>(e, ws, s);
  return hipGetLastError();
}

hipError_t run_embed_grad(const iso_embed& e, int dt, int dt_grad, bool accumulate, uint8_t* ws, hipStream_t s) {
  const EmbedPlan P = embed_plan(e.tokens, e.vocab, e.dim);
  const Ids ids = ids_of(e);
  uint32_t* const start = (uint32_t*)(ws + P.start);
  k_embed_count<<<(unsigned)P.tiles, 256, 0, s>>>(ids, e.tokens, P.tile, P.shift, P.buckets, (uint32_t*)(ws + P.hist),
                                                  (uint32_t*)(ws + P.bad), (int32_t*)(ws + P.task), P.slots);
  int bits = 0;
  while ((1 << bits) < P.buckets) ++bits;
  k_embed_scatter<<<(unsigned)P.tiles, 256, 0, s>>>(ids, e.tokens, P.tile, P.shift, P.buckets, bits,
                                                    (const uint32_t*)(ws + P.hist), (const uint32_t*)(ws + P.bad),
                                                    (uint32_t*)(ws + P.bucket0), (uint2*)(ws + P.pairs), (uint32_t*)ws);
  k_embed_bucket<<<(unsigned)P.buckets, 512, sizeof(uint32_t) * 8 * ((size_t)1 << P.shift), s>>>(
      e.vocab, P.shift, P.buckets, (const uint32_t*)(ws + P.bucket0), (const uint2*)(ws + P.pairs),
      (uint32_t*)(ws + P.perm), (uint32_t*)(ws + P.sid), start, (int32_t*)(ws + P.task));
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  RowArgs a{(const uint32_t*)(ws + P.perm), (const uint32_t*)(ws + P.sid), start, (const int32_t*)(ws + P.task),
            e.x, (float*)(ws + P.part), e.grad, 0, e.dim, e.ld_x, 0, 0, (float)e.scale};
  auto go = [&](auto f) { return f(a, e.vocab, e.tokens, P.slots, accumulate, s); };
  const bool vec = vector_rows(e.dim, e.ld_x, dt == ISO_BF16 ? 8 : 4);
  if (dt == ISO_BF16 && dt_grad == ISO_BF16)
    return go(vec ? launch_rows<ISO_BF16, ISO_BF16, 8> : launch_rows<ISO_BF16, ISO_BF16, 1>);
  if (dt == ISO_BF16) return go(vec ? launch_rows<ISO_BF16, ISO_F32, 8> : launch_rows<ISO_BF16, ISO_F32, 1>);
  if (dt_grad == ISO_BF16) return go(vec ? launch_rows<ISO_F32, ISO_BF16, 4> : launch_rows<ISO_F32, ISO_BF16, 1>);
  return go(vec ? launch_rows<ISO_F32, ISO_F32, 4> : launch_rows<ISO_F32, ISO_F32, 1>);
}

}  // namespace iso
