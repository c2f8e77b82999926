// Weight gradients of linear layers from 8-bit activation checkpoints: G = [G +] dY^T X, X[t, i] = q 2^k.
//
// X is exact in bf16, so the products of a bf16 dY are exact and bf16 matrix instructions with binary32 accumulators
// lose nothing but the sum's own rounding; a binary32 dY is the sum of three bf16 parts of 8 bits each (cut, not
// rounded: every remainder is exact), which makes it three products with the same X, added least part first.
//
// A call is up to three launches per 16 layers (fewer where a gradient repeats).  k_wgrad_prep brings operands into the form that the product reads,
// bf16 rows aligned to 16 bytes: X always (once per checkpoint, however many layers share it), dY where it is fp32 or
// its rows are not aligned.  k_wgrad forms the tiles of all layers' gradients.  k_wgrad_join adds up tiles whose
// tokens were split.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "iso.h"
#include "iso_device.h"
#include "iso_grad.h"
#include "iso_grad_device.h"
#include "iso_mfma.h"

namespace iso {

namespace {

constexpr int kStages = 4;           // steps in LDS

// A workgroup's tile of G, 256 x 256 or 128 x 128.
template <int TILE>
struct Tile {
  static constexpr int kQuarter = TILE / 2;                 // a wave has kQuarter x kQuarter
  static constexpr int kFrags = kQuarter / 32;              // fragments of 32 columns of a panel a wave reads
  static constexpr int kRowBytes = TILE * 2;                // a token's row of a panel
  static constexpr int kPanel = kStep * kRowBytes;
  static constexpr int kStage = 2 * kPanel;
  static constexpr int kLoads = TILE / 64;                  // 16-byte loads a lane and panel
  static constexpr int kOutBytes = (kQuarter + 4) * 4;      // a row of the result in LDS
};

// ---- operand preparation -------------------------------------------------------------------------------------------

// Eight columns of one row a thread.  X: q 2^k, whose upper 16 bits are the whole value.  dY: its bf16 parts, least
// first, rows up to a whole step zero (X has none there, and 0 times what lies there may be NaN).
template <int DT>
__device__ __forceinline__ void prep_block(const PrepTable& T, uint32_t b) {
  int j = 0;
  while (j + 1 < T.n && b >= T.p[j + 1].block0) ++j;
  const Prep& a = T.p[j];
  const int64_t block = b - a.block0, base = block * 256, r0 = base / a.per_row;
  const uint32_t c = (uint32_t)(base - r0 * a.per_row) + threadIdx.x, d = c / a.per_row;
  const int64_t row = r0 + d;
  const uint32_t col = (c - d * a.per_row) * 8;
  auto put = [&](int64_t at, const uint32_t* w) {
    *(gmem((u32x4_t*)(a.dst + at * a.per_row * 8 + col))) = u32x4_t{w[0], w[1], w[2], w[3]};
  };
  if (a.e != nullptr) {
    if (row >= a.rows) return;
    const int64_t at = row * a.ld + col;
    const u32x2_t q = *gmem((const u32x2_t*)((const int8_t*)a.src + at));
    const float s = f32_from_bits((uint32_t)gmem(a.e)[at >> 5] << 23);
    const uint32_t u[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};
    uint32_t w[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const uint32_t v = u[h >> 1] >> (16 * (h & 1));
      const uint32_t lo = bits_from_f32(((float)(v & 0xFFu) - 128.0f) * s);
      const uint32_t hi = bits_from_f32(((float)((v >> 8) & 0xFFu) - 128.0f) * s);
      w[h] = lo >> 16 | (hi & 0xFFFF0000u);
    }
    put(row, w);
    return;
  }
  if (row >= a.part) return;
  const int64_t left = row < a.rows ? (int64_t)a.cols - col : 0;
  uint32_t w[4];
  if constexpr (DT == ISO_BF16) {
    const u32x4_t y = load_raw<DT>(a.src, row * a.ld + col, left);
#pragma unroll
    for (int h = 0; h < 4; ++h) w[h] = y[h];
    put(row, w);
  } else {
    uint32_t y[8], p[3][8];
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      const u32x4_t v = load_raw<DT>(a.src, row * a.ld + col + h, left - h);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[h + j] = v[j];
    }
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      const bool finite = (y[h] & 0x7F800000u) != 0x7F800000u;
      uint32_t hi = y[h] & 0xFFFF0000u;
      if (!finite && (y[h] & 0x7FFFFFu)) hi |= 0x400000u;   // a NaN stays one
      float r = finite ? f32_from_bits(y[h]) - f32_from_bits(hi) : 0.0f;
      const uint32_t mid = bits_from_f32(r) & 0xFFFF0000u;
      r -= f32_from_bits(mid);
      p[2][h] = hi, p[1][h] = mid, p[0][h] = bits_from_f32(r);
    }
#pragma unroll
    for (int part = 0; part < 3; ++part) {
#pragma unroll
      for (int h = 0; h < 4; ++h) w[h] = p[part][2 * h] >> 16 | (p[part][2 * h + 1] & 0xFFFF0000u);
      put(part * a.part + row, w);
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(256) k_wgrad_prep(PrepTable T) {
  if (blockIdx.x == 0 && threadIdx.x == 0) *T.status = 0;
  for (uint32_t b = blockIdx.x; b < T.blocks; b += gridDim.x) prep_block<DT>(T, b);
}

// ---- the product ---------------------------------------------------------------------------------------------------

// 32 rows of a wave's part of G from row m, column n on, as it reads and writes them: 16 bytes a lane, whole rows.  `old`
// holds what a lane adds to.
template <int TILE, int DTG>
struct Rows32 {
  static constexpr int V = kVec<DTG>, kLanes = Tile<TILE>::kQuarter / V, kRows = 64 / kLanes, kCount = 32 / kRows;
  u32x4_t old[kCount];

  __device__ __forceinline__ void load(const Layer& a, int m, int n, int lane) {
    const int row = lane / kLanes, c = lane % kLanes * V, left = a.cols - n - c;
#pragma unroll
    for (int h = 0; h < kCount; ++h)
      if (left > 0 && m + h * kRows + row < a.rows)
        old[h] = load_raw<DTG>(a.g, (int64_t)(m + h * kRows + row) * a.cols + n + c, left);
  }

  template <bool ADD>
  __device__ __forceinline__ void store(const Layer& a, int m, int n, uint32_t lds, int lane) const {
    const int row = lane / kLanes, c = lane % kLanes * V, left = a.cols - n - c;
    if (left <= 0) return;
#pragma unroll
    for (int h = 0; h < kCount; ++h) {
      const int r = h * kRows + row;
      if (m + r >= a.rows) continue;
      float v[V];
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const f32x4_t x = *(lds_f32x4)(uintptr_t)(lds + r * Tile<TILE>::kOutBytes + (c + j) * 4);
        v[j] = x.x, v[j + 1] = x.y, v[j + 2] = x.z, v[j + 3] = x.w;
      }
      if constexpr (ADD) {
        float o[V];
        unpack_raw<DTG>(old[h], o);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += o[j];
      }
      store_elems<DTG, V>(a.g, (int64_t)(m + r) * a.cols + n + c, v, left);
    }
  }
};

__device__ __forceinline__ int layer_of(const LayerTable& T, uint32_t tile) {
  int j = 0;
  while (j + 1 < T.n && tile >= T.l[j + 1].tile0) ++j;
  return j;
}

// Origin of a layer's tile: bands of eight tile rows, walked down their columns, so that the 32 tiles an XCD works on
// at once are 8 x 4 and share 12 panels in its L2.
template <int TILE>
__device__ __forceinline__ void tile_origin(const Layer& a, uint32_t tile, int& m0, int& n0) {
  const int t = (int)(tile - a.tile0);
  const int band = t / (8 * a.across), r0 = band * 8, h = min(8, a.down - r0), in = t - r0 * a.across;
  m0 = (r0 + in % h) * TILE;
  n0 = in / h * TILE;
}

// Consecutive pieces of [0, n) for the workgroups of one XCD (workgroup b runs on XCD b % 8).
__device__ __forceinline__ uint32_t by_xcd(uint32_t b, uint32_t n) {
  const uint32_t x = b & 7u, each = n >> 3, more = n & 7u;
  return x * each + min(x, more) + (b >> 3);
}

// One tile of G (or a share of its tokens) a workgroup of four waves, each with a quarter of it in accumulators: 256 registers
// a lane for 256 x 256, 64 for 128 x 128.
//   Steps of 32 tokens go from memory straight into LDS, four stages deep (two panels each, a token's row of 512 or 256
// bytes); both operands have their tokens along the slow dimension, so fragments come through the transposing LDS read,
// 16 lanes a 4 token x 16 column block.  The four 64-byte pieces that the first (or second) half of a wave reads at once
// come from four successive token rows; piece c of row t lies at c ^ (t & 3), which puts the four into different quarters
// of the 64 banks (no conflicts counted), while 64 bytes of memory stay together.
//   The loop is laid out by hand, one LDS read or load between two matrix instructions (1335 -> 1600 TFLOP/s on zeros, 1170 ->
// 1290 on random values at 4096 x 4096 of 8192 tokens): fragments of the next half step are read, and loads issued, under
// the products of the current one.  At the middle of a step all its fragments are in registers: one barrier there frees its
// stage and vouches for the next.
//   Bound by the power that matrix products of random values take (the clock falls to about 1.9 GHz) and the loads' issue.
template <int TILE, int DTG, bool ADD>
__global__ void __launch_bounds__(256, 1) k_wgrad(LayerTable T) {
  using S = Tile<TILE>;
  constexpr int F = S::kFrags, L = S::kLoads, kReads = 4 * F;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  uint32_t tile, piece = 0, pieces = 1;
  if (blockIdx.x < T.whole) {
    tile = by_xcd(blockIdx.x, T.whole);
  } else {
    const uint32_t rest = T.tiles - T.whole, u = by_xcd(blockIdx.x - T.whole, rest * T.split);
    pieces = T.split;
    piece = u / rest;
    tile = T.whole + u - piece * rest;
  }
  const Layer& a = T.l[layer_of(T, tile)];
  int m0, n0;
  tile_origin<TILE>(a, tile, m0, n0);
  const int all = a.steps * a.parts;
  const int first = (int)((int64_t)all * piece / pieces), last = (int)((int64_t)all * (piece + 1) / pieces);
  const int steps = last - first;

  // loads: a wave's 1024 bytes are kAtOnce token rows; load j takes 16-byte column c of row 4 kAtOnce j + row
  constexpr int kAtOnce = 1024 / S::kRowBytes, kAcross = 64 / kAtOnce;
  const int row = w * kAtOnce + lane / kAcross, c = lane % kAcross;
  const uint32_t col = (uint32_t)(((c >> 2) ^ (row & 3)) * 64 + (c & 3) * 16);
  uint32_t vy[L], vx[L];
#pragma unroll
  for (int j = 0; j < L; ++j) {
    vy[j] = (uint32_t)(row + 4 * kAtOnce * j) * (uint32_t)a.y_ld + col;
    vx[j] = (uint32_t)(row + 4 * kAtOnce * j) * (uint32_t)a.x_ld + col;
  }
  const uint8_t* const x_base = a.x + 2 * (int64_t)n0;
  const int64_t x_left0 = a.x_bytes - 2 * (int64_t)n0, y_step = kStep * a.y_ld, x_step = kStep * a.x_ld;
  int x_at = a.steps > 0 ? first % a.steps : 0;
  const uint8_t *yp = a.y + 2 * (int64_t)m0 + first * y_step, *xp = x_base + x_at * x_step;
  int64_t y_left = a.y_bytes - 2 * (int64_t)m0 - first * y_step, x_left = x_left0 - x_at * x_step;
  int to_load = steps;
  u32x4_t yb, xb;
  auto next = [&] {   // descriptors of the next step's panels; empty past the last
    yb = buffer_of(yp, to_load > 0 ? y_left : 0);
    xb = buffer_of(xp, to_load > 0 ? x_left : 0);
    --to_load;
    yp += y_step, y_left -= y_step, xp += x_step, x_left -= x_step;
    if (++x_at == a.steps) x_at = 0, xp = x_base, x_left = x_left0;
  };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_u8*)smem);
  auto load_y = [&](int j, int stage) { load_lds(yb, lds0 + stage * S::kStage + w * 1024 + j * 4096, vy[j]); };
  auto load_x = [&](int j, int stage) { load_lds(xb, lds0 + stage * S::kStage + S::kPanel + w * 1024 + j * 4096, vx[j]); };

  // fragments f of 32 columns: lane's token rows (lane / 32) * 8 ..., columns lane % 32
  const int g = lane >> 4, i = lane & 15;
  uint32_t ay[F], ax[F];
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const uint32_t at = lds0 + ((g >> 1) * 8 + (i >> 2)) * S::kRowBytes + (g & 1) * 32 + (i & 3) * 8;
    ay[f] = at + (((w >> 1) * F + f) ^ (i >> 2)) * 64;
    ax[f] = at + (((w & 1) * F + f) ^ (i >> 2)) * 64 + S::kPanel;
  }
  struct Frag {
    s16x4_t h[2];
  };
  Frag fx[2][F], fy[2][F];
  auto read = [&](int set, int q, uint32_t offset) {   // piece q: x0 y0 y1 ... x1 x2 ..., two halves each
    const int n = q >> 1, h = q & 1;
    const uint32_t at = (n == 0 ? ax[0] : n <= F ? ay[n - 1] : ax[n - F]) + offset + h * (4 * S::kRowBytes);
    const s16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_frag)(uintptr_t)at);
    if (n == 0) fx[set][0].h[h] = v;
    else if (n <= F) fy[set][n - 1].h[h] = v;
    else fx[set][n - F].h[h] = v;
  };
  f32x16_t acc[F][F];
#pragma unroll
  for (int p = 0; p < F; ++p)
#pragma unroll
    for (int q = 0; q < F; ++q) acc[p][q] = 0.0f;
  auto multiply = [&](int set, int q) {
    acc[q / F][q % F] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fx[set][q / F]),
                                                               __builtin_bit_cast(bf16x8_t, fy[set][q % F]),
                                                               acc[q / F][q % F], 0, 0, 0);
  };

  // the last stage's X panel is loaded in the first step
  for (int s = 0; s < kStages; ++s) {
    next();
#pragma unroll
    for (int j = 0; j < L; ++j) load_y(j, s);
    if (s < kStages - 1)
#pragma unroll
      for (int j = 0; j < L; ++j) load_x(j, s);
  }
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * 2 * L + L) : "memory");
#pragma unroll
  for (int q = 0; q < kReads; ++q) read(0, q, 0);
  int stage = 0, before = kStages - 1;
  for (int t = 0; t < steps; ++t) {
    const int after = stage + 1 == kStages ? 0 : stage + 1;
#pragma unroll
    for (int q = 0; q < kReads; ++q) {
      read(1, q, stage * S::kStage + 16 * S::kRowBytes);
      if (q * F % 4 == 0) multiply(0, q * F / 4);
      if ((q & 3) == 1) load_x(q >> 2, before);
      __builtin_amdgcn_sched_barrier(0);
    }
    next();
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 2) * 2 * L) : "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < kReads; ++q) {
      read(0, q, after * S::kStage);
      if (q * F % 4 == 0) multiply(1, q * F / 4);
      if ((q & 3) == 1) load_y(q >> 2, stage);
      __builtin_amdgcn_sched_barrier(0);
    }
    before = stage;
    stage = after;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // no load may reach LDS after the workgroup's end

  // a lane holds four consecutive columns of a row in every four registers
  if (pieces > 1) {
    float* const out = T.part + ((int64_t)(tile - T.whole) * pieces + piece) * (TILE * TILE) + w * (S::kQuarter * S::kQuarter);
#pragma unroll
    for (int q = 0; q < F; ++q)
#pragma unroll
      for (int p = 0; p < F; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          store_elems<ISO_F32, 4>(out, ((q * F + p) * 4 + r) * 256 + lane * 4, (const float*)&acc[p][q] + 4 * r);
    return;
  }
  // through LDS, 32 rows of the wave's quarter at a time, so that memory sees whole rows; where G is added to, the next 32
  // rows of it are under way meanwhile
  const int mw = m0 + (w >> 1) * S::kQuarter, nw = n0 + (w & 1) * S::kQuarter;
  Rows32<TILE, DTG> rows[2];
  if constexpr (ADD) rows[0].load(a, mw, nw, lane);
  asm volatile("s_barrier" ::: "memory");   // every wave is past its last fragment
  const uint32_t own = lds0 + w * (32 * S::kOutBytes);
#pragma unroll
  for (int q = 0; q < F; ++q) {
    if constexpr (ADD)
      if (q + 1 < F) rows[(q + 1) & 1].load(a, mw + q * 32 + 32, nw, lane);
#pragma unroll
    for (int p = 0; p < F; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(lds_f32x4)(uintptr_t)(own + (lane & 31) * S::kOutBytes + (p * 32 + r * 8 + (lane >> 5) * 4) * 4) =
            f32x4_t{acc[p][q][4 * r], acc[p][q][4 * r + 1], acc[p][q][4 * r + 2], acc[p][q][4 * r + 3]};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    rows[q & 1].template store<ADD>(a, mw + q * 32, nw, own, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// Adds up the pieces of the split tiles, in order: a thread four columns of a row.
template <int TILE, int DTG, bool ADD>
__global__ void __launch_bounds__(256) k_wgrad_join(LayerTable T) {
  constexpr int F = Tile<TILE>::kFrags, kQuarter = Tile<TILE>::kQuarter, kBlocks = TILE * TILE / 1024;
  const uint32_t r = blockIdx.x / kBlocks, tile = T.whole + r;
  const Layer& a = T.l[layer_of(T, tile)];
  int m0, n0;
  tile_origin<TILE>(a, tile, m0, n0);
  const int at = (int)(blockIdx.x % kBlocks) * 1024 + threadIdx.x * 4;
  const float* const in = T.part + (int64_t)r * T.split * (TILE * TILE) + at;
  const int w = at / (kQuarter * kQuarter), q = at / (F * 1024) % F, p = at / 1024 % F, h = (at >> 8) & 3, lane = (at >> 2) & 63;
  const int m = m0 + (w >> 1) * kQuarter + q * 32 + (lane & 31);
  const int n = n0 + (w & 1) * kQuarter + p * 32 + h * 8 + (lane >> 5) * 4;
  if (m >= a.rows || n >= a.cols) return;
  float sum[4] = {};
  for (uint32_t s = 0; s < T.split; s += 8) {
    u32x4_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < T.split) v[j] = load_raw<ISO_F32>(in, (int64_t)(s + j) * (TILE * TILE));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < T.split)
#pragma unroll
        for (int h = 0; h < 4; ++h) sum[h] += f32_from_bits(v[j][h]);
  }
  const int64_t to = (int64_t)m * a.cols + n;
  if constexpr (ADD) {
    float old[4];
    load_elems<DTG, 4>(a.g, to, old, a.cols - n);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] += old[j];
  }
  store_elems<DTG, 4>(a.g, to, sum, a.cols - n);
}

// ---- host ----------------------------------------------------------------------------------------------------------

template <int TILE, int DTG, bool ADD>
void launch_tiles(const LayerTable& L, hipStream_t s) {
  // the result passes through LDS too: no more of it than the stages take
  static_assert(4 * 32 * Tile<TILE>::kOutBytes <= kStages * Tile<TILE>::kStage, "result rows fit into the stages");
  const uint32_t rest = L.tiles - L.whole;
  k_wgrad<TILE, DTG, ADD><<<L.whole + rest * L.split, 256, kStages * Tile<TILE>::kStage, s>>>(L);
  if (rest > 0) k_wgrad_join<TILE, DTG, ADD><<<rest * (TILE * TILE / 1024), 256, 0, s>>>(L);
}

template <int DTG, bool ADD>
void launch(const WeightGradPlan& P, hipStream_t s) {
  P.tile == 128 ? launch_tiles<128, DTG, ADD>(P.layers, s) : launch_tiles<256, DTG, ADD>(P.layers, s);
}

}  // namespace

hipError_t run_weight_grad(const iso_weight_grad* g, int n, int dt, int dt_grad, bool accumulate, uint8_t* ws, hipStream_t s) {
  // Launches take up to 16 layers; a repeated gradient cuts one of these short, so that the workspace, which was asked for
  // without a look at the gradients, holds what they need.
  int j = 0, many;
  do {
    many = weight_grad_group(g + j, std::min(kLayers - j % kLayers, n - j), dt_grad);
    const WeightGradPlan P = plan_weight_grad(g + j, many, dt, accumulate, ws);
    const unsigned grid = std::min(std::max(P.prep.blocks, 1u), 1u << 22);
    if (dt == ISO_BF16) k_wgrad_prep<ISO_BF16><<<grid, 256, 0, s>>>(P.prep);
    else k_wgrad_prep<ISO_F32><<<grid, 256, 0, s>>>(P.prep);
    if (P.layers.tiles > 0) {
      if (dt_grad == ISO_BF16) accumulate ? launch<ISO_BF16, true>(P, s) : launch<ISO_BF16, false>(P, s);
      else accumulate ? launch<ISO_F32, true>(P, s) : launch<ISO_F32, false>(P, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    j += many;
  } while (j < n);
  return hipSuccess;
}

}  // namespace iso
