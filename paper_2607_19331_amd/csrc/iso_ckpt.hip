// 8-bit activation checkpoints: packing, unpacking, and the gated activation's backward pass from them.
//
// A group of 32 columns of a row shares 2^k, the least power of two with max|x| <= 127 2^k (k >= -126); q = rne(x / 2^k).
// Why a power of two: x / 2^k and q 2^k are exact, so the only rounding is the one to an integer, and q 2^k (7 bits times
// a power of two that is no denormal) is a bf16 value: the weight gradient's matrix instructions take it as it is.  A
// scale max|x| / 127 would use up to one bit more of q, and every use would then round again.
// Why int8 and not an 8-bit float with the same exponents: three bits of significand leave 2^-4 of each value, against
// at most 2^-7 of the group's largest here; activations of one token in 32 neighbouring channels are of one order.
//
// All three are bound by the bytes: each reads its inputs and writes its outputs once (4096 tokens of a 7B layer's activations,
// 277e6 values in bf16: packed in 133 to 145 us, 5.8 to 6.3 TB/s, unpacked in 143 to 159; the gate's gradients of 8192 x 18944 in
// 205 us, 6.1 TB/s).  A lane holds eight neighbouring
// columns (16 bytes of bf16, 8 bytes of q), four lanes a group; q and e are written in their own order, contiguously.
// Tables of tensors go to the kernel as an argument, up to 16 a launch, so a call copies nothing from the host.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "iso.h"
#include "iso_device.h"
#include "iso_grad.h"
#include "iso_grad_device.h"

namespace iso {

namespace {

// Groups of eight columns a thread: 4096 tokens of a 7B layer's activations there and back take 327, 298 and 309 us with
// one, two and four (outputs kept in the caches), the gate's gradients of 8192 x 18944 213, 222 and 229 us.
constexpr int kItems = 2;
constexpr int kGateItems = 1;

struct CkptArg {
  int8_t* q;
  uint8_t* e;
  void* x;
  int64_t rows, ld_x;
  uint32_t cols, per_row;      // columns; groups of eight in a row of q
};

struct CkptTable {
  CkptArg t[kTable];
  uint32_t block0[kTable + 1];
  int n;
};

struct GateArg {
  const int8_t *gq, *uq;
  const uint8_t *ge, *ue;
  const void* dh;
  void *dgate, *dup;
  int64_t rows, ld;
  uint32_t cols, per_row;
};

struct GateTable {
  GateArg t[kTable];
  uint32_t block0[kTable + 1];
  int n;
};

template <class Table>
__device__ __forceinline__ int table_entry(const Table& T) {
  int j = 0;
  while (j + 1 < T.n && blockIdx.x >= T.block0[j + 1]) ++j;
  return j;
}

// Where the items of this thread lie: item i of a tensor is group of eight i % per_row of row i / per_row.
struct Place {
  int64_t row;
  uint32_t c8;
};
template <int ITEMS>
__device__ __forceinline__ Place place(int64_t block, uint32_t per_row, int q) {
  const int64_t base = block * (256 * ITEMS), r0 = base / per_row;
  const uint32_t c = (uint32_t)(base - r0 * per_row) + q * 256 + threadIdx.x, d = c / per_row;
  return Place{r0 + d, c - d * per_row};
}

// Exponent byte of a group from the bits of its largest magnitude: max|x| = m 2^E <= 127 2^k iff k >= E - 6 where
// m <= 127/64, E - 5 otherwise; the sum carries into the exponent exactly where the significand is past that of 127.
__device__ __forceinline__ uint32_t exponent_of(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const int e = (int)((top + 0x1FFFFu) >> 23) - 6;
  return (uint32_t)max(e, 1);
}

// Eight stored values: q 2^(e - 127); e = 255 gives 0 Inf, a NaN.  A byte biased by 128 converts unsigned in one
// instruction; the bias comes off before the scale, for 128 2^k overflows where q 2^k does not.
__device__ __forceinline__ void stored8(uint2 q, uint32_t e, float v[8]) {
  const float s = f32_from_bits(e << 23);
  const uint32_t w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = ((float)((w[j / 4] >> (8 * (j & 3))) & 0xFFu) - 128.0f) * s;
}

template <int DT, bool STREAM>
__global__ void __launch_bounds__(256) k_ckpt_pack(CkptTable T) {
  const int j = table_entry(T);
  const CkptArg& a = T.t[j];
  const int64_t block = blockIdx.x - T.block0[j];
  float v[kItems][8];
  Place p[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    p[i] = place<kItems>(block, a.per_row, i);
    const uint32_t col = p[i].c8 * 8;
    const uint32_t left = p[i].row < a.rows && col < a.cols ? a.cols - col : 0u;
    load_elems<DT, 8>(a.x, p[i].row * a.ld_x + col, v[i], (int64_t)left);
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    uint32_t top = 0;
#pragma unroll
    for (int h = 0; h < 8; ++h) top = max(top, bits_from_f32(v[i][h]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t e = exponent_of(top);
    // adding 1.5 2^23 rounds to an integer (nearest even) and leaves it in the low byte as two's complement
    const float inv = f32_from_bits((254u - min(e, 254u)) << 23);
    if (e == 249u) {   // 64 2^122 is no finite number
      const float lim = 63.0f * f32_from_bits(249u << 23);
#pragma unroll
      for (int h = 0; h < 8; ++h) v[i][h] = fminf(fmaxf(v[i][h], -lim), lim);
    }
    uint32_t w[8];
#pragma unroll
    for (int h = 0; h < 8; ++h)
      w[h] = e == 255u ? 0u : bits_from_f32(__builtin_fmaf(v[i][h], inv, 12582912.0f)) & 0xFFu;
    if (p[i].row >= a.rows) continue;
    const int64_t item = p[i].row * a.per_row + p[i].c8;
    const u32x2_t out = {w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24, w[4] | w[5] << 8 | w[6] << 16 | w[7] << 24};
    if constexpr (STREAM) __builtin_nontemporal_store(out, gmem((u32x2_t*)a.q) + item);
    else *(gmem((u32x2_t*)a.q) + item) = out;
    if ((p[i].c8 & 3u) == 0) gmem(a.e)[item >> 2] = (uint8_t)e;
  }
}

template <int DT, bool STREAM>
__global__ void __launch_bounds__(256) k_ckpt_unpack(CkptTable T) {
  const int j = table_entry(T);
  const CkptArg& a = T.t[j];
  const int64_t block = blockIdx.x - T.block0[j];
  u32x2_t q[kItems];
  uint32_t e[kItems];
  Place p[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    p[i] = place<kItems>(block, a.per_row, i);
    if (p[i].row >= a.rows) continue;
    const int64_t item = p[i].row * a.per_row + p[i].c8;
    q[i] = *(gmem((const u32x2_t*)a.q) + item);
    e[i] = gmem((const uint8_t*)a.e)[item >> 2];
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const uint32_t col = p[i].c8 * 8;
    if (p[i].row >= a.rows || col >= a.cols) continue;
    float v[8];
    stored8(make_uint2(q[i].x, q[i].y), e[i], v);
    store_elems<DT, 8, STREAM>(a.x, p[i].row * a.ld_x + col, v, a.cols - col);
  }
}

// sigmoid(g).  bf16 results take the hardware's exponential and reciprocal (relative error about 2^-21 where the
// sigmoid is not negligible, against the 2^-9 of their rounding), fp32 ones the full-precision functions.
template <int DT>
__device__ __forceinline__ float sigmoid_of(float g) {
  if constexpr (DT == ISO_BF16) return __builtin_amdgcn_rcpf(1.0f + __expf(-g));
  else return 1.0f / (1.0f + expf(-g));
}

template <int DT, bool STREAM>
__global__ void __launch_bounds__(256) k_gate_grad(GateTable T) {
  const int j = table_entry(T);
  const GateArg& a = T.t[j];
  const int64_t block = blockIdx.x - T.block0[j];
  u32x2_t gq[kGateItems], uq[kGateItems];
  uint32_t ge[kGateItems], ue[kGateItems];
  float dh[kGateItems][8];
  Place p[kGateItems];
#pragma unroll
  for (int i = 0; i < kGateItems; ++i) {
    p[i] = place<kGateItems>(block, a.per_row, i);
    const uint32_t col = p[i].c8 * 8;
    if (p[i].row >= a.rows || col >= a.cols) continue;
    const int64_t item = p[i].row * a.per_row + p[i].c8;
    gq[i] = *(gmem((const u32x2_t*)a.gq) + item);
    uq[i] = *(gmem((const u32x2_t*)a.uq) + item);
    ge[i] = gmem(a.ge)[item >> 2];
    ue[i] = gmem(a.ue)[item >> 2];
    load_elems<DT, 8>(a.dh, p[i].row * a.ld + col, dh[i], a.cols - col);
  }
#pragma unroll
  for (int i = 0; i < kGateItems; ++i) {
    const uint32_t col = p[i].c8 * 8;
    if (p[i].row >= a.rows || col >= a.cols) continue;
    float g[8], u[8];
    stored8(make_uint2(gq[i].x, gq[i].y), ge[i], g);
    stored8(make_uint2(uq[i].x, uq[i].y), ue[i], u);
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      const float s = sigmoid_of<DT>(g[h]), d = dh[i][h];
      const float silu = g[h] * s;
      g[h] = d * u[h] * (s * (1.0f + g[h] * (1.0f - s)));
      u[h] = d * silu;
    }
    const int64_t at = p[i].row * a.ld + col;
    store_elems<DT, 8, STREAM>(a.dgate, at, g, a.cols - col);
    store_elems<DT, 8, STREAM>(a.dup, at, u, a.cols - col);
  }
}

CkptArg arg_of(const iso_ckpt& c) {
  return CkptArg{c.q, c.e, c.x, c.rows, c.ld_x, (uint32_t)c.cols, (uint32_t)(ckpt_ld(c.cols) / 8)};
}
GateArg arg_of(const iso_gate_grad& g) {
  return GateArg{g.gate.q, g.up.q,    g.gate.e, g.up.e, g.dh, g.dgate, g.dup, g.gate.rows, g.ld, (uint32_t)g.gate.cols,
                 (uint32_t)(ckpt_ld(g.gate.cols) / 8)};
}

// Queues a table.
template <class Table, class Entry, class Launch>
hipError_t run_tables(const Entry* c, int n, int items, int size, Launch launch) {
  for_tables<Table>(c, n, items, size, [](const Entry& x) { return arg_of(x); },
                    [&](const Table& T, unsigned grid, int64_t bytes) { launch(T, grid, streamed(bytes)); });
  return hipGetLastError();
}

}  // namespace

hipError_t run_ckpt_pack(const iso_ckpt* c, int n, int dt, hipStream_t s) {
  return run_tables<CkptTable>(c, n, kItems, 8, [&](const CkptTable& T, unsigned grid, bool stream) {
    auto go = [&](auto k) { k<<<grid, 256, 0, s>>>(T); };
    if (dt == ISO_BF16) stream ? go(k_ckpt_pack<ISO_BF16, true>) : go(k_ckpt_pack<ISO_BF16, false>);
    else stream ? go(k_ckpt_pack<ISO_F32, true>) : go(k_ckpt_pack<ISO_F32, false>);
  });
}

hipError_t run_ckpt_unpack(const iso_ckpt* c, int n, int dt, hipStream_t s) {
  return run_tables<CkptTable>(c, n, kItems, dt == ISO_BF16 ? 16 : 32, [&](const CkptTable& T, unsigned grid, bool stream) {
    auto go = [&](auto k) { k<<<grid, 256, 0, s>>>(T); };
    if (dt == ISO_BF16) stream ? go(k_ckpt_unpack<ISO_BF16, true>) : go(k_ckpt_unpack<ISO_BF16, false>);
    else stream ? go(k_ckpt_unpack<ISO_F32, true>) : go(k_ckpt_unpack<ISO_F32, false>);
  });
}

hipError_t run_gate_grad(const iso_gate_grad* g, int n, int dt, hipStream_t s) {
  return run_tables<GateTable>(g, n, kGateItems, dt == ISO_BF16 ? 32 : 64, [&](const GateTable& T, unsigned grid, bool stream) {
    auto go = [&](auto k) { k<<<grid, 256, 0, s>>>(T); };
    if (dt == ISO_BF16) stream ? go(k_gate_grad<ISO_BF16, true>) : go(k_gate_grad<ISO_BF16, false>);
    else stream ? go(k_gate_grad<ISO_F32, true>) : go(k_gate_grad<ISO_F32, false>);
  });
}

}  // namespace iso
