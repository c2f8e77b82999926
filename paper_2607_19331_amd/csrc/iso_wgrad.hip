// Weight gradients of linear layers from 8-bit activation checkpoints: G = [G +] dY^T X, X[t, i] = q 2^k.
//
// X is exact in bf16, so the products of a bf16 dY are exact and bf16 matrix instructions with binary32 accumulators
// lose nothing but the sum's own rounding; a binary32 dY is the sum of three bf16 parts of 8 bits each (cut, not
// rounded: every remainder is exact), which gives three products with the same X.
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

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct Job {
  const int8_t* q;
  const uint8_t* e;
  const void* dy;
  void* grad;
  int64_t tokens, ld_dy, ld_q;
  int32_t rows, cols;
};

constexpr int kTile = 64, kStep = 32, kLd = kStep + 8;

// One 64 x 64 tile of G a workgroup, four waves of 32 x 32; a step of 32 tokens is staged in LDS token-innermost.
template <int DT, int DTG, bool ADD>
__global__ void __launch_bounds__(256) k_wgrad(Job a) {
  constexpr int kParts = DT == ISO_F32 ? 3 : 1;
  __shared__ uint16_t A[kParts][kTile][kLd], B[kTile][kLd];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t across = (a.cols + kTile - 1) / kTile;
  const int64_t m0 = blockIdx.x / across * kTile, n0 = blockIdx.x % across * kTile;
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
  f32x4_t acc[2][2] = {};
  for (int64_t t0 = 0; t0 < a.tokens; t0 += kStep) {
    __syncthreads();
    for (int i = tid; i < kTile * kStep; i += 256) {
      const int c = i & 63, t = i >> 6;
      const int64_t tok = t0 + t, m = m0 + c, n = n0 + c;
      uint32_t y = 0, x = 0;
      if (tok < a.tokens && m < a.rows) y = elem_bits<DT>(a.dy, tok * a.ld_dy + m);
      if (tok < a.tokens && n < a.cols)
        x = bits_from_f32((float)a.q[tok * a.ld_q + n] * f32_from_bits((uint32_t)a.e[(tok * a.ld_q + n) >> 5] << 23));
      B[c][t] = (uint16_t)(x >> 16);
      if constexpr (DT == ISO_BF16) {
        A[0][c][t] = (uint16_t)y;
      } else {
        const bool finite = (y & 0x7F800000u) != 0x7F800000u;
        float r = f32_from_bits(y);
        uint32_t hi = y & 0xFFFF0000u;
        if (!finite && (y & 0x7FFFFFu)) hi |= 0x400000u;   // a NaN stays one
        r = finite ? r - f32_from_bits(hi) : 0.0f;
        const uint32_t mid = bits_from_f32(r) & 0xFFFF0000u;
        r -= f32_from_bits(mid);
        A[0][c][t] = (uint16_t)(hi >> 16);
        A[1][c][t] = (uint16_t)(mid >> 16);
        A[2][c][t] = (uint16_t)(bits_from_f32(r) >> 16);
      }
    }
    __syncthreads();
    const int k = (lane >> 4) * 8, r = lane & 15;
    bf16x8_t b[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) b[j] = *(const bf16x8_t*)&B[wn + 16 * j + r][k];
#pragma unroll
    for (int p = kParts - 1; p >= 0; --p)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf16x8_t x = *(const bf16x8_t*)&A[p][wm + 16 * i + r][k];
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, b[j], acc[i][j], 0, 0, 0);
      }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int64_t m = m0 + wm + 16 * i + (lane >> 4) * 4 + h, n = n0 + wn + 16 * j + (lane & 15);
        if (m >= a.rows || n >= a.cols) continue;
        float g = acc[i][j][h];
        if constexpr (ADD) {
          float o;
          load_elems<DTG, 1>(a.grad, m * a.cols + n, &o);
          g += o;
        }
        store_elems<DTG, 1>(a.grad, m * a.cols + n, &g);
      }
}

}  // namespace

size_t weight_grad_workspace_bytes(const iso_weight_grad*, int, int) { return kStatusBytes; }

hipError_t run_weight_grad(const iso_weight_grad* g, int n, int dt, int dt_grad, bool accumulate, uint8_t* ws,
                           hipStream_t s) {
  const hipError_t e = fill_u32((uint32_t*)ws, kStatusBytes / 4, 0u, s);
  if (e != hipSuccess) return e;
  for (int j = 0; j < n; ++j) {
    const iso_weight_grad& x = g[j];
    if (x.rows == 0 || x.in.cols == 0) continue;
    const Job a{x.in.q, x.in.e, x.dy, x.grad, x.in.rows, x.ld_dy, ckpt_ld(x.in.cols), (int32_t)x.rows, (int32_t)x.in.cols};
    const unsigned grid = (unsigned)(((x.in.cols + kTile - 1) / kTile) * ((x.rows + kTile - 1) / kTile));
    auto go = [&](auto k) { k<<<grid, 256, 0, s>>>(a); };
    if (dt == ISO_BF16 && dt_grad == ISO_BF16) accumulate ? go(k_wgrad<ISO_BF16, ISO_BF16, true>) : go(k_wgrad<ISO_BF16, ISO_BF16, false>);
    else if (dt == ISO_BF16) accumulate ? go(k_wgrad<ISO_BF16, ISO_F32, true>) : go(k_wgrad<ISO_BF16, ISO_F32, false>);
    else if (dt_grad == ISO_BF16) accumulate ? go(k_wgrad<ISO_F32, ISO_BF16, true>) : go(k_wgrad<ISO_F32, ISO_BF16, false>);
    else accumulate ? go(k_wgrad<ISO_F32, ISO_F32, true>) : go(k_wgrad<ISO_F32, ISO_F32, false>);
  }
  return hipGetLastError();
}

}  // namespace iso
