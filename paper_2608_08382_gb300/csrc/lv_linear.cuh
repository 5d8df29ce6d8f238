// Products of a step's tokens with a layer's weights (lv_linear, lv_gated_linear).
#pragma once

#include "lv_attend.cuh"

namespace lv {

struct LinearArgs {
  const void *x, *w[2];      // w[1]: the gated form's second weights
  const void *bias[2];
  const void *residual;
  void *y;
  int64_t x_stride, w_stride, r_stride, y_stride;
  int64_t n_tok;
  int d_in, d_out, act;
  int *status;
};

template <bool F16>
__device__ __forceinline__ float value_of(uint16_t b) {
  return F16 ? __half2float(__ushort_as_half(b)) : __uint_as_float((uint32_t)b << 16);
}

// The activation in fp32.  1 + exp(-x) is infinite where x is below -88: x over it is
// then -0 where the exact value is above -1e-36, and below every normal number of the
// 16-bit types.  The two forms of GELU are written without the difference of nearly
// equal numbers that 1 + erf and 1 + tanh have at the left: erfc, and 1 + tanh u =
// 2 / (1 + exp(-2u)).
__device__ __forceinline__ float activated(float x, int act) {
  switch (act) {
    case LV_ACT_SILU: return x / (1.f + __expf(-x));
    case LV_ACT_GELU: return 0.5f * x * erfcf(x * -0.70710678118654752f);
    case LV_ACT_GELU_TANH: return x / (1.f + __expf(-1.5957691216057308f * (x + 0.044715f * x * x * x)));
    case LV_ACT_RELU: return x < 0.f ? 0.f : x;
    default: return x;
  }
}

// Each CTA forms 64 tokens by 64 outputs, a thread 4 by 4 of them, 16 terms a step
// through shared memory in fp32.
constexpr int kLinTile = 64, kLinStep = 16;

template <bool GATED, bool F16>
__global__ void __launch_bounds__(256) k_linear(const LinearArgs a) {
  constexpr int kW = GATED ? 2 : 1;
  __shared__ float xs[kLinStep][kLinTile + 1], ws[kW][kLinStep][kLinTile + 1];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int across = (a.d_out + kLinTile - 1) / kLinTile;
  const int64_t t0 = (int64_t)(blockIdx.x / across) * kLinTile;
  const int o0 = (int)(blockIdx.x % across) * kLinTile;
  float sum[kW][4][4] = {};
  for (int i0 = 0; i0 < a.d_in; i0 += kLinStep) {
    for (int e = threadIdx.x; e < kLinTile * kLinStep; e += 256) {
      const int r = e / kLinStep, i = e % kLinStep;
      const bool in = i0 + i < a.d_in;
      xs[i][r] = in && t0 + r < a.n_tok ? value_of<F16>(((const uint16_t *)a.x)[(t0 + r) * a.x_stride + i0 + i]) : 0.f;
      for (int k = 0; k < kW; ++k)
        ws[k][i][r] = in && o0 + r < a.d_out ? value_of<F16>(((const uint16_t *)a.w[k])[(o0 + r) * a.w_stride + i0 + i]) : 0.f;
    }
    __syncthreads();
    for (int i = 0; i < kLinStep; ++i)
#pragma unroll
      for (int k = 0; k < kW; ++k)
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
          for (int q = 0; q < 4; ++q) sum[k][p][q] += xs[i][ty + 16 * p] * ws[k][i][tx + 16 * q];
    __syncthreads();
  }
#pragma unroll
  for (int p = 0; p < 4; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t t = t0 + ty + 16 * p;
      const int o = o0 + tx + 16 * q;
      if (t >= a.n_tok || o >= a.d_out) continue;
      float v[kW];
      for (int k = 0; k < kW; ++k) v[k] = sum[k][p][q] + (a.bias[k] ? value_of<F16>(((const uint16_t *)a.bias[k])[o]) : 0.f);
      float y = activated(v[0], a.act);
      if (GATED) y *= v[kW - 1];
      if (a.residual) y += value_of<F16>(((const uint16_t *)a.residual)[t * a.r_stride + o]);
      ((uint16_t *)a.y)[t * a.y_stride + o] = (uint16_t)pack_out<F16>(y, 0.f);
    }
}

}  // namespace lv
