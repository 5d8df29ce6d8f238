// Norms of query and key heads with their rotation (lv_qk_rotate).
#pragma once

#include "lv_linear.cuh"

namespace lv {

struct RotateArgs {
  const void *x[2];          // queries, keys
  void *y[2];
  const void *weight[2];     // or null: no norm
  int64_t x_stride[2], y_stride[2];
  int64_t n_tok;
  const int64_t *offsets;    // or null: one token a request
  const int32_t *c;          // or null
  int64_t n_req;
  int heads[2];
  int dim, neighbours;
  float eps;
  int *status;
  uint64_t turn[64];         // 2^64 freq / 2 pi: a token on, in 2^-64 of a turn
};

// Request of token t: the last one whose offset is at most t; -1 where t is before the
// first or past the last.
__device__ __forceinline__ int64_t request_of(const int64_t *offsets, int64_t n_req, int64_t t) {
  if (t < offsets[0] || t >= offsets[n_req]) return -1;
  int64_t lo = 0, hi = n_req;  // offsets[lo] <= t < offsets[hi]
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) >> 1;
    if (offsets[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// cos and sin of a turn's fraction.  n * turn[j] wraps at whole turns, so the angle of
// any position is reduced exactly; what is left, in [-1/2, 1/2) turns, is rounded to
// 24 bits once.
__device__ __forceinline__ void angle_of(uint64_t turns, float *cos, float *sin) {
  sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, sin, cos);
}

// A warp takes one head of one token, D / 32 elements a lane, through shared memory.
template <int D, bool F16>
__global__ void __launch_bounds__(128) k_rotate(const __grid_constant__ RotateArgs a) {
  constexpr int kPer = D / 32;
  __shared__ float rows[4][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float *const row = rows[warp];
  const int64_t heads = a.heads[0] + a.heads[1], items = a.n_tok * heads;
  bool bad = false;
  if (a.offsets)
    for (int64_t i = (int64_t)blockIdx.x * 128 + threadIdx.x; i < a.n_req; i += (int64_t)gridDim.x * 128)
      bad |= a.offsets[i] < 0 || a.offsets[i + 1] < a.offsets[i] || a.offsets[i + 1] > a.n_tok;
  for (int64_t u = (int64_t)blockIdx.x * 4 + warp; u < items; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / heads;
    int h = (int)(u % heads);
    const int which = h >= a.heads[0];
    if (which) h -= a.heads[0];
    const int64_t i = a.offsets ? request_of(a.offsets, a.n_req, t) : t;
    if (i < 0) continue;
    int64_t pos = a.offsets ? t - a.offsets[i] : 0;
    if (a.c) {
      const int c = a.c[i];
      bad |= c < 0;
      pos += max(c, 0);
    }
    const uint16_t *x = (const uint16_t *)a.x[which] + t * a.x_stride[which] + (int64_t)h * D;
    float v[kPer], sum = 0.f, top = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      v[k] = value_of<F16>(x[lane + 32 * k]);
      sum += v[k] * v[k];
      top = fmaxf(top, fabsf(v[k]));
    }
    if (a.weight[which]) {
#pragma unroll
      for (int s = 16; s; s >>= 1) {
        sum += __shfl_xor_sync(~0u, sum, s);
        top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
      }
      float by = 1.f, eps = a.eps;
      if ((!(sum < 0x1p120f) || (sum < 0x1p-90f && eps < 0x1p-60f)) && top > 0.f && top < INFINITY) {
        // The squares again, relative to a power of two near the largest element, or to
        // eps where that is larger still: what is far below either does not count
        const int e = max(max(ilogbf(top), eps > 0.f ? ilogbf(eps) / 2 : -126), -126);
        by = scalbnf(1.f, -e);
        eps = eps * by * by;
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < kPer; ++k) sum += v[k] * by * (v[k] * by);
#pragma unroll
        for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(~0u, sum, s);
      }
      const float r = 1.f / sqrtf(sum / D + eps);
#pragma unroll
      for (int k = 0; k < kPer; ++k) v[k] = v[k] * by * r * value_of<F16>(((const uint16_t *)a.weight[which])[lane + 32 * k]);
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kPer; ++k) row[lane + 32 * k] = v[k];
    __syncwarp();
    for (int j = lane; j < a.dim / 2; j += 32) {
      const int m = a.neighbours ? 2 * j : j, n = a.neighbours ? 2 * j + 1 : j + a.dim / 2;
      float cos, sin;
      angle_of((uint64_t)pos * a.turn[j], &cos, &sin);
      const float p = row[m], q = row[n];
      row[m] = p * cos - q * sin;
      row[n] = p * sin + q * cos;
    }
    __syncwarp();
    uint16_t *y = (uint16_t *)a.y[which] + t * a.y_stride[which] + (int64_t)h * D;
#pragma unroll
    for (int k = 0; k < kPer; ++k) y[lane + 32 * k] = (uint16_t)pack_out<F16>(row[lane + 32 * k], 0.f);
  }
  if (bad) flag(a.status, kStatusData);
}

}  // namespace lv
