// Norms of query and key heads with their rotation (lv_qk_rotate).
//
// Each element is read and written once, 16 bytes a lane: D / 8 lanes hold a head.
// The squares of a head are added up among them; a pair of elements that stand apart
// (halves) is brought together by a shuffle.  Cosines and sines are the same for all
// heads of a token: a warp forms them once, two a lane, for the heads that it takes,
// and keeps those that a lane's elements need in registers.
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
  int parts, part;           // warps of a token, heads of a warp (queries first, then keys)
  float eps;
  int *status;
  uint64_t turn[64];         // 2^64 freq / 2 pi: a token on, in 2^-64 of a turn
};

// Request of token t: the last one whose offset is at most t; -1 where t is before the
// first or past the last.  By a whole warp, 32 ways at a time.
__device__ __forceinline__ int64_t request_of(const int64_t *offsets, int64_t n_req, int64_t t, int lane) {
  if (t < offsets[0] || t >= offsets[n_req]) return -1;
  int64_t lo = 0, hi = n_req;  // offsets[lo] <= t < offsets[hi]
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 32) / 33, at = lo + (lane + 1) * step;
    const unsigned below = __ballot_sync(~0u, at < hi && offsets[at] <= t);
    // where offsets decrease the first lane that is not below ends the search
    const int n = below == ~0u ? 32 : __ffs(~below) - 1;
    const int64_t from = lo + n * step;
    if (n < 32) hi = min(hi, from + step);
    lo = from;
  }
  return lo;
}

// cos and sin of a turn's fraction.  n * turn[j] wraps at whole turns, so the angle of
// any position is reduced exactly; what is left, in [-1/2, 1/2) turns, is rounded to
// 24 bits once.
__device__ __forceinline__ float2 angle_of(uint64_t turns) {
  float2 r;
  sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &r.y, &r.x);
  return r;
}

constexpr int kRoWarps = 4;  // of a CTA; nothing among them
constexpr int kAsked = 4;    // loads of a lane at a time

template <int D, bool F16>
__global__ void __launch_bounds__(kRoWarps * 32) k_rotate(const __grid_constant__ RotateArgs a) {
  constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;  // lanes of a head, heads of a warp at a time
  __shared__ float2 turned[kRoWarps][64];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int l = lane % kLanes, sub = lane / kLanes;
  let_next();
  wait_previous();
  bool bad = false;
  if (a.offsets)
    for (int64_t i = (int64_t)blockIdx.x * (kRoWarps * 32) + threadIdx.x; i < a.n_req; i += (int64_t)gridDim.x * (kRoWarps * 32))
      bad |= a.offsets[i] < 0 || a.offsets[i + 1] < a.offsets[i] || a.offsets[i + 1] > a.n_tok;
  const bool normed = a.weight[0] || a.weight[1];
  uint4 weight[2];  // the lane's eight, of queries and keys
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    uint32_t packed[4] = {};
    if (a.weight[w])
#pragma unroll
      for (int k = 0; k < 8; ++k) packed[k >> 1] |= (uint32_t)((const uint16_t *)a.weight[w])[l * 8 + k] << (k & 1) * 16;
    weight[w] = make_uint4(packed[0], packed[1], packed[2], packed[3]);
  }
  // the lane's elements in a rotation by halves: its own and its partner's are pairs
  // first .. first + 7
  const int turn_lanes = a.dim / 8, half_lanes = turn_lanes / 2;
  const bool turns = l < turn_lanes, upper = l >= half_lanes;
  const int partner = !turns || a.neighbours ? lane : upper ? lane - half_lanes : lane + half_lanes;
  const int first = a.neighbours ? l * 4 : (upper ? l - half_lanes : l) * 8;
  const int64_t units = a.n_tok * a.parts;
  for (int64_t u = (int64_t)blockIdx.x * kRoWarps + warp; u < units; u += (int64_t)gridDim.x * kRoWarps) {
    const int64_t t = a.parts == 1 ? u : quotient(u, a.parts);
    const int h0 = (int)(u - t * a.parts) * a.part, h1 = min(h0 + a.part, a.heads[0] + a.heads[1]);
    const int64_t i = a.offsets ? request_of(a.offsets, a.n_req, t, lane) : t;
    if (i < 0) continue;
    int64_t pos = a.offsets ? t - a.offsets[i] : 0;
    if (a.c) {
      const int c = a.c[i];
      bad |= c < 0;
      pos += max(c, 0);
    }
    __syncwarp();
    for (int j = lane; j < a.dim / 2; j += 32) turned[warp][j] = angle_of((uint64_t)pos * a.turn[j]);
    __syncwarp();
    float2 cs[8];  // by neighbours four of them
    if (turns) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        cs[k] = turned[warp][(first + k) & 63];
        if (!a.neighbours && !upper) cs[k].y = -cs[k].y;  // a cos - b sin below, b cos + a sin above
      }
    }
    for (int g0 = h0; g0 < h1; g0 += kAtOnce * kAsked) {
      uint4 raw[kAsked];
#pragma unroll
      for (int b = 0; b < kAsked; ++b) {
        const int h = g0 + b * kAtOnce + sub, which = h >= a.heads[0];
        raw[b] = make_uint4(0, 0, 0, 0);
        if (h < h1)
          raw[b] = *(const uint4 *)((const uint16_t *)a.x[which] + t * a.x_stride[which] +
                                    (int64_t)(which ? h - a.heads[0] : h) * D + l * 8);
      }
#pragma unroll
      for (int b = 0; b < kAsked; ++b) {
        if (g0 + b * kAtOnce >= h1) break;
        const int h = g0 + b * kAtOnce + sub, which = h >= a.heads[0];
        float v[8];
        unpack8<F16>(raw[b], v);
        if (normed) {
          const bool own_norm = a.weight[which] != nullptr;
          float sum = 0.f, eps = a.eps;
#pragma unroll
          for (int k = 0; k < 8; ++k) sum += v[k] * v[k];
#pragma unroll
          for (int s = kLanes / 2; s; s >>= 1) sum += __shfl_xor_sync(~0u, sum, s);
          const bool far = !(sum < 0x1p120f) || (sum < 0x1p-90f && eps < 0x1p-60f);
          if (__any_sync(~0u, far)) {
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(v[k]));
#pragma unroll
            for (int s = kLanes / 2; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
            // The squares again, relative to a power of two near the largest element, or to
            // eps where that is larger still: what is far below either does not count
            const bool again = far && own_norm && top > 0.f && top < INFINITY;
            const int e = max(max(ilogbf(again ? top : 1.f), eps > 0.f ? ilogbf(eps) / 2 : -126), -126);
            const float by = again ? scalbnf(1.f, -e) : 1.f;
            float other = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              v[k] *= by;
              other += v[k] * v[k];
            }
#pragma unroll
            for (int s = kLanes / 2; s; s >>= 1) other += __shfl_xor_sync(~0u, other, s);
            if (again) {
              sum = other;
              eps = eps * by * by;
            }
          }
          if (own_norm) {
            const float scale = rsqrtf(sum * (1.f / D) + eps);
            float w[8];
            unpack8<F16>(which ? weight[1] : weight[0], w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = v[k] * scale * w[k];
          }
        }
        if (a.neighbours) {
          if (turns)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float p = v[2 * k], q = v[2 * k + 1];
              v[2 * k] = p * cs[k].x - q * cs[k].y;
              v[2 * k + 1] = p * cs[k].y + q * cs[k].x;
            }
        } else if (a.dim > 0) {
          float other[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) other[k] = __shfl_sync(~0u, v[k], partner);
          if (turns)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = v[k] * cs[k].x + other[k] * cs[k].y;
        }
        if (h < h1)
          *(uint4 *)((uint16_t *)a.y[which] + t * a.y_stride[which] + (int64_t)(which ? h - a.heads[0] : h) * D + l * 8) =
              make_uint4(pack_out<F16>(v[0], v[1]), pack_out<F16>(v[2], v[3]), pack_out<F16>(v[4], v[5]),
                         pack_out<F16>(v[6], v[7]));
      }
    }
  }
  if (bad) flag(a.status, kStatusData);
}

}  // namespace lv
