// Norms of query and key heads with their rotation (lv_qk_rotate).
//
// Each element is read and written once, 16 bytes a lane: D / 8 lanes hold a head.
// With x' = x s w (s of the head, w the weight) an element and its partner p give
// x' cos -+ p' sin = s (x A + p B), A = w cos, B = -+ w_p sin, which are the same for all
// heads of a token.  A warp takes a token's heads, or some of them: it forms the angles
// once, two a lane, and a lane its eight A and B; a head then costs the sum of its
// squares among its lanes, the partners by a shuffle of the 16-bit values, and three
// multiplications a pair of elements.  The next heads are asked for meanwhile.
//
// Measured: 8,005 tokens of 32 + 8 heads of 128, bf16, 34 us, 4.8 TB/s (0.71 of the measured
// rate; 209 us for a head a warp through shared memory, 56 with norm, weight and angle
// applied one after another).  Neither memory (0.42 busy) nor the issue slots (0.62) are
// full: about 136 instructions for two heads of a token, which wait for one another's
// shuffles and conversions, and with 95 registers a thread (and 8 bytes in local memory, a
// load a token) there are 20 warps an SM to fill the gaps.
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
  int dim;
  int parts, part;           // warps of a token, heads of a warp (queries first, then keys)
  float eps;
  int *status;
  uint64_t turn[64];         // 2^64 freq / 2 pi: a token on, in 2^-64 of a turn
};

// Request of token t: the last one whose offset is at most t; -1 where t is before the
// first, at `begin`, or past the last one's end.  By a whole warp, 32 ways at a time.
__device__ __forceinline__ int64_t request_of(const int64_t *offsets, int64_t n_req, int64_t begin, int64_t end, int64_t t,
                                              int lane) {
  if (t < begin || t >= end) return -1;
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

constexpr int kRoWarps = 4;  // of a CTA
constexpr int kAsked = 4;    // loads of a lane at a time
constexpr int kRoCtas = 5;   // of an SM

__device__ __forceinline__ float rsqrt_fast(float x) {  // of a normal number
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void swap_pair(uint64_t x, uint64_t *y) {
  float a, b;
  unpair(x, &a, &b);
  *y = pair(b, a);
}
// The eight elements of lane `from`, or zeros: 0 times an infinity would be NaN.
__device__ __forceinline__ uint4 partners(const uint4 &mine, int from, bool turns) {
  uint4 r;
  r.x = __shfl_sync(~0u, mine.x, from);
  r.y = __shfl_sync(~0u, mine.y, from);
  r.z = __shfl_sync(~0u, mine.z, from);
  r.w = __shfl_sync(~0u, mine.w, from);
  return turns ? r : make_uint4(0, 0, 0, 0);
}

template <int D, bool F16, bool NORM, bool NEXT>
__global__ void __launch_bounds__(kRoWarps * 32, kRoCtas) k_rotate(const __grid_constant__ RotateArgs a) {
  constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;  // lanes of a head, heads of a warp at a time
  __shared__ __align__(16) float2 turned[kRoWarps][64];  // a token's cosines and sines
  __shared__ __align__(16) float weight[2][D];
  // An element times its weight is formed before the head's scale is known, and leaves
  // fp32's range where either is extreme (of bf16; fp16's stay within it).  A head whose sum
  // of squares is not within these limits is brought near 1 first.  Up to 2^120 an element
  // is below 2^60, and below 2^128 times a weight of at most 2^64.  An underflow counts where
  // the scale, at most 1 / sqrt(mean + eps), lifts it back: from mean + eps of 2^-24 on it
  // ends below 2^-126 again, whatever the weight; with weights of at least 2^-4, which leave
  // 2^-137 of the least element, it is exact enough down to 2^-97.
  __shared__ float least, most;
  constexpr bool kFar = NORM && !F16;
  if (NORM && threadIdx.x == 0) {
    least = a.eps < 0x1p-60f ? 0x1p-90f : 0.f;
    most = 0x1p120f;
  }
  if (kFar) __syncthreads();  // beside the kernel before
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int l = lane % kLanes, sub = lane / kLanes, heads = a.heads[0] + a.heads[1];
  let_next();
  wait_previous();
  bool bad = false;
  if (a.offsets)
    for (int64_t i = (int64_t)blockIdx.x * (kRoWarps * 32) + threadIdx.x; i < a.n_req; i += (int64_t)gridDim.x * (kRoWarps * 32))
      bad |= a.offsets[i] < 0 || a.offsets[i + 1] < a.offsets[i] || a.offsets[i + 1] > a.n_tok;
  // by halves the lane's eight elements are of pairs first .. first + 7, and their
  // partners another lane's; by neighbours they are pairs first .. first + 3
  const int half_lanes = a.dim / 16;
  const bool turns = l < 2 * half_lanes, upper = !NEXT && l >= half_lanes;
  const int away = !turns || NEXT ? 0 : upper ? -half_lanes : half_lanes;
  const int first = NEXT ? l * 4 : (upper ? l - half_lanes : l) * 8;
  constexpr int kBatch = kAtOnce * kAsked;  // heads that a warp has asked for
  const int64_t units = a.n_tok * a.parts;
  int64_t u = (int64_t)blockIdx.x * kRoWarps + warp, t = 0;
  int at0 = 0, end0 = 0, at1 = 0, end1 = 0;  // the warp's queries, then its keys
  uint4 next[kAsked];
  auto ask = [&](int w, int from) {
    const uint16_t *const x = (const uint16_t *)a.x[w] + t * a.x_stride[w] + (from + sub) * D + l * 8;
    const int end = w ? end1 : end0;
#pragma unroll
    for (int b = 0; b < kAsked; ++b) {
      next[b] = make_uint4(0, 0, 0, 0);
      if (from + b * kAtOnce + sub < end) next[b] = *(const uint4 *)(x + b * kAtOnce * D);
    }
  };
  auto begin = [&] {  // unit u: its heads, and the first of them asked for
    t = a.parts == 1 ? u : quotient(u, a.parts);
    const int h0 = (int)(u - t * a.parts) * a.part, h1 = min(h0 + a.part, heads);
    at0 = min(h0, a.heads[0]), end0 = min(h1, a.heads[0]);
    at1 = max(h0 - a.heads[0], 0), end1 = max(h1 - a.heads[0], 0);
    ask(at0 < end0 ? 0 : 1, at0 < end0 ? at0 : at1);
  };
  if (u < units) begin();
  const int64_t begin_tok = a.offsets ? a.offsets[0] : 0, end_tok = a.offsets ? a.offsets[a.n_req] : 0;
  for (int k = threadIdx.x; k < 2 * D; k += kRoWarps * 32) {
    const void *const w = k < D ? a.weight[0] : a.weight[1];
    const float v = w ? value_of<F16>(((const uint16_t *)w)[k % D]) : 1.f;
    weight[k / D][k % D] = v;
    // whoever writes a limit writes the same
    if (kFar && fabsf(v) > 0x1p64f) most = 0.f;
    if (kFar && v != 0.f && fabsf(v) < 0x1p-4f && a.eps < 0x1p-24f) least = D * 0x1p-24f;
  }
  __syncthreads();
  for (bool begun = true; u < units; u += (int64_t)gridDim.x * kRoWarps, begun = false) {
    if (!begun) begin();
    const int64_t i = a.offsets ? request_of(a.offsets, a.n_req, begin_tok, end_tok, t, lane) : t;
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
#pragma unroll 1
    for (int w = 0; w < 2; ++w) {
      const int at = w ? at1 : at0, end = w ? end1 : end0;
      if (at >= end) continue;
      uint64_t A[4], B[4];
      // the lane's weights and its partners', and the pairs' cosines and sines, 16 bytes a load
      const float4 *const own = (const float4 *)(weight[w] + l * 8), *const theirs = own + away * 2;
      const float4 *const angle = (const float4 *)(turned[warp] + (first & 63));
#pragma unroll
      for (int k = 0; k < 8; k += 4) {
        const float4 x = own[k / 4];
        if (NEXT) {
          float4 e = make_float4(1.f, 0.f, 1.f, 0.f);
          if (turns) e = angle[k / 4];
          A[k / 2] = pair(x.x * e.x, x.y * e.x), A[k / 2 + 1] = pair(x.z * e.z, x.w * e.z);
          B[k / 2] = turns ? pair(x.y * -e.y, x.x * e.y) : 0;
          B[k / 2 + 1] = turns ? pair(x.w * -e.w, x.z * e.w) : 0;
        } else {
          float4 e = make_float4(1.f, 0.f, 1.f, 0.f), f = e;
          if (turns) e = angle[k / 2], f = angle[k / 2 + 1];
          float4 p = make_float4(0.f, 0.f, 0.f, 0.f);  // nothing of a weight that is infinite
          if (turns) p = theirs[k / 4];
          if (!upper) p.x = -p.x, p.y = -p.y, p.z = -p.z, p.w = -p.w;
          A[k / 2] = pair(x.x * e.x, x.y * e.z), A[k / 2 + 1] = pair(x.z * f.x, x.w * f.z);
          B[k / 2] = pair(p.x * e.y, p.y * e.w), B[k / 2 + 1] = pair(p.z * f.y, p.w * f.w);
        }
      }
      const bool normed = NORM && a.weight[w];
      uint16_t *y = (uint16_t *)a.y[w] + t * a.y_stride[w] + (at + sub) * D + l * 8;
#pragma unroll 1
      for (int from = at; from < end; from += kBatch, y += kBatch * D) {
        uint4 raw[kAsked];
#pragma unroll
        for (int b = 0; b < kAsked; ++b) raw[b] = next[b];
        if (from + kBatch < end)
          ask(w, from + kBatch);
        else if (w == 0)
          ask(1, at1);
        // a head's outputs, its elements multiplied by `by` first
        auto turn = [&](int b, float by, float scale) {
          uint64_t v[4], o[4];
          unpack_pairs<F16>(raw[b], v);
          if (NEXT) {
#pragma unroll
            for (int k = 0; k < 4; ++k) swap_pair(turns ? v[k] : 0, &o[k]);
          } else {
            unpack_pairs<F16>(partners(raw[b], lane + away, turns), o);
          }
          uint32_t r[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (by != 1.f) v[k] = mul2(v[k], pair(by, by)), o[k] = mul2(o[k], pair(by, by));
            float p, q;
            const uint64_t z = fma2(v[k], A[k], mul2(o[k], B[k]));
            unpair(normed ? mul2(z, pair(scale, scale)) : z, &p, &q);
            r[k] = pack_out<F16>(p, q);
          }
          if (from + b * kAtOnce + sub < end) *(uint4 *)(y + b * kAtOnce * D) = make_uint4(r[0], r[1], r[2], r[3]);
        };
        float sum[kAsked];
        bool far = false;
        if (normed) {
#pragma unroll
          for (int b = 0; b < kAsked; ++b) {
            uint64_t v[4], s2;
            unpack_pairs<F16>(raw[b], v);
            s2 = mul2(v[0], v[0]);
#pragma unroll
            for (int k = 1; k < 4; ++k) s2 = fma2(v[k], v[k], s2);
            float s1;
            unpair(s2, &sum[b], &s1);
            sum[b] += s1;
          }
#pragma unroll
          for (int s = kLanes / 2; s; s >>= 1)
#pragma unroll
            for (int b = 0; b < kAsked; ++b) sum[b] += __shfl_xor_sync(~0u, sum[b], s);
          const float low = least, high = most;
#pragma unroll
          for (int b = 0; b < kAsked; ++b)
            far |= from + b * kAtOnce + sub < end && (!(sum[b] < high) || sum[b] < low);
        }
        if (__any_sync(~0u, far)) {
#pragma unroll
          for (int b = 0; b < kAsked; ++b) {
            // The squares again, relative to a power of two above twice the largest element (so
            // that two of them times a weight are within range), or to eps where that is larger
            // still: what is far below either does not count
            float e8[8], top = 0.f, again = 0.f, by = 1.f, eps = a.eps;
            unpack8<F16>(raw[b], e8);
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(e8[k]));
#pragma unroll
            for (int s = kLanes / 2; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, s));
            if (top > 0.f && top < INFINITY)
              by = scalbnf(1.f, -2 - max(max(ilogbf(top), eps > 0.f ? ilogbf(eps) / 2 : -126), -126));
#pragma unroll
            for (int k = 0; k < 8; ++k) again += e8[k] * by * (e8[k] * by);
#pragma unroll
            for (int s = kLanes / 2; s; s >>= 1) again += __shfl_xor_sync(~0u, again, s);
            turn(b, by, rsqrtf(again * (1.f / D) + eps * by * by));
          }
        } else {
#pragma unroll
          for (int b = 0; b < kAsked; ++b) turn(b, 1.f, normed ? rsqrt_fast(sum[b] * (1.f / D) + a.eps) : 1.f);
        }
      }
    }
  }
  if (bad) flag(a.status, kStatusData);
}

}  // namespace lv
