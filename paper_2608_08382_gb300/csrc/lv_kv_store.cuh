// New keys and values appended to a cache held in e4m3 with a scale for each
// block and head (lv_kv_store).
//
// A run is the new tokens of one block: they stand next to each other, and a
// token begins one where its slot is a block's first or does not follow the slot
// before it.  One warp does a run's keys or values of one head: the largest
// magnitude, the scale 2^e, the codes; where the scale of a block with tokens in
// it grows it also rounds those again.  16 bytes a load, a run of up to 16 tokens
// of 128 stays in registers between the two steps: memory is read and written
// once, and that bounds all but small calls.
//
// A CTA looks through a window of tokens for the runs that begin there and deals
// them out, run by run and head by head, to its warps.  The window is small where
// there are few tokens (a step of single tokens: every one is a run).
//
// Measured: 32,768 tokens of packed prompts, 8 heads of 128, 201 MB: 40 us, 5.1 TB/s,
// 0.75 of the copy rate, the rest instructions and the windows' beginnings (windows of
// 16 tokens 43, CTAs of 4 warps 42, three CTAs an SM 44); 2,048 single tokens, 4 heads:
// 11.6 us in a graph, 15 as a call.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "lv_base.cuh"

namespace lv {

struct StoreArgs {
  const void *x[2];  // keys, values
  int64_t stride[2];
  uint8_t *code[2];
  float *scale[2];
  const int64_t *slots;
  int64_t n_tok, n_blocks;
  int log_b, heads;
  int *status;
};

// Two 16-bit floats as fp32.
template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t u) {
  if (F16) return __half22float2(*reinterpret_cast<__half2 *>(&u));
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}

// The least power of two s >= 2^-100 with amax <= 448 s (448 = 1.75 * 2^8 is the
// largest e4m3 value): the exponent of amax less 8, one more where its mantissa
// is above 1.75.
__device__ __forceinline__ float pow2_scale(float amax) {
  const uint32_t b = __float_as_uint(amax);
  int e = (int)(b >> 23) - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);
  e = max(e, 127 - 100);
  return __uint_as_float((uint32_t)e << 23);
}

// e4m3 of four values of at most 448 (nearest even; NaN and infinities to NaN).
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

__device__ __forceinline__ float no_inf(float x) { return isinf(x) ? __int_as_float(0x7fffffff) : x; }

constexpr int kStoreWarps = 8;
constexpr int kStoreWindow = 32;  // tokens of a window, at most
constexpr int kStoreRun = 128;    // tokens of a run, at most: a block's

// Products and quotients that a rounding to e4m3 follows, under a scale that is no
// power of two: cut, with the last bit set where something was cut off, so that the
// two roundings together are one.
__device__ __forceinline__ float odd_product(float a, float b) {
  const float p = __fmul_rz(a, b);
  return __fmaf_rn(a, b, -p) != 0.f ? __uint_as_float(__float_as_uint(p) | 1) : p;
}
__device__ __forceinline__ float odd_quotient(float a, float b) {
  const float q = __fdiv_rz(a, b);
  return __fmaf_rn(-q, b, a) != 0.f ? __uint_as_float(__float_as_uint(q) | 1) : q;
}

// The larger ones of two pairs of 16 bits.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Four codes as fp32.
__device__ __forceinline__ void decode4(uint32_t q, float *v) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)q));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(q >> 16)));
  const float2 a = __half22float2(*reinterpret_cast<__half2 *>(&lo)), b = __half22float2(*reinterpret_cast<__half2 *>(&hi));
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}

template <int D, bool F16>
__global__ void __launch_bounds__(kStoreWarps * 32, 4) k_kv_store(StoreArgs a, int window) {
  constexpr int kLanes = D / 8, kRows = 32 / kLanes;   // lanes of a token, tokens of a load
  constexpr int kHeld = 16 / kRows;                    // loads of 16 tokens
  __shared__ int64_t slot[kStoreWindow + kStoreRun];
  __shared__ int run_at[kStoreWindow], run_n[kStoreWindow], runs;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t0 = (int64_t)blockIdx.x * window, B = 1ll << a.log_b, cap = a.n_blocks << a.log_b;
  // slots of the window and as far as a run of it may go; what is not in the cache is -1
  bool bad = false;
  const int look = (int)min(a.n_tok - t0, (int64_t)window + (B - 1));
  for (int i = threadIdx.x; i < look; i += kStoreWarps * 32) {
    int64_t s = a.slots[t0 + i];
    if (s >= cap) {
      bad |= i < window;
      s = -1;
    }
    slot[i] = s;
  }
  __syncthreads();
  if (warp == 0) {
    // the runs that begin in the window
    bool begins = false;
    if (lane < window && lane < look && slot[lane] >= 0) {
      const int64_t s = slot[lane], before = lane > 0 ? slot[lane - 1] : t0 > 0 ? a.slots[t0 - 1] : -1;
      begins = (s & (B - 1)) == 0 || before != s - 1;
    }
    const unsigned all = __ballot_sync(~0u, begins);
    if (begins) {
      const int k = __popc(all & ((1u << lane) - 1));
      int n = 1;
      while (lane + n < look && slot[lane + n] == slot[lane] + n && (slot[lane + n] & (B - 1)) != 0) ++n;
      run_at[k] = lane;
      run_n[k] = n;
    }
    if (lane == 0) runs = __popc(all);
  }
  __syncthreads();
  const int per = 2 * a.heads, items = runs * per;
  const int sub = lane % kLanes, of = lane / kLanes;
  for (int item = warp; item < items; item += kStoreWarps) {
    const int run = item / per, h = (item % per) >> 1, kv = item & 1, n = run_n[run];
    const int64_t s0 = slot[run_at[run]], blk = s0 >> a.log_b, off = s0 & (B - 1);
    const int64_t stride = kv ? a.stride[1] : a.stride[0];
    float *sp = (kv ? a.scale[1] : a.scale[0]) + blk * a.heads + h;
    const float old = off > 0 ? *sp : 0.f;
    const uint16_t *x = reinterpret_cast<const uint16_t *>(kv ? a.x[1] : a.x[0]) +
                        (t0 + run_at[run] + of) * stride + (int64_t)h * D + sub * 8;
    uint4 v[kHeld];
    auto load = [&](int from) {
      const uint16_t *y = x + from * stride;
#pragma unroll
      for (int k = 0; k < kHeld; ++k, y += kRows * stride)
        v[k] = from + k * kRows + of < n ? *reinterpret_cast<const uint4 *>(y) : make_uint4(0, 0, 0, 0);
    };
    // the largest magnitude by its bits, two elements at a time; where it is not
    // finite, once more over those that are
    uint32_t top = 0;
    for (int from = 0; from < n; from += 16) {
      load(from);
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (from + k * kRows >= n) break;
        top = max2(max2(top, v[k].x & 0x7fff7fff), max2(v[k].y & 0x7fff7fff, max2(v[k].z & 0x7fff7fff, v[k].w & 0x7fff7fff)));
      }
    }
    top = __reduce_max_sync(~0u, max(top & 0xffff, top >> 16));
    const uint32_t infinite = F16 ? 0x7c00 : 0x7f80;
    const bool all_finite = top < infinite;
    if (!all_finite) {
      top = 0;
#pragma unroll 1
      for (int j = 0; j + of < n; j += kRows) {
        const uint4 y = *reinterpret_cast<const uint4 *>(x + j * stride);
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const uint32_t lo = w[z] & 0x7fff, hi = w[z] >> 16 & 0x7fff;
          top = max(top, max(lo < infinite ? lo : 0, hi < infinite ? hi : 0));
        }
      }
      top = __reduce_max_sync(~0u, top);
    }
    const float amax = unpack2<F16>(top).x;
    uint8_t *const code = (kv ? a.code[1] : a.code[0]) + ((blk * a.heads + h) << a.log_b) * D;
    float s = pow2_scale(amax);
    if (off > 0) {
      if (old >= s) {
        s = old;
      } else {
        const float r = old / s;
        for (int64_t i = lane * 16; i < off * D; i += 512) {
          uint4 q = *reinterpret_cast<const uint4 *>(code + i);
          uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            float f[4];
            decode4(w[y], f);
            w[y] = encode4(odd_product(f[0], r), odd_product(f[1], r), odd_product(f[2], r), odd_product(f[3], r));
          }
          *reinterpret_cast<uint4 *>(code + i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
    if (lane == 0) *sp = s;
    // Eight codes of a lane.  By a power of two a product is the quotient; the longer
    // way is for a scale of another kind (the caller's own) and values that are not
    // finite, and kept out of the loop that all else takes (with both in one loop 52 us
    // for what takes 40).
    uint8_t *to = code + (off + of) * D + sub * 8;
    const float inv = 1.f / s;
    if (all_finite && (__float_as_uint(s) & 0x7fffff) == 0) {
      for (int from = 0; from < n; from += 16) {
        if (n > 16) load(from);
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
          const float2 p0 = unpack2<F16>(v[k].x), p1 = unpack2<F16>(v[k].y), p2 = unpack2<F16>(v[k].z), p3 = unpack2<F16>(v[k].w);
          if (from + k * kRows + of < n)
            *reinterpret_cast<uint2 *>(to + (from + k * kRows) * D) =
                make_uint2(encode4(p0.x * inv, p0.y * inv, p1.x * inv, p1.y * inv),
                           encode4(p2.x * inv, p2.y * inv, p3.x * inv, p3.y * inv));
        }
      }
    } else {
#pragma unroll 1
      for (int j = 0; j + of < n; j += kRows) {
        const uint4 y = *reinterpret_cast<const uint4 *>(x + j * stride);
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
        float f[8];
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const float2 p = unpack2<F16>(w[z]);
          f[2 * z] = no_inf(odd_quotient(p.x, s)), f[2 * z + 1] = no_inf(odd_quotient(p.y, s));
        }
        *reinterpret_cast<uint2 *>(to + j * D) = make_uint2(encode4(f[0], f[1], f[2], f[3]), encode4(f[4], f[5], f[6], f[7]));
      }
    }
  }
  if (bad) flag(a.status, kStatusData);
}

}  // namespace lv
