// New keys and values appended to a cache held in e4m3 with a scale for each
// block and head (lv_kv_store).
//
// A run is the new tokens of one block: they stand next to each other, and a
// token begins one where its slot is a block's first or does not follow the slot
// before it.  One warp does a run's keys or values of one head: the largest
// magnitude, the scale 2^e, the codes; where the scale of a block with tokens in
// it grows it also rounds those again.
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

template <int D, bool F16>
__global__ void __launch_bounds__(256) k_kv_store(StoreArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int per = 2 * a.heads;
  const int64_t t0 = unit / per;
  if (t0 >= a.n_tok) return;
  const int h = (int)(unit % per) >> 1, kv = (int)unit & 1;
  const int64_t B = 1ll << a.log_b, slot = a.slots[t0];
  if (slot < 0) return;
  const int64_t blk = slot >> a.log_b, off = slot & (B - 1);
  if (blk >= a.n_blocks) {
    flag(a.status, kStatusData);
    return;
  }
  if (off != 0 && t0 > 0 && a.slots[t0 - 1] == slot - 1) return;  // inside a run
  // the run's length
  int n = 1;
  while (off + n < B && t0 + n < a.n_tok && a.slots[t0 + n] == slot + n) ++n;
  constexpr int kPart = D / 32;  // elements of a lane
  const uint16_t *x = reinterpret_cast<const uint16_t *>(a.x[kv]) + (int64_t)h * D + lane * kPart;
  auto load = [&](int64_t t, float *v) {
#pragma unroll
    for (int k = 0; k < kPart; k += 2) {
      const float2 f = unpack2<F16>(*reinterpret_cast<const uint32_t *>(x + t * a.stride[kv] + k));
      v[k] = f.x;
      v[k + 1] = f.y;
    }
  };
  float amax = 0.f;
  for (int j = 0; j < n; ++j) {
    float v[kPart];
    load(t0 + j, v);
#pragma unroll
    for (int k = 0; k < kPart; ++k)
      if (fabsf(v[k]) <= 3.4028235e38f) amax = fmaxf(amax, fabsf(v[k]));
  }
  for (int d = 16; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
  float *sp = a.scale[kv] + blk * a.heads + h;
  uint8_t *code = a.code[kv] + ((blk * a.heads + h) << a.log_b) * D;
  float s = pow2_scale(amax);
  if (off > 0) {
    const float old = *sp;
    if (old >= s) {
      s = old;
    } else {
      const float r = old / s;
      for (int64_t i = lane; i < off * D; i += 32) {
        __nv_fp8_e4m3 q;
        q.__x = code[i];
        code[i] = (uint8_t)encode4((float)q * r, 0.f, 0.f, 0.f);
      }
    }
  }
  __syncwarp();
  if (lane == 0) *sp = s;
  for (int j = 0; j < n; ++j) {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    load(t0 + j, v);
#pragma unroll
    for (int k = 0; k < kPart; ++k) v[k] = no_inf(v[k] / s);
    const uint32_t q = encode4(v[0], v[1], v[2], v[3]);
    uint8_t *to = code + (off + j) * D + lane * kPart;
    if (kPart == 4)
      *reinterpret_cast<uint32_t *>(to) = q;
    else
      *reinterpret_cast<uint16_t *>(to) = (uint16_t)q;
  }
}

}  // namespace lv
