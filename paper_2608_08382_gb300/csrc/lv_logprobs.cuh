// Log probabilities of given tokens, entropy and the largest logits
// (lv_token_logprobs): with m the row's largest logit, S = sum exp(x - m) and
// W = sum exp(x - m) (x - m),
//   lse = m + log S,  log p_v = (x_v - m) - log S,  entropy = log S - W / S.
#pragma once

#include "lv_linear.cuh"

namespace lv {

struct LogprobArgs {
  const void *x;
  int64_t stride, n_tok;
  int vocab, n_top;
  const int32_t *ids;
  float *logp, *entropy, *lse;
  int32_t *top_ids;
  float *top_logp;
  int *status;
};

constexpr int kTypeF32 = LV_F32;

template <int TYPE>
__device__ __forceinline__ float logit_at(const void *x, int64_t at) {
  if (TYPE == kTypeF32) return ((const float *)x)[at];
  return value_of<TYPE == LV_F16>(((const uint16_t *)x)[at]);
}

// Keys in the order of the logits: unsigned 32-bit numbers that compare as the values
// do, the two zeros alike and a NaN above everything but the number that no key has.
constexpr uint32_t kNanKey = 0xfffffffeu;
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // -0 + 0 = 0
  if (v != v) return kNanKey;
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  if (k == kNanKey) return NAN;
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// With the index: of equal values the lowest index is the largest.  0 is below all.
__device__ __forceinline__ uint64_t full_key(uint32_t key, uint32_t index) { return (uint64_t)key << 32 | (uint32_t)~index; }

template <class T, class F>
__device__ __forceinline__ T block_join(T v, T *room, F f) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v = f(v, __shfl_xor_sync(~0u, v, s));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  v = room[0];
  for (int k = 1; k < (int)blockDim.x / 32; ++k) v = f(v, room[k]);
  return v;
}

// A CTA a row: a pass for the maximum, one for the sums, one for each of the largest.
template <int TYPE>
__global__ void __launch_bounds__(256) k_logprobs(const LogprobArgs a) {
  __shared__ uint64_t keys[8];
  __shared__ float sums[8];
  auto larger = [](uint64_t p, uint64_t q) { return p > q ? p : q; };
  auto add = [](float p, float q) { return p + q; };
  for (int64_t t = blockIdx.x; t < a.n_tok; t += gridDim.x) {
    const int64_t at = t * a.stride;
    uint64_t best = 0;
    for (int v = threadIdx.x; v < a.vocab; v += 256) best = larger(best, full_key(order_key(logit_at<TYPE>(a.x, at + v)), v));
    best = block_join(best, keys, larger);
    const float m = key_value((uint32_t)(best >> 32));
    float S = 0.f, W = 0.f;
    for (int v = threadIdx.x; v < a.vocab; v += 256) {
      const float d = logit_at<TYPE>(a.x, at + v) - m, e = __expf(d);
      S += e;
      if (e != 0.f) W += e * d;
    }
    S = block_join(S, sums, add);
    W = block_join(W, sums, add);
    const bool none = m == -INFINITY;
    const float log_s = logf(S);
    if (threadIdx.x == 0) {
      if (a.lse) a.lse[t] = m == INFINITY || none ? m : m + log_s;
      if (a.entropy) a.entropy[t] = none ? 0.f : log_s - W / S;
      if (a.logp) {
        const int id = a.ids[t];
        float lp = NAN;
        if (id >= 0 && id < a.vocab) {
          const float x = logit_at<TYPE>(a.x, at + id);
          lp = none ? m : m == INFINITY ? x - m : (x - m) - log_s;
        } else if (id != -1) {
          flag(a.status, kStatusData);
        }
        a.logp[t] = lp;
      }
    }
    uint64_t below = ~0ull;
    for (int k = 0; k < a.n_top; ++k) {
      uint64_t next = 0;
      for (int v = threadIdx.x; v < a.vocab; v += 256) {
        const uint64_t key = full_key(order_key(logit_at<TYPE>(a.x, at + v)), v);
        if (key < below) next = larger(next, key);
      }
      below = next = block_join(next, keys, larger);
      if (threadIdx.x == 0) {
        const float x = key_value((uint32_t)(next >> 32));
        a.top_ids[t * a.n_top + k] = next ? (int32_t)~(uint32_t)next : -1;
        a.top_logp[t * a.n_top + k] = !next || none ? -INFINITY : m == INFINITY ? x - m : (x - m) - log_s;
      }
    }
  }
}

}  // namespace lv
