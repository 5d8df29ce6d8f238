// Attention over the cache (lv_kv_attend) and over whole prompts
// (lv_prompt_attend): o = softmax(scale q K^T) V with the running maximum m and
// sum l of the row, o and l scaled by exp(m_old - m_new) where m grows.
#pragma once

#include "lv_kv_store.cuh"

namespace lv {

struct CacheView {
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  int64_t n_blocks;
  int log_b, heads;
};

struct AttendArgs {
  CacheView cache;          // lv_kv_attend
  const void *q, *k, *v;    // k, v: lv_prompt_attend
  int64_t q_stride, k_stride, v_stride;
  int64_t n_tok;
  const int64_t *offsets;   // [n_req + 1], or null: one query a request
  const int32_t *c;
  int64_t n_req;
  const int32_t *table;
  int64_t width;
  int hq, hkv;
  float scale;              // of q . k, for exp2: includes log2(e)
  void *o;
  float *lse;
  int *status;
};

// One warp per (token, query head), a lane holds D / 32 elements.
template <int D, bool F16, bool PAGED>
__global__ void __launch_bounds__(128) k_attend_rows(AttendArgs a) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int64_t t = row / a.hq;
  const int h = (int)(row % a.hq), g = h / (a.hq / a.hkv);
  if (t >= a.n_tok) return;
  // the request of token t
  int64_t i = t, first = t;
  if (a.offsets) {
    int64_t found = -1;
    bool bad = false;
    for (int64_t r = lane; r < a.n_req; r += 32) {
      const int64_t x0 = a.offsets[r], x1 = a.offsets[r + 1];
      if (x0 < 0 || x1 < x0 || x1 > a.n_tok)
        bad = true;
      else if (x0 <= t && t < x1)
        found = r;
    }
    if (bad) flag(a.status, kStatusData);
    for (int d = 16; d; d >>= 1) found = max(found, (int64_t)__shfl_xor_sync(~0u, found, d));
    if (found < 0) return;
    i = found;
    first = a.offsets[i];
  }
  float q[E], o[E];
  const uint16_t *qp = (const uint16_t *)a.q + t * a.q_stride + h * D + lane * E;
#pragma unroll
  for (int k = 0; k < E; k += 2) {
    const float2 f = unpack2<F16>(*(const uint32_t *)(qp + k));
    q[k] = f.x * a.scale, q[k + 1] = f.y * a.scale;
    o[k] = o[k + 1] = 0.f;
  }
  int64_t n = t - first + 1;
  if (PAGED) {
    const int32_t c = a.c[i];
    n = c < 0 ? 0 : n + c;
    if (c < 0 || n > (a.width << a.cache.log_b)) {
      flag(a.status, kStatusData);
      n = min(n, a.width << a.cache.log_b);
    }
  }
  float m = -INFINITY, l = 0.f;
  for (int64_t j = 0; j < n; ++j) {
    float kf[E], vf[E];
    if (PAGED) {
      const CacheView &cv = a.cache;
      const int32_t b = a.table[i * a.width + (j >> cv.log_b)];
      if (b < 0 || b >= cv.n_blocks) {
        if (b != -1) flag(a.status, kStatusData);
        continue;
      }
      const int64_t bh = (int64_t)b * cv.heads + g;
      const int64_t at = ((bh << cv.log_b) + (j & ((1 << cv.log_b) - 1))) * D + lane * E;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        __nv_fp8_e4m3 x;
        x.__x = cv.k[at + k];
        kf[k] = (float)x * cv.k_scale[bh];
        x.__x = cv.v[at + k];
        vf[k] = (float)x * cv.v_scale[bh];
      }
    } else {
      const uint16_t *kp = (const uint16_t *)a.k + (first + j) * a.k_stride + g * D + lane * E;
      const uint16_t *vp = (const uint16_t *)a.v + (first + j) * a.v_stride + g * D + lane * E;
#pragma unroll
      for (int k = 0; k < E; k += 2) {
        float2 f = unpack2<F16>(*(const uint32_t *)(kp + k));
        kf[k] = f.x, kf[k + 1] = f.y;
        f = unpack2<F16>(*(const uint32_t *)(vp + k));
        vf[k] = f.x, vf[k + 1] = f.y;
      }
    }
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) s += q[k] * kf[k];
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn;
    const float up = exp2f(m - base), w = exp2f(s - base);
    l = l * up + w;
#pragma unroll
    for (int k = 0; k < E; ++k) o[k] = o[k] * up + w * vf[k];
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;  // a NaN stays
  uint16_t *op = (uint16_t *)a.o + (t * a.hq + h) * D + lane * E;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    if (F16)
      ((__half *)op)[k] = __float2half_rn(o[k] * inv);
    else
      ((__nv_bfloat16 *)op)[k] = __float2bfloat16_rn(o[k] * inv);
  }
  if (a.lse && lane == 0) a.lse[t * a.hq + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace lv
