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

// Over the cache a weight w meets its value as w vs / ref in fp16, vs the value scale
// of the key's block and ref the largest so far: a scale far below ref takes bits
// from its weights, though ref may be of keys whose values are zeros.  Beyond 2^-15
// of the largest weight a row is done again alone (redo_row).  A scale of at most
// kLeastScale, the least that an append sets and so a block of zeros, brings nothing.
constexpr float kLeastScale = 0x1p-100f;
// ref is never below the normal range, where its reciprocal could be infinite.
constexpr float kLeastRef = 0x1p-126f;

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

template <bool F16>
__device__ __forceinline__ uint32_t pack_out(float a, float b) {
  if (F16) return pack_half2(a, b);
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// 64 bytes in a row: whole sectors at a time where the address allows it.
__device__ __forceinline__ void store64(void *p, const uint32_t *w, bool wide) {
  if (wide) {
#pragma unroll
    for (int k = 0; k < 16; k += 8)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"((uint32_t *)p + k), "r"(w[k]),
                   "r"(w[k + 1]), "r"(w[k + 2]), "r"(w[k + 3]), "r"(w[k + 4]), "r"(w[k + 5]), "r"(w[k + 6]), "r"(w[k + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < 16; k += 4) *reinterpret_cast<uint4 *>((uint32_t *)p + k) = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
  }
}

// a / b for 0 <= a, 0 < b: a 64-bit division is a long chain of instructions, and
// hardly ever needed.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Running sums of units(k), k < n <= kScan, by a block of T threads, into
// S[0 .. n], from base up; returns the last.  A thread takes neighbours, no more
// than there must be, and asks for all of them before it adds up any.
constexpr int kScan = 1024;  // requests whose running sums fit in shared memory

template <int T, class F>
__device__ __forceinline__ int64_t scan_units(int n, int64_t *S, int64_t base, F units) {
  constexpr int kPer = (kScan + T - 1) / T;
  __shared__ int64_t warp_sum[T / 32];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, per = (n + T - 1) / T;
  int64_t u[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = tid * per + k;
    u[k] = k < per && i < n ? units(i) : 0;
    sum += u[k];
  }
  int64_t x = sum;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, x, s);
    if (lane >= s) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sum[w] = x;
  __syncthreads();
  int64_t total = 0, before = 0;
#pragma unroll
  for (int k = 0; k < T / 32; ++k) {
    if (k < w) before += warp_sum[k];
    total += warp_sum[k];
  }
  x += base + before - sum;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = tid * per + k;
    if (k < per && i < n) S[i] = x;
    x += u[k];
  }
  if (tid == 0) S[n] = base + total;
  __syncthreads();
  return base + total;
}

// The request whose range of the running sums S[0 .. n] holds u.
__device__ __forceinline__ int64_t find_unit(const int64_t *S, int64_t n, int64_t u) {
  int64_t i = 0;
  while (n - i > 1) {
    const int64_t m = (i + n) >> 1;
    if (S[m] <= u) i = m; else n = m;
  }
  return i;
}

// Row (query t, head h) of request i, whose tokens start at `first`, once more by
// one warp, key by key over the first n keys, in fp32 alone.  With `all` false,
// where the row came out with a NaN that is not its own.  The rows of a tile see
// different numbers of keys, and a NaN or infinity among the values that only later
// rows see reaches the others through a weight of zero.  So first it is looked
// whether there is one in the up to 144 keys from n on, below `bound`, that the
// tile's products went over; and the walk ends early where the row's own keys
// explain what it has.  With `all` true, where its value scales lie so far apart
// that a weight in 16 bits may have been lost.  The largest score first: a weight is
// at most 1, and an infinite value is not scaled by zero on its way.
template <int D, bool PAGED>
__device__ __forceinline__ int64_t value_place(const AttendArgs &a, int64_t first, int64_t i, int g, int64_t j, int64_t *bh) {
  if (!PAGED) return (first + j) * a.v_stride + (int64_t)g * D;
  const CacheView &cv = a.cache;
  const int32_t b = a.table[i * a.width + (j >> cv.log_b)];
  if (b < 0 || b >= cv.n_blocks) return -1;
  *bh = (int64_t)b * cv.heads + g;
  return ((*bh << cv.log_b) + (j & ((1 << cv.log_b) - 1))) * D;
}

template <int D, bool F16, bool PAGED>
__device__ __noinline__ void redo_row(const AttendArgs &a, int64_t first, int64_t i, int64_t t, int h, int64_t n, int64_t bound, bool all = false) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, g = h / (a.hq / a.hkv);
  const CacheView &cv = a.cache;
  auto value = [&](int64_t at, int64_t bh, float *v) {
    if (PAGED) {
#pragma unroll
      for (int k = 0; k < E; ++k) {
        __nv_fp8_e4m3 e;
        e.__x = cv.v[at + lane * E + k];
        v[k] = (float)e * cv.v_scale[bh];
      }
    } else {
#pragma unroll
      for (int k = 0; k < E; k += 2) {
        const float2 y = unpack2<F16>(*(const uint32_t *)((const uint16_t *)a.v + at + lane * E + k));
        v[k] = y.x, v[k + 1] = y.y;
      }
    }
  };
  bool odd = all;
  for (int64_t j = n; !all && j < min(n + 144, bound); ++j) {
    int64_t bh = 0;
    const int64_t at = value_place<D, PAGED>(a, first, i, g, j, &bh);
    if (at < 0) continue;
    float v[E];
    value(at, bh, v);
#pragma unroll
    for (int k = 0; k < E; ++k) odd |= !isfinite(v[k]);
  }
  if (!__any_sync(~0u, odd)) return;
  const uint16_t *qp = (const uint16_t *)a.q + t * a.q_stride + h * D + lane * E;
  uint16_t *op = (uint16_t *)a.o + (t * a.hq + h) * D + lane * E;
  float q[E], o[E];
  bool has[E];  // what came out as NaN and is not explained yet
#pragma unroll
  for (int k = 0; k < E; k += 2) {
    const float2 f = unpack2<F16>(*(const uint32_t *)(qp + k)), y = unpack2<F16>(*(const uint32_t *)(op + k));
    q[k] = f.x * a.scale, q[k + 1] = f.y * a.scale;
    has[k] = isnan(y.x), has[k + 1] = isnan(y.y);
    o[k] = o[k + 1] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int pass = 0; pass < 2; ++pass)
    for (int64_t j = 0; j < n; ++j) {
      int64_t bh = 0;
      const int64_t at = value_place<D, PAGED>(a, first, i, g, j, &bh);
      if (at < 0) continue;
      float x = 0.f, v[E];
      value(at, bh, v);
      if (PAGED) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
          __nv_fp8_e4m3 e;
          e.__x = cv.k[at + lane * E + k];
          x += q[k] * (float)e;
        }
        x *= cv.k_scale[bh];
      } else {
        const uint16_t *kp = (const uint16_t *)a.k + (first + j) * a.k_stride + g * D + lane * E;
#pragma unroll
        for (int k = 0; k < E; k += 2) {
          const float2 f = unpack2<F16>(*(const uint32_t *)(kp + k));
          x += q[k] * f.x + q[k + 1] * f.y;
        }
      }
      for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
      if (pass == 0) {
        if (isnan(x)) return;  // all of the row's own is NaN
        m = fmaxf(m, x);
        bool open = false;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          has[k] = has[k] && !isnan(v[k]);
          open |= has[k];
        }
        if (!all && !__any_sync(~0u, open)) return;  // every NaN that it has is one that it sees
        continue;
      }
      const float w = m == -INFINITY ? 0.f : exp2f(x - m);
      l += w;
#pragma unroll
      for (int k = 0; k < E; ++k) o[k] += w * v[k];
    }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int k = 0; k < E; k += 2) *(uint32_t *)(op + k) = pack_out<F16>(o[k] * inv, o[k + 1] * inv);
}

}  // namespace lv
