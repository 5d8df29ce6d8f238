// Log probabilities of given tokens, entropy and the largest logits
// (lv_token_logprobs): with m the row's largest logit, S = sum exp(x - m) and
// W = sum exp(x - m) (x - m),
//   lse = m + log S,  log p_v = (x_v - m) - log S,  entropy = log S - W / S.
//
// One pass over a row, by the 256 threads of a CTA, 16 bytes a load, four in a row; a
// thread keeps its own m, S and W, which are scaled again where its m grows, and where
// its largest logit stands.  Few rows are shared by clusters of up to eight CTAs, whose
// sums and largest meet in the first one's shared memory.
//
// The n_top largest: of the 32 groups of eight threads each has a largest logit, and the
// n_top-th of those bounds the row's n_top-th from below.  Only threads whose own
// largest reaches the bound hold candidates; their warps read their logits once more
// (a few of 256, still in L2) and the candidates are put in order by counting for each
// those above it.  Where there are more candidates than room (a row in descending
// order), or the row has a NaN or +inf, the largest are looked for one after another.
// Every comparison is of a value and its index, so that nothing depends on an order of
// arrival.
#pragma once

#include "lv_linear.cuh"

namespace lv {

struct LogprobArgs {
  const void *x;
  int64_t stride, n_tok;
  int vocab, n_top;
  int cluster;       // CTAs of a row
  const int32_t *ids;
  float *logp, *entropy, *lse;
  int32_t *top_ids;
  float *top_logp;
  int *status;
};

template <int TYPE>
__device__ __forceinline__ float logit_at(const void *x, int64_t at) {
  if (TYPE == LV_F32) return ((const float *)x)[at];
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
__device__ __forceinline__ uint64_t larger(uint64_t a, uint64_t b) { return a > b ? a : b; }

constexpr int kLpThreads = 256, kLpWarps = kLpThreads / 32;
constexpr int kLpGroups = kLpThreads / 8;
constexpr int kLpRoom = 2048;   // candidates; also the logits of a row that leaves a group empty
constexpr int kLpCluster = 8;
static_assert(kLpGroups >= LV_MAX_TOP && kLpGroups * 8 * 8 <= kLpRoom, "a bound from the groups, or all logits");

// A difference of logits beyond which the exponential is 0, and that times it too.
constexpr float kLpFar = -1e30f;

struct LpPart {       // of a CTA's share of a row
  float m, S, W;      // W in units of the natural logarithm
  uint32_t top;       // the largest's order key
};
struct LpSmem {
  uint64_t room[kLpRoom];
  uint64_t of_cluster[kLpCluster * LV_MAX_TOP];  // the first CTA's: everyone's largest
  uint64_t group[kLpGroups];
  uint64_t warp_key[kLpWarps];
  LpPart warp[kLpWarps], part[kLpCluster];
  uint64_t bound;
  int n;
};

__device__ __forceinline__ uint4 load_once(const void *p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
// A 16-byte vector of logits as pairs of floats.
template <int TYPE>
__device__ __forceinline__ void logit_pairs(const uint4 &b, uint64_t *v) {
  if (TYPE == LV_F32) {
    v[0] = pair(__uint_as_float(b.x), __uint_as_float(b.y));
    v[1] = pair(__uint_as_float(b.z), __uint_as_float(b.w));
  } else {
    unpack_pairs<TYPE == LV_F16>(b, v);
  }
}

// A thread's running m, S, W.
struct LpRun {
  float m = -INFINITY, base = 0.f;  // base: m, or 0 while there is none
  uint64_t S = 0, W = 0;            // two sums each
  int where = -1;                   // vector of the first logit that equals m
  __device__ __forceinline__ void grow(float to) {
    const float f = m == -INFINITY ? 0.f : exp2_fast((m - to) * 1.4426950408889634f), d = m == -INFINITY ? 0.f : fmaxf(m - to, kLpFar);
    W = mul2(fma2(S, pair(d, d), W), pair(f, f));
    S = mul2(S, pair(f, f));
    m = base = to;
  }
  template <int N>
  __device__ __forceinline__ void add(const uint64_t (&v)[N]) {
    const uint64_t by = pair(1.4426950408889634f, 1.4426950408889634f), less = pair(-base, -base);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint64_t d2 = add2(v[k], less);
      float a, b, p, q;
      unpair(d2, &a, &b);
      unpair(mul2(d2, by), &p, &q);
      const uint64_t e = pair(exp2_fast(p), exp2_fast(q));
      S = add2(S, e);
      W = fma2(e, pair(fmaxf(a, kLpFar), fmaxf(b, kLpFar)), W);  // 0 of a logit of -inf
    }
  }
};
template <int N>
__device__ __forceinline__ float largest_of(const uint64_t (&v)[N]) {
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float a, b;
    unpair(v[k], &a, &b);
    top = fmaxf(top, fmaxf(a, b));
  }
  return top;
}

// Two parts together.
__device__ __forceinline__ LpPart join(const LpPart &a, const LpPart &b) {
  LpPart r;
  r.m = fmaxf(a.m, b.m);
  r.top = max(a.top, b.top);
  const float da = a.m == r.m ? 0.f : fmaxf(a.m - r.m, kLpFar), db = b.m == r.m ? 0.f : fmaxf(b.m - r.m, kLpFar);
  const float fa = exp2_fast(da * 1.4426950408889634f), fb = exp2_fast(db * 1.4426950408889634f);
  // a part of m = -inf has no sums
  r.S = a.S * fa + b.S * fb;
  r.W = (a.m == -INFINITY ? 0.f : fa * (a.W + a.S * da)) + (b.m == -INFINITY ? 0.f : fb * (b.W + b.S * db));
  return r;
}

template <int TYPE>
__global__ void __launch_bounds__(kLpThreads, 4) k_logprobs(const LogprobArgs a) {
  constexpr int kSize = TYPE == LV_F32 ? 4 : 2, kE = 16 / kSize, kAsk = 4;
  __shared__ LpSmem sm;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t t = blockIdx.x / a.cluster;
  const uint32_t rank = blockIdx.x % a.cluster;
  let_next();
  wait_previous();
  // the row in vectors of 16 bytes from a 16-byte boundary on, `lead` elements of the
  // first before the row; the CTA's are from .. to - 1, and all of `whole0 .. whole1 - 1`
  // are the row's throughout
  const char *const row = (const char *)a.x + t * a.stride * kSize;
  const int lead = (int)((uintptr_t)row & 15) / kSize;
  const char *const line = row - lead * kSize;
  const int vectors = (lead + a.vocab + kE - 1) / kE;
  const int from = (int)((int64_t)vectors * rank / a.cluster), to = (int)((int64_t)vectors * (rank + 1) / a.cluster);
  const int whole0 = max(from, lead > 0 ? 1 : 0), whole1 = max(whole0, min(to, (lead + a.vocab) / kE));
  const bool head = from < whole0 && from < to, tail = to > whole1 && !(head && to == 1);
  auto index = [&](int j, int e) { return j * kE + e - lead; };
  auto logit = [&](int j, int e) { return logit_at<TYPE>(line, (int64_t)j * kE + e); };
  auto in_row = [&](int i) { return i >= 0 && i < a.vocab; };
  float given = NAN;  // the given token's logit
  if (tid == 0 && rank == 0 && a.logp) {
    const int id = a.ids[t];
    if (in_row(id))
      given = logit_at<TYPE>(row, id);
    else if (id != -1)
      flag(a.status, kStatusData);
  }
  // ---- one pass
  LpRun run;
  auto edge = [&](int j) {  // a vector that is the row's in part
    uint64_t v[kE / 2];
#pragma unroll
    for (int e = 0; e < kE; e += 2)
      v[e / 2] = pair(in_row(index(j, e)) ? logit(j, e) : -INFINITY, in_row(index(j, e + 1)) ? logit(j, e + 1) : -INFINITY);
    const float top = largest_of(v);
    if (run.where < 0) run.where = j;
    if (top > run.m) {
      run.grow(top);
      run.where = j;
    }
    run.add(v);
  };
  if (head && tid == 0) edge(from);
  for (int j = whole0 + tid; j < whole1; j += kLpThreads * kAsk) {
    uint4 raw[kAsk];
    const int n = min(kAsk, (whole1 - j + kLpThreads - 1) / kLpThreads);
#pragma unroll
    for (int k = 0; k < kAsk; ++k)
      if (k < n) raw[k] = load_once(line + (int64_t)(j + k * kLpThreads) * 16);
    if (run.where < 0) run.where = j;
    float top[kAsk], most = -INFINITY;
#pragma unroll
    for (int k = 0; k < kAsk; ++k) {
      uint64_t v[kE / 2];
      logit_pairs<TYPE>(raw[k], v);
      top[k] = k < n ? largest_of(v) : -INFINITY;
      most = fmaxf(most, top[k]);
    }
    if (most > run.m) {
      bool found = false;
#pragma unroll
      for (int k = 0; k < kAsk; ++k)
        if (!found && top[k] == most) run.where = j + k * kLpThreads, found = true;
      run.grow(most);
    }
#pragma unroll
    for (int k = 0; k < kAsk; ++k) {
      uint64_t v[kE / 2];
      logit_pairs<TYPE>(raw[k], v);
      if (k < n) run.add(v);
    }
  }
  if (tail && tid == kLpThreads - 1) edge(to - 1);
  // ---- the CTA's sums
  float s0, s1, w0, w1;
  unpair(run.S, &s0, &s1);
  unpair(run.W, &w0, &w1);
  LpPart part{run.m, s0 + s1, w0 + w1, run.where < 0 ? 0 : order_key(run.m)};
#pragma unroll
  for (int s = 16; s; s >>= 1) {
    const LpPart other{__shfl_xor_sync(~0u, part.m, s), __shfl_xor_sync(~0u, part.S, s), __shfl_xor_sync(~0u, part.W, s),
                       __shfl_xor_sync(~0u, part.top, s)};
    // the same way in both lanes
    part = lane & s ? join(other, part) : join(part, other);
  }
  if (lane == 0) sm.warp[warp] = part;
  // each thread's largest, and its group's
  uint64_t best = 0;
  if (a.n_top > 0) {
    if (run.where >= 0) {
      int e = 0;
      for (; e < kE - 1; ++e)
        if (in_row(index(run.where, e)) && logit(run.where, e) == run.m) break;
      best = full_key(order_key(run.m), index(run.where, e));
    }
    uint64_t top = best;
#pragma unroll
    for (int s = 4; s; s >>= 1) top = larger(top, __shfl_xor_sync(~0u, top, s));
    if ((lane & 7) == 0) sm.group[tid >> 3] = top;
  }
  if (tid == 0) sm.n = 0;
  __syncthreads();
  part = sm.warp[0];
#pragma unroll
  for (int k = 1; k < kLpWarps; ++k) part = join(part, sm.warp[k]);
  bool slow = part.S != part.S;  // a NaN, or an infinity less itself
  if (a.n_top > 0 && !slow) {
    // ---- candidates
    if (warp == 0) {
      const uint64_t mine = sm.group[lane];
      int above = 0;
#pragma unroll
      for (int k = 0; k < kLpGroups; ++k) above += sm.group[k] > mine;
      // the n_top-th, or everything where there is none; empty groups are all 0 and equal
      const unsigned at = __ballot_sync(~0u, above < a.n_top && mine != 0);
      uint64_t least = mine != 0 && above < a.n_top ? mine : ~0ull;
#pragma unroll
      for (int s = 16; s; s >>= 1) {
        const uint64_t other = __shfl_xor_sync(~0u, least, s);
        least = other < least ? other : least;
      }
      if (lane == 0) sm.bound = __popc(at) < a.n_top ? 1 : least;
    }
    __syncthreads();
    const uint64_t bound = sm.bound;
    unsigned hits = __ballot_sync(~0u, best >= bound);
    while (hits) {
      const int h = __ffs(hits) - 1, ht = warp * 32 + h;
      hits &= hits - 1;
      auto look = [&](int j) {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const int i = index(j, e);
          if (!in_row(i)) continue;
          const uint64_t key = full_key(order_key(logit(j, e)), i);
          if (key >= bound) {
            const int n = atomicAdd(&sm.n, 1);
            if (n < kLpRoom) sm.room[n] = key;
          }
        }
      };
      for (int j = whole0 + ht + lane * kLpThreads; j < whole1; j += 32 * kLpThreads) look(j);
      if (head && ht == 0 && lane == 0) look(from);
      if (tail && ht == kLpThreads - 1 && lane == 0) look(to - 1);
    }
    __syncthreads();
    slow = sm.n > kLpRoom;
  }
  const int k_top = a.n_top;
  if (slow) {
    // one after another
    uint64_t below = ~0ull;
    for (int k = 0; k < max(k_top, 1); ++k) {
      uint64_t next = 0;
      for (int j = from + tid; j < to; j += kLpThreads)
        for (int e = 0; e < kE; ++e) {
          const int i = index(j, e);
          if (!in_row(i)) continue;
          const uint64_t key = full_key(order_key(logit(j, e)), i);
          if (key < below) next = larger(next, key);
        }
#pragma unroll
      for (int s = 16; s; s >>= 1) next = larger(next, __shfl_xor_sync(~0u, next, s));
      __syncthreads();
      if (lane == 0) sm.warp_key[warp] = next;
      __syncthreads();
      for (int w = 0; w < kLpWarps; ++w) next = larger(next, sm.warp_key[w]);
      if (k == 0) part.top = max(part.top, (uint32_t)(next >> 32));
      if (tid == 0) sm.room[k] = next;
      below = next;
    }
    __syncthreads();
  }
  int n = slow ? k_top : a.n_top > 0 ? sm.n : 0;
  if (a.cluster > 1) {
    // to the first CTA: the sums, and the largest in order
    cluster_sync();  // it is there
    if (tid < 4) store_peer(peer_addr((float *)&sm.part[rank] + tid, 0),
                            tid == 0 ? part.m : tid == 1 ? part.S : tid == 2 ? part.W : __uint_as_float(part.top));
    auto send = [&](int at, uint64_t key) {
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_addr(&sm.of_cluster[rank * LV_MAX_TOP + at], 0)), "l"(key) : "memory");
    };
    for (int i = tid; i < n; i += kLpThreads) {
      const uint64_t mine = sm.room[i];
      int above = 0;
      for (int k = 0; k < n; ++k) above += sm.room[k] > mine;
      if (above < k_top && mine) send(above, mine);
    }
    for (int i = n + tid; i < k_top; i += kLpThreads) send(i, 0);
    if (slow)
      for (int i = tid; i < k_top; i += kLpThreads)
        if (!sm.room[i]) send(i, 0);
    cluster_sync();
    if (rank != 0) return;
    part = sm.part[0];
    for (int k = 1; k < a.cluster; ++k) part = join(part, sm.part[k]);
    n = 0;
    for (int i = tid; i < a.cluster * k_top; i += kLpThreads) sm.room[i] = sm.of_cluster[i / k_top * LV_MAX_TOP + i % k_top];
    n = a.cluster * k_top;
    __syncthreads();
  }
  // ---- the row's values
  const float m = key_value(part.top), log_s = logf(part.S);
  const bool none = m == -INFINITY;
  auto log_p = [&](float x) { return none ? m : m == INFINITY ? x - m : (x - m) - log_s; };
  if (tid == 0) {
    if (a.lse) a.lse[t] = none || m == INFINITY ? m : m + log_s;
    if (a.entropy) a.entropy[t] = none ? 0.f : m == INFINITY ? NAN : log_s - part.W / part.S;
    if (a.logp) a.logp[t] = given != given ? NAN : log_p(given);
  }
  if (k_top > 0) {
    int32_t *const ids = a.top_ids + t * k_top;
    float *const lp = a.top_logp + t * k_top;
    for (int i = tid; i < n; i += kLpThreads) {
      const uint64_t mine = sm.room[i];
      if (!mine) continue;
      int above = 0;
      for (int k = 0; k < n; ++k) above += sm.room[k] > mine;
      if (above < k_top) {
        ids[above] = (int32_t)~(uint32_t)mine;
        lp[above] = log_p(key_value((uint32_t)(mine >> 32)));
      }
    }
    for (int i = a.vocab + tid; i < k_top; i += kLpThreads) {  // past the vocabulary's end
      ids[i] = -1;
      lp[i] = -INFINITY;
    }
  }
}

}  // namespace lv
