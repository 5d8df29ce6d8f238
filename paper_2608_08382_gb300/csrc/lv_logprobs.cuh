// Log probabilities of given tokens, entropy and the largest logits
// (lv_token_logprobs): with m the row's largest logit, S = sum exp(x - m) and
// W = sum exp(x - m) (x - m),
//   lse = m + log S,  log p_v = (x_v - m) - log S,  entropy = log S - W / S.
//
// One pass over a row, by the threads of a CTA, 16 bytes a load, four asked for while
// four are added up; a thread keeps S and W relative to a logit of its own, which it
// takes anew only where one comes that is more than 8 above it (a scale that follows
// the maximum costs every warp a scaling every few loads), and which of its vectors
// holds its largest logit.  Few rows are shared by clusters of up to eight CTAs, whose
// sums and largest meet in the first one's shared memory.
//
// The n_top largest: of 32 groups of its threads each has a largest logit, and the
// n_top-th of those bounds the row's n_top-th from below (of equal ones by index; that of
// its vector will do); the threads' own do so more closely, at the cost of 256
// comparisons each.  Only threads whose own
// largest reaches the bound hold candidates; their logits are read once more, by all
// threads (a few threads' logits, still in L2; by the warps that had them, one hit after
// another: 9 us for 20 of 128,000), and the candidates are put in order by counting for each
// those above it.  Where there are more candidates than room (a row's largest all in one
// group's places: sorted rows have n_top times 64 at most), or the row has a NaN or
// +inf, the largest are looked for one after another.
// Every comparison is of a value and its index, so that nothing depends on an order of
// arrival.
//
// Measured: 4,096 rows of 32,000 in bf16 52 us, 5.0 TB/s (0.74 of the measured rate): 10.5
// instructions a logit keep 0.7 of the issue slots busy, through 3.4 rounds of rows of which
// the last is in part (with 20 alternatives 78 us); 256 fp32 rows of 128,000 with five
// alternatives 26.5 us (19.3 of bytes): the rows are one wave, and what follows its loads
// (4 us) lies behind them; one row of 128,000 with 20 alternatives 9.1 us.
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

constexpr int kLpGroups = 32;
constexpr int kLpRoom = 2048;   // candidates; also the logits of a row that leaves a group empty
constexpr int kLpFew = 256;     // candidates that are put in order as they are
constexpr int kLpCluster = 8;
static_assert(kLpGroups >= LV_MAX_TOP, "a bound from the groups");

// A difference of logits beyond which the exponential is 0, and that times it too (and
// times the largest sum there can be is finite).
constexpr float kLpFar = -1e20f;

struct LpPart {       // of a CTA's share of a row
  float base, S, W;   // sums of exp(x - base) and of that times (x - base)
  uint32_t top;       // the largest's order key, 0 where there is no logit
};
template <int WARPS>
struct LpSmem {
  uint64_t room[kLpRoom];
  uint64_t of_cluster[kLpCluster * LV_MAX_TOP];  // the first CTA's: everyone's largest
  uint64_t group[kLpGroups], key[WARPS * 32];  // bounds from below of a group's and a thread's largest
  uint64_t warp_key[WARPS];
  float warp_base[WARPS], warp_S[WARPS], warp_W[WARPS];
  uint32_t warp_top[WARPS];
  LpPart part[kLpCluster];
  uint64_t bound;
  uint16_t hit[WARPS * 32];  // threads with a largest that reaches the bound
  int hits, n;
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

// The largest logit of a vector; NaNs are passed over.
template <int TYPE>
__device__ __forceinline__ float largest_of(const uint4 &b) {
  if (TYPE == LV_F32)
    return fmaxf(fmaxf(__uint_as_float(b.x), __uint_as_float(b.y)), fmaxf(__uint_as_float(b.z), __uint_as_float(b.w)));
  if (TYPE == LV_F16) {
    const __half2 m = __hmax2(__hmax2(*(const __half2 *)&b.x, *(const __half2 *)&b.y),
                              __hmax2(*(const __half2 *)&b.z, *(const __half2 *)&b.w));
    return fmaxf(__low2float(m), __high2float(m));
  }
  const __nv_bfloat162 m = __hmax2(__hmax2(*(const __nv_bfloat162 *)&b.x, *(const __nv_bfloat162 *)&b.y),
                                   __hmax2(*(const __nv_bfloat162 *)&b.z, *(const __nv_bfloat162 *)&b.w));
  return fmaxf(__low2float(m), __high2float(m));
}

// A thread's running sums.
constexpr float kLpLazy = 8.f;
struct LpRun {
  float m = -INFINITY;     // its largest logit
  float base = 0.f;        // what the sums are relative to, once `set`
  bool set = false;
  uint64_t S = 0, W = 0;   // two sums each
  int where = -1;          // the first vector with a logit that equals m
  __device__ __forceinline__ void rebase() {  // before what makes m as it is is added
    if (set ? m > base + kLpLazy : m > -INFINITY) {
      if (set) {  // else there is nothing yet
        const float d = fmaxf(base - m, kLpFar), f = exp2_fast(d * 1.4426950408889634f);
        W = mul2(fma2(S, pair(d, d), W), pair(f, f));
        S = mul2(S, pair(f, f));
      }
      base = m;
      set = true;
    }
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

// Sums relative to another base, at least their own.
__device__ __forceinline__ void rescale(float base, float to, float *S, float *W) {
  const float d = fmaxf(base - to, kLpFar), f = exp2_fast(d * 1.4426950408889634f);
  *W = f * (*W + *S * d);
  *S *= f;
}

template <int TYPE, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_logprobs(const LogprobArgs a) {
  constexpr int kSize = TYPE == LV_F32 ? 4 : 2, kE = 16 / kSize, kAsk = 4;
  constexpr int kWarps = THREADS / 32, kLanes = THREADS / kLpGroups;  // lanes of a group
  // where a group has no logit there is none past it either, but for two vectors in part
  static_assert((THREADS - kLanes + 2) * kE <= kLpRoom, "all logits");
  __shared__ LpSmem<kWarps> sm;
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
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < kE; e += 2) {
      const float p = in_row(index(j, e)) ? logit(j, e) : -INFINITY, q = in_row(index(j, e + 1)) ? logit(j, e + 1) : -INFINITY;
      v[e / 2] = pair(p, q);
      top = fmaxf(top, fmaxf(p, q));
    }
    if (run.where < 0 || top > run.m) run.where = j;
    run.m = fmaxf(run.m, top);
    run.rebase();
    run.add(v);
  };
  if (head && tid == 0) edge(from);
  uint4 next[kAsk];
  auto ask = [&](int j) {
#pragma unroll
    for (int k = 0; k < kAsk; ++k)
      if (j + k * THREADS < whole1) next[k] = load_once(line + (int64_t)(j + k * THREADS) * 16);
  };
  ask(whole0 + tid);
  auto batch = [&](int j, auto there) {  // the vectors in `next`, or those that there are
    uint4 raw[kAsk];
#pragma unroll
    for (int k = 0; k < kAsk; ++k) raw[k] = next[k];
    ask(j + THREADS * kAsk);
    float top[kAsk], most = -INFINITY;
#pragma unroll
    for (int k = 0; k < kAsk; ++k) {
      top[k] = there(k) ? largest_of<TYPE>(raw[k]) : -INFINITY;
      most = fmaxf(most, top[k]);
    }
    if (run.where < 0) run.where = j;
    if (most > run.m) {
      run.m = most;
#pragma unroll
      for (int k = kAsk - 1; k >= 0; --k)
        if (top[k] == most) run.where = j + k * THREADS;
      run.rebase();
    }
#pragma unroll
    for (int k = 0; k < kAsk; ++k)
      if (there(k)) {
        uint64_t v[kE / 2];
        logit_pairs<TYPE>(raw[k], v);
        run.add(v);
      }
  };
  int j = whole0 + tid;
  for (; j + (kAsk - 1) * THREADS < whole1; j += THREADS * kAsk) batch(j, [](int) { return true; });
  if (j < whole1) batch(j, [&](int k) { return j + k * THREADS < whole1; });
  if (tail && tid == THREADS - 1) edge(to - 1);
  // ---- the CTA's sums, relative to the largest base
  LpPart part{run.set ? run.base : -INFINITY, 0.f, 0.f, run.where < 0 ? 0 : order_key(run.m)};
#pragma unroll
  for (int s = 16; s; s >>= 1) {
    part.base = fmaxf(part.base, __shfl_xor_sync(~0u, part.base, s));
    part.top = max(part.top, __shfl_xor_sync(~0u, part.top, s));
  }
  if (lane == 0) sm.warp_base[warp] = part.base, sm.warp_top[warp] = part.top;
  // the vector's last index for a bound from below, its first one for one from above
  uint64_t reach = 0;
  if (a.n_top > 0) {
    uint64_t least = 0;
    if (run.where >= 0) {
      const uint32_t key = order_key(run.m);
      least = full_key(key, min(index(run.where, kE - 1), a.vocab - 1));
      reach = full_key(key, max(index(run.where, 0), 0));
    }
    sm.key[tid] = least;
#pragma unroll
    for (int s = kLanes / 2; s; s >>= 1) least = larger(least, __shfl_xor_sync(~0u, least, s));
    if (lane % kLanes == 0) sm.group[tid / kLanes] = least;
  }
  if (tid == 0) sm.n = sm.hits = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWarps; ++k) {
    part.base = fmaxf(part.base, sm.warp_base[k]);
    part.top = max(part.top, sm.warp_top[k]);
  }
  {
    float s0, s1, w0, w1;
    unpair(run.S, &s0, &s1);
    unpair(run.W, &w0, &w1);
    part.S = s0 + s1;
    part.W = w0 + w1;
    if (run.set) rescale(run.base, part.base, &part.S, &part.W);  // else they are 0, or NaN
  }
#pragma unroll
  for (int s = 16; s; s >>= 1) {
    part.S += __shfl_xor_sync(~0u, part.S, s);
    part.W += __shfl_xor_sync(~0u, part.W, s);
  }
  if (lane == 0) sm.warp_S[warp] = part.S, sm.warp_W[warp] = part.W;
  // the n_top-th of the groups' largest, or everything where there is none
  if (a.n_top > 0 && warp == 1) {
    const uint64_t mine = sm.group[lane];
    int above = 0;
#pragma unroll
    for (int k = 0; k < kLpGroups; ++k) above += sm.group[k] > mine;
    const bool counts = mine != 0 && above < a.n_top;
    uint64_t least = counts ? mine : ~0ull;
#pragma unroll
    for (int s = 16; s; s >>= 1) {
      const uint64_t other = __shfl_xor_sync(~0u, least, s);
      least = other < least ? other : least;
    }
    const unsigned at = __ballot_sync(~0u, counts);
    if (lane == 0) sm.bound = __popc(at) < a.n_top ? 1 : least;
  }
  __syncthreads();
  part.S = sm.warp_S[0], part.W = sm.warp_W[0];
#pragma unroll
  for (int k = 1; k < kWarps; ++k) part.S += sm.warp_S[k], part.W += sm.warp_W[k];
  bool slow = part.S != part.S;  // a NaN, or an infinity less itself
  if (a.n_top > 0 && !slow) {
    // ---- candidates: above the groups' bound, and where there is none (a short row) or
    // they are many (equal logits, masks) above the threads', which takes longer to find
    for (bool fine = sm.bound == 1;; fine = true) {
      if (fine) {
        __syncthreads();
        if (tid == 0) sm.bound = 1, sm.n = sm.hits = 0;
        __syncthreads();
        const uint64_t mine = sm.key[tid];
        int above = 0;
#pragma unroll 8
        for (int k = 0; k < THREADS; ++k) above += sm.key[k] > mine;
        if (mine != 0 && above == a.n_top - 1) sm.bound = mine;
        __syncthreads();
      }
      const uint64_t bound = sm.bound;
      const uint32_t bound_key = (uint32_t)(bound >> 32);
      const bool hit = reach >= bound;
      const unsigned hits = __ballot_sync(~0u, hit);
      if (hits) {
        int at = 0;
        if (lane == 0) at = atomicAdd(&sm.hits, __popc(hits));
        at = __shfl_sync(~0u, at, 0) + __popc(hits & ((1u << lane) - 1));
        if (hit) sm.hit[at] = (uint16_t)tid;
      }
      auto keep = [&](int j, int e, float v) {
        const uint64_t key = full_key(order_key(v), index(j, e));
        if (key < bound) return;
        const int n = atomicAdd(&sm.n, 1);
        if (n < kLpRoom) sm.room[n] = key;
      };
      if (head && tid == 0 && hit)
        for (int e = 0; e < kE; ++e)
          if (in_row(index(from, e))) keep(from, e, logit(from, e));
      if (tail && tid == THREADS - 1 && hit)
        for (int e = 0; e < kE; ++e)
          if (in_row(index(to - 1, e))) keep(to - 1, e, logit(to - 1, e));
      __syncthreads();
      // all the hits' vectors, dealt out to all threads
      const unsigned per = (unsigned)(whole1 - whole0 + THREADS - 1) / THREADS, looks = sm.hits * per;
#pragma unroll 2
      for (unsigned i = tid; i < looks; i += THREADS) {
        const unsigned h = i / per;
        const int j = whole0 + sm.hit[h] + (int)(i - h * per) * THREADS;
        if (j >= whole1) continue;
        const uint4 raw = load_once(line + (int64_t)j * 16);
        if (order_key(largest_of<TYPE>(raw)) < bound_key) continue;
        uint64_t v[kE / 2];
        logit_pairs<TYPE>(raw, v);
#pragma unroll
        for (int e = 0; e < kE; e += 2) {
          float p, q;
          unpair(v[e / 2], &p, &q);
          keep(j, e, p);
          keep(j, e + 1, q);
        }
      }
      __syncthreads();
      if (fine || sm.n <= kLpFew) break;
    }
    slow = sm.n > kLpRoom;
  }
  const int k_top = a.n_top;
  if (slow) {
    // one after another
    uint64_t below = ~0ull;
    for (int k = 0; k < max(k_top, 1); ++k) {
      uint64_t next = 0;
      for (int j = from + tid; j < to; j += THREADS)
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
      for (int w = 0; w < kWarps; ++w) next = larger(next, sm.warp_key[w]);
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
                            tid == 0 ? part.base : tid == 1 ? part.S : tid == 2 ? part.W : __uint_as_float(part.top));
    auto send = [&](int at, uint64_t key) {
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(peer_addr(&sm.of_cluster[rank * LV_MAX_TOP + at], 0)), "l"(key) : "memory");
    };
    for (int i = tid; i < n; i += THREADS) {
      const uint64_t mine = sm.room[i];
      int above = 0;
      for (int k = 0; k < n; ++k) above += sm.room[k] > mine;
      if (above < k_top && mine) send(above, mine);
    }
    for (int i = n + tid; i < k_top; i += THREADS) send(i, 0);
    if (slow)
      for (int i = tid; i < k_top; i += THREADS)
        if (!sm.room[i]) send(i, 0);
    cluster_sync();
    if (rank != 0) return;
    float most = sm.part[0].base;
    for (int k = 1; k < a.cluster; ++k) most = fmaxf(most, sm.part[k].base);
    part = LpPart{most, 0.f, 0.f, 0};
    for (int k = 0; k < a.cluster; ++k) {
      LpPart p = sm.part[k];
      rescale(p.base, most, &p.S, &p.W);
      part.S += p.S;
      part.W += p.W;
      part.top = max(part.top, p.top);
    }
    for (int i = tid; i < a.cluster * k_top; i += THREADS) sm.room[i] = sm.of_cluster[i / k_top * LV_MAX_TOP + i % k_top];
    n = a.cluster * k_top;
    __syncthreads();
  }
  // ---- the row's values
  const float m = key_value(part.top);
  const bool none = m == -INFINITY;
  // to the largest, whose exponential is 1
  if (m == m && m != INFINITY && !none) rescale(part.base, m, &part.S, &part.W);
  const float log_s = m == m ? logf(part.S) : NAN;
  auto log_p = [&](float x) { return none ? m : m == INFINITY ? x - m : (x - m) - log_s; };
  if (tid == 0) {
    if (a.lse) a.lse[t] = none || m == INFINITY ? m : m + log_s;
    if (a.entropy) a.entropy[t] = none ? 0.f : m == INFINITY ? NAN : log_s - part.W / part.S;
    if (a.logp) a.logp[t] = given != given ? NAN : log_p(given);
  }
  if (k_top > 0) {
    int32_t *const ids = a.top_ids + t * k_top;
    float *const lp = a.top_logp + t * k_top;
    for (int i = tid; i < n; i += THREADS) {
      const uint64_t mine = sm.room[i];
      if (!mine) continue;
      int above = 0;
      for (int k = 0; k < n; ++k) above += sm.room[k] > mine;
      if (above < k_top) {
        ids[above] = (int32_t)~(uint32_t)mine;
        lp[above] = log_p(key_value((uint32_t)(mine >> 32)));
      }
    }
    for (int i = a.vocab + tid; i < k_top; i += THREADS) {  // past the vocabulary's end
      ids[i] = -1;
      lp[i] = -INFINITY;
    }
  }
}

}  // namespace lv
