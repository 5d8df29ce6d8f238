// Block tables and slot maps of a step from its requests' lengths (lv_kv_plan).
//
// need_i = ceil((c_i + p_i)/B) - ceil(c_i/B); X and E are the running sums of p
// and need.  Everything else is addressed by X_i and E_i: request i's new table
// entries are free[E_i ..], its tokens' slots stand at slots[X_i ..].
//
// Requests go in tiles of kPlanTile, a CTA scans one tile in registers and shared
// memory.  Of a call with several tiles k_plan_sums first writes each tile's
// sums, and a CTA adds up those before its own.  Several CTAs take one tile
// together, each forms the same scan (a few microseconds, mostly latency) and
// then every gridDim.x-th piece of the tile's tokens and blocks, since the work is in the
// slots and one long prompt has as many as thousands of decodes.
#pragma once

#include "lv_base.cuh"

namespace lv {

constexpr int kPlanThreads = 512;
constexpr int kPlanPer = 4;                             // requests of one thread
constexpr int kPlanTile = kPlanThreads * kPlanPer;      // requests of a tile
constexpr int kPlanSpan = 128;                          // entries or slots of a warp's turn

struct PlanArgs {
  const int32_t *p, *c;
  int64_t n_req;
  int log_b;  // block_tokens = 1 << log_b
  const int32_t *free;
  int64_t n_free;
  int32_t *table;
  int64_t width;
  int64_t *offsets, *slots;
  int64_t n_slots;
  int64_t *counts;
  int64_t *sums;  // [tiles][2] tokens and blocks of each tile, or null for one tile
  int *status;
};

__device__ __forceinline__ int64_t ceil_blocks(int64_t tokens, int log_b) {
  return (tokens + (1ll << log_b) - 1) >> log_b;
}

// A request's lengths, a bad one as no request.
__device__ __forceinline__ bool plan_load(const PlanArgs &a, int64_t i, int32_t *p, int32_t *c) {
  *p = *c = 0;
  if (i >= a.n_req) return false;
  *p = a.p[i];
  *c = a.c[i];
  if (*p >= 0 && *c >= 0) return false;
  *p = *c = 0;
  return true;
}

__device__ __forceinline__ int64_t plan_need(int32_t p, int32_t c, int log_b) {
  return ceil_blocks((int64_t)c + p, log_b) - ceil_blocks(c, log_b);
}

__global__ void __launch_bounds__(kPlanThreads) k_plan_sums(PlanArgs a) {
  __shared__ int64_t part[kPlanThreads / 32][2];
  const int64_t base = (int64_t)blockIdx.x * kPlanTile;
  int64_t tok = 0, blk = 0;
  for (int k = 0; k < kPlanPer; ++k) {
    int32_t p, c;
    plan_load(a, base + k * kPlanThreads + threadIdx.x, &p, &c);
    tok += p;
    blk += plan_need(p, c, a.log_b);
  }
  for (int d = 16; d; d >>= 1) {
    tok += __shfl_xor_sync(~0u, tok, d);
    blk += __shfl_xor_sync(~0u, blk, d);
  }
  if ((threadIdx.x & 31) == 0) {
    part[threadIdx.x >> 5][0] = tok;
    part[threadIdx.x >> 5][1] = blk;
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    int64_t s = 0;
    for (int w = 0; w < kPlanThreads / 32; ++w) s += part[w][threadIdx.x];
    a.sums[2 * (int64_t)blockIdx.x + threadIdx.x] = s;
  }
}

struct PlanSmem {
  int64_t X[kPlanTile + 1], E[kPlanTile + 1];
  int32_t c[kPlanTile];
  int64_t warp[kPlanThreads / 32][2];
  int64_t before[2];
};

// The last request of lo .. hi - 1 whose range [S[i], S[i+1]) begins at or before
// x; S[lo] <= x.
__device__ __forceinline__ int plan_find(const int64_t *S, int64_t x, int lo, int hi) {
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (S[m] <= x) lo = m; else hi = m;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) k_plan(PlanArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  PlanSmem &s = *reinterpret_cast<PlanSmem *>(raw);
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int64_t tile = blockIdx.y, base = tile * kPlanTile;
  wait_previous();
  // the sums of the tiles before
  if (tid < 2) s.before[tid] = 0;
  __syncthreads();
  if (a.sums && tile > 0) {
    int64_t tok = 0, blk = 0;
    for (int64_t t = tid; t < tile; t += kPlanThreads) {
      tok += a.sums[2 * t];
      blk += a.sums[2 * t + 1];
    }
    for (int d = 16; d; d >>= 1) {
      tok += __shfl_xor_sync(~0u, tok, d);
      blk += __shfl_xor_sync(~0u, blk, d);
    }
    if (lane == 0 && (tok | blk)) {
      atomicAdd((unsigned long long *)&s.before[0], (unsigned long long)tok);
      atomicAdd((unsigned long long *)&s.before[1], (unsigned long long)blk);
    }
  }
  // scan of the tile: a thread's kPlanPer neighbours, the warp, the warps
  int32_t p[kPlanPer], c[kPlanPer];
  int64_t tok = 0, blk = 0;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kPlanPer; ++k) {
    bad |= plan_load(a, base + tid * kPlanPer + k, &p[k], &c[k]);
    tok += p[k];
    blk += plan_need(p[k], c[k], a.log_b);
  }
  int64_t x = tok, e = blk;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t xx = __shfl_up_sync(~0u, x, d), ee = __shfl_up_sync(~0u, e, d);
    if (lane >= d) x += xx, e += ee;
  }
  if (lane == 31) s.warp[w][0] = x, s.warp[w][1] = e;
  __syncthreads();
  x += s.before[0] - tok;
  e += s.before[1] - blk;
  for (int k = 0; k < w; ++k) x += s.warp[k][0], e += s.warp[k][1];
#pragma unroll
  for (int k = 0; k < kPlanPer; ++k) {
    const int i = tid * kPlanPer + k;
    s.X[i] = x;
    s.E[i] = e;
    s.c[i] = c[k];
    x += p[k];
    e += plan_need(p[k], c[k], a.log_b);
  }
  if (tid == kPlanThreads - 1) s.X[kPlanTile] = x, s.E[kPlanTile] = e;
  __syncthreads();
  const int64_t n = min((int64_t)kPlanTile, a.n_req - base);  // requests of this tile
  const int64_t first = (int64_t)blockIdx.x * kPlanThreads + tid, step = (int64_t)gridDim.x * kPlanThreads;
  for (int64_t i = first; i < n; i += step) a.offsets[base + i] = s.X[i];
  const bool last = tile == gridDim.y - 1;
  if (last && first == 0) {
    a.offsets[a.n_req] = s.X[kPlanTile];
    a.counts[0] = s.X[kPlanTile];
    a.counts[1] = s.E[kPlanTile];
    bad |= s.X[kPlanTile] > a.n_slots;
  }
  // Where there is little, a quarter of the warps takes the entries and the others
  // the slots, so that one does not wait for the other.
  const bool little = s.X[kPlanTile] - s.X[0] <= 12 * kPlanSpan && s.E[kPlanTile] - s.E[0] <= 4 * kPlanSpan && gridDim.x == 1;
  const int top = (int)n;  // requests to search among
  // A warp takes 128 entries or slots at a time: two searches find the requests of
  // the first and the last of them, and the lanes search between those (a long
  // prompt's tokens not at all).
  const int64_t wfirst = ((int64_t)blockIdx.x * (kPlanThreads / 32) + w) * kPlanSpan, wstep = step * (kPlanSpan / 32);
  const int64_t efirst = !little ? wfirst : w % 4 == 0 ? w / 4 * kPlanSpan : 4 * kPlanSpan;
  const int64_t xfirst = !little ? wfirst : w % 4 != 0 ? (w / 4 * 3 + w % 4 - 1) * kPlanSpan : 12 * kPlanSpan;
  // new table entries
  const int64_t e1 = s.E[kPlanTile];
  for (int64_t k0 = s.E[0] + efirst; k0 < e1; k0 += wstep) {
    const int lo = plan_find(s.E, k0, 0, top), hi = plan_find(s.E, min(k0 + kPlanSpan, e1) - 1, lo, kPlanTile) + 1;
#pragma unroll
    for (int y = 0; y < kPlanSpan; y += 32) {
      const int64_t k = k0 + y + lane;
      if (k >= e1) break;
      const int i = plan_find(s.E, k, lo, hi);
      const int64_t col = ceil_blocks(s.c[i], a.log_b) + (k - s.E[i]);
      if (col < a.width)
        a.table[(base + i) * a.width + col] = s.E[i + 1] <= a.n_free ? a.free[k] : -1;
      else
        bad = true;
    }
  }
  // slots
  const int64_t x1 = min(s.X[kPlanTile], a.n_slots);
  for (int64_t t1 = s.X[0] + xfirst; t1 < x1; t1 += wstep) {
    const int lo = plan_find(s.X, t1, 0, top), hi = plan_find(s.X, min(t1 + kPlanSpan, x1) - 1, lo, kPlanTile) + 1;
#pragma unroll
    for (int y = 0; y < kPlanSpan; y += 32) {
      const int64_t t = t1 + y + lane;
      if (t >= x1) break;
      const int i = plan_find(s.X, t, lo, hi);
      const int64_t pos = (int64_t)s.c[i] + (t - s.X[i]), col = pos >> a.log_b;
      const int64_t fresh = col - ceil_blocks(s.c[i], a.log_b);  // which of the new blocks
      int64_t b = -1;
      if (col >= a.width)
        bad = true;
      else if (fresh < 0)
        b = a.table[(base + i) * a.width + col];
      else if (s.E[i + 1] <= a.n_free)
        b = a.free[s.E[i] + fresh];
      a.slots[t] = b < 0 ? -1 : (b << a.log_b) + (pos & ((1 << a.log_b) - 1));
    }
  }
  if (last)
    for (int64_t t = s.X[kPlanTile] + first; t < a.n_slots; t += step) a.slots[t] = -1;
  if (bad) flag(a.status, kStatusData);
}

}  // namespace lv
