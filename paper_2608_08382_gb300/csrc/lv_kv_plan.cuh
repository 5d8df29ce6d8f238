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
// then its warps' stretches of the tile's slots and blocks, since the work is in
// the slots and one long prompt has as many as thousands of decodes.
//
// Measured: 20,000 requests, 2.6 million tokens: 22.5 us, 21 MB of slots written;
// 128 single tokens: 6.1 us in a graph, 8 as a call: a chain of dependent loads.
#pragma once

#include <climits>

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

// The requests of items x .. x + 127 (below x1), four a lane: item x + 32 y + lane's
// goes to i[y].  *lo is that of an item at or before x and moves to the last one's.
// The warp looks ahead from *lo for the last item's request in steps that double,
// and the lanes search between, all four in step (a long prompt's tokens not at all).
__device__ __forceinline__ void plan_requests(const int64_t *S, int n, int64_t x, int64_t x1, int lane, int *lo, int *i) {
  const int64_t last = min(x + kPlanSpan, x1) - 1;
  int from = *lo, to = from + 1;  // S[from] <= last; S[to] > last at the end, or to = n
  for (int step = 1; to < n && S[to] <= last; step *= 2) {
    from = to;
    to = min(n, to + step);
  }
  const int end = plan_find(S, last, from, to) + 1;
  int len = end - *lo;
#pragma unroll
  for (int y = 0; y < kPlanSpan / 32; ++y) i[y] = *lo;
  while (len > 1) {
    const int half = len >> 1;
#pragma unroll
    for (int y = 0; y < kPlanSpan / 32; ++y)
      if (S[i[y] + half] <= x + 32 * y + lane) i[y] += half;
    len -= half;
  }
  *lo = end - 1;
}

__global__ void __launch_bounds__(kPlanThreads, 2) k_plan(PlanArgs a) {
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
  // Each warp its own stretch of the tile's entries and of its slots, 128 at a time.
  const int64_t warps = little ? 1 : (int64_t)gridDim.x * (kPlanThreads / 32), me = (int64_t)blockIdx.x * (kPlanThreads / 32) + w;
  auto stretch = [&](int64_t all, int64_t share, int64_t of) { return (all + of * kPlanSpan - 1) / (of * kPlanSpan) * kPlanSpan * share; };
  // new table entries
  {
    const int64_t e0 = s.E[0], e1 = s.E[kPlanTile], of = little ? 4 : warps, mine = little ? (w % 4 == 0 ? w / 4 : of) : me;
    const int64_t k1 = min(e1, e0 + stretch(e1 - e0, mine + 1, of));
    int64_t k0 = e0 + stretch(e1 - e0, mine, of);
    int lo = k0 < k1 ? plan_find(s.E, k0, 0, top) : 0;
    for (; k0 < k1; k0 += kPlanSpan) {
      int i[kPlanSpan / 32];
      plan_requests(s.E, top, k0, k1, lane, &lo, i);
      int32_t id[kPlanSpan / 32];
#pragma unroll
      for (int y = 0; y < kPlanSpan / 32; ++y) {
        const int64_t k = k0 + 32 * y + lane;
        id[y] = k < k1 && s.E[i[y] + 1] <= a.n_free ? a.free[k] : -1;
      }
#pragma unroll
      for (int y = 0; y < kPlanSpan / 32; ++y) {
        const int64_t k = k0 + 32 * y + lane, col = ceil_blocks(s.c[i[y]], a.log_b) + (k - s.E[i[y]]);
        if (k >= k1) continue;
        if (col < a.width)
          a.table[(base + i[y]) * a.width + col] = id[y];
        else
          bad = true;
      }
    }
  }
  // slots
  {
    const int64_t x0 = s.X[0], x1 = min(s.X[kPlanTile], a.n_slots), of = little ? 12 : warps;
    const int64_t mine = little ? (w % 4 != 0 ? w / 4 * 3 + w % 4 - 1 : of) : me;
    const int64_t t1 = min(x1, x0 + stretch(x1 - x0, mine + 1, of));
    int64_t t0 = x0 + stretch(x1 - x0, mine, of);
    int lo = t0 < t1 ? plan_find(s.X, t0, 0, top) : 0;
    for (; t0 < t1; t0 += kPlanSpan) {
      const int64_t next = s.X[lo + 1];
      if (next >= min(t0 + kPlanSpan, t1) && t0 + kPlanSpan <= t1) {
        // all 128 are one request's: what is theirs alone in 32 bits (a thread's part of
        // the general way is five times as long, and prompts have most tokens)
        const int64_t pos0 = (int64_t)s.c[lo] + (t0 - s.X[lo]), col0 = pos0 >> a.log_b;
        const int64_t held = ceil_blocks(s.c[lo], a.log_b), room = a.width - col0;
        const int32_t *const row = a.table + (base + lo) * a.width + col0;
        const int32_t *const fresh = s.E[lo + 1] <= a.n_free ? a.free + s.E[lo] + (col0 - held) : nullptr;
        const int mask = (1 << a.log_b) - 1, x0 = ((int)pos0 & mask) + lane;
        const int old = (int)max((int64_t)-1, min((int64_t)INT32_MAX, held - col0));  // columns that were held before
        int64_t b[kPlanSpan / 32];
#pragma unroll
        for (int y = 0; y < kPlanSpan / 32; ++y) {
          const int col = (x0 + 32 * y) >> a.log_b;
          b[y] = -1;
          if (col >= room)
            bad = true;
          else if (col < old)
            b[y] = row[col];
          else if (fresh)
            b[y] = fresh[col];
        }
#pragma unroll
        for (int y = 0; y < kPlanSpan / 32; ++y)
          a.slots[t0 + 32 * y + lane] = b[y] < 0 ? -1 : (b[y] << a.log_b) + ((x0 + 32 * y) & mask);
        continue;
      }
      int i[kPlanSpan / 32];
      plan_requests(s.X, top, t0, t1, lane, &lo, i);
      // the blocks' numbers are all asked for before the first is waited for
      int64_t b[kPlanSpan / 32];
      int off[kPlanSpan / 32];
#pragma unroll
      for (int y = 0; y < kPlanSpan / 32; ++y) {
        const int64_t t = t0 + 32 * y + lane, pos = (int64_t)s.c[i[y]] + (t - s.X[i[y]]), col = pos >> a.log_b;
        const int64_t fresh = col - ceil_blocks(s.c[i[y]], a.log_b);  // which of the new blocks
        const int32_t *from = nullptr;
        off[y] = (int)pos & ((1 << a.log_b) - 1);
        if (t < t1) {
          if (col >= a.width)
            bad = true;
          else if (fresh < 0)
            from = a.table + (base + i[y]) * a.width + col;
          else if (s.E[i[y] + 1] <= a.n_free)
            from = a.free + s.E[i[y]] + fresh;
        }
        b[y] = from ? *from : -1;
      }
#pragma unroll
      for (int y = 0; y < kPlanSpan / 32; ++y)
        if (t0 + 32 * y + lane < t1) a.slots[t0 + 32 * y + lane] = b[y] < 0 ? -1 : (b[y] << a.log_b) + off[y];
    }
  }
  if (last)
    for (int64_t t = s.X[kPlanTile] + first; t < a.n_slots; t += step) a.slots[t] = -1;
  if (bad) flag(a.status, kStatusData);
}

}  // namespace lv
