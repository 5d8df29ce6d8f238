// Causal attention over packed prompts (lv_prompt_attend) on the tensor cores.
//
// S = Q K^T and O += P V cost 4 D FLOPs a (query, key, head), and that bounds all
// but the shortest calls; the softmax between them costs an exponential a score.
// A work item is two tiles of up to 128 rows of one key/value head.  A row is a
// (token, query head) pair and a tile holds whole tokens, 128 / G of them with
// all G query heads that share the keys, so the keys are fetched once for the
// group and few of a tile's scores are masked (a tile spans 128 / G tokens).
//
// One CTA a SM, three warpgroups:
//   warps 0-3, 4-7  softmax of tile 0 and of tile 1, a row a thread;
//   warp 8          issues every tcgen05.mma (one lane);
//   warp 9          takes the items and issues every TMA load (one lane); warps 10
//                   and 11 only fill the warpgroup.
// A row's 128 scores stay in its thread's registers: the softmax warpgroups take
// 216 a thread, the third 72, together the 384 x 168 that the block starts with.
// Tensor memory holds both tiles' scores and outputs, 128 + D columns each.  The
// weights go back over the scores' columns as 16-bit values and are the second
// product's A operand from there.  The issue order PV_0(j) QK_0(j+1) PV_1(j)
// QK_1(j+1) has the tensor core at one tile while the other's softmax runs; it is
// in order, so a tile's scores are overwritten only after its weights were used,
// and when a tile's scores are ready the product before them is done as well and its
// outputs may be rescaled.
//
// The running maximum that a row's weights refer to moves only when the true
// one is more than 2^8 above it (weights are at most 2^8, sums are fp32): after
// the first blocks of keys hardly any output is read back to be rescaled.
// Weights are rounded to the inputs' 16-bit type, as V is; those of f16 are 2^7 times
// as large, so that 2^-32 of the largest is the first that is lost (bf16 has fp32's
// range).  Half of a block's weights go to the products while the other half is
// formed.
//
// Items are handed out by a counter, longest first within a sequence and the
// longest sequence first (twelve prompts of up to 4,096 tokens: 84 us in the order
// that they came), and the loads run ahead of the products across items.
//
// Measured: one prompt of 8,192 tokens, 20/4 heads of 128, bf16: 224 us, 1,530
// TFLOP/s (0.80 of the measured rate); two of 25,001 tokens in all, 10/2 heads, fp16:
// 540 us; twelve of 8,005 tokens in all, 32/8 heads: 73 us, of which an item's
// beginning and its stores are a third.  A block of both tiles takes 3,000 clocks,
// the products 2,048: a tile's softmax (1,500) and its two products (1,024) follow
// each other, and with both tiles' scores and outputs tensor memory is full, so the
// next scores have no place before the weights were used.
#pragma once

#include <climits>

#include "lv_attend.cuh"
#include "lv_tc.cuh"

namespace lv {

constexpr int kPrThreads = 384;
constexpr int kPrBlock = 128;   // keys of a block
constexpr int kSort = 512;      // sequences that are taken longest first
constexpr float kPrLazy = 8.f;  // growth of the maximum, in powers of two, that weights absorb
constexpr float kPrExp = 7.f;   // f16 weights are 2^7 at the maximum they refer to, and so up to 2^15

struct PromptArgs {
  AttendArgs a;
  int tile;             // tokens of a tile: 128 / G
  bool wide;            // o is 32-byte aligned
  int64_t *prefix;      // [n_req + 1] items before each sequence, given for more than kScan
  bool given;
  unsigned long long *counter; // items handed out beyond the first of each CTA; CTAs done (zero between launches)
};

struct PromptItem {
  int first;      // the sequence's first token
  int t0, len;    // first token of the item in the sequence, the sequence's length
  int head;       // key/value head, or -1: no more items
  int n[2];       // key blocks of each tile
  int tail[2];    // keys of the last one that its rows see, in steps of 16
};

template <int D>
struct PromptSmem {
  static constexpr int kRowBytes = 128;                    // a row of 64 elements
  static constexpr int kTile = 128 * D * 2;                // bytes of a tile of Q or a block of K or V
  static constexpr int kStages = 4;                        // blocks of keys or values
  unsigned char q[2][kTile];
  unsigned char kv[kStages][kTile];
  uint64_t q_full[2], q_empty[2], kv_full[kStages], kv_empty[kStages], s_full[2], p_half[2], p_full[2], o_full[2];
  uint64_t item_full[2], item_empty[2];
  PromptItem item[2];
  int64_t sums[kScan + 1];
  int order[kSort], length[kSort];  // sequences, longest first; a sequence's items
  uint32_t tmem;
  int stop[3];  // see bar_wait
};

// Items of sequence i.
__device__ __forceinline__ int64_t prompt_items(const PromptArgs &p, int64_t i, bool *bad) {
  const int64_t x0 = p.a.offsets[i], x1 = p.a.offsets[i + 1];
  if (x0 < 0 || x1 < x0 || x1 > p.a.n_tok) {
    *bad = true;
    return 0;
  }
  return (x1 - x0 + 2 * p.tile - 1) / (2 * p.tile) * p.a.hkv;
}

__global__ void __launch_bounds__(kScan) k_prompt_prefix(PromptArgs p) {
  bool bad = false;
  int64_t base = 0;
  for (int64_t i0 = 0; i0 < p.a.n_req; i0 += kScan) {
    const int n = (int)min((int64_t)kScan, p.a.n_req - i0);
    base = scan_units<kScan>(n, p.prefix + i0, base, [&](int k) { return prompt_items(p, i0 + k, &bad); });
  }
  if (bad) flag(p.a.status, kStatusData);
}

// The lanes' rows of `again` once more, one after another by the whole warp: token tok
// of request i, which begins at `first`, head h, on n keys.  A function of its own:
// inlined, its state takes registers from the loop over blocks.
template <int D, bool F16, bool PAGED>
__device__ __noinline__ void redo_rows(const AttendArgs &a, int64_t first, int64_t i, int tok, int h, int64_t n, int64_t bound,
                                       unsigned again, bool all, volatile int *stop) {
  slow_begin(stop);
  while (again) {
    const int r = __ffs(again) - 1;
    again &= again - 1;
    const int rt = __shfl_sync(~0u, tok, r), rh = __shfl_sync(~0u, h, r);
    const int64_t rn = __shfl_sync(~0u, n, r);
    redo_row<D, F16, PAGED>(a, first, i, first + rt, rh, rn, bound, all);
  }
  slow_end(stop);
}

// A place in a ring of stages.
struct RingAt {
  uint32_t st, phase;
  __device__ __forceinline__ RingAt next(uint32_t stages) const {
    return st + 1 == stages ? RingAt{0, phase ^ 1} : RingAt{st + 1, phase};
  }
};

// The warp that issues every product, for kernels of two tiles of rows.
// One instruction takes 64 clocks and few wait in line, so what this warp does
// between two of them soon stops the tensor core.  The loop over whole blocks of
// two tiles has one look at a barrier in each gap, constant descriptors and no
// decision; what comes before and after it goes through `step`.  (With the
// decisions in the loop and waits that answer: 3,900 clocks for a block of both
// tiles with the softmax taken out, 2,048 of them the products'.)
template <int D, bool F16, class Smem>
__device__ __forceinline__ void issue_products(Smem &sm, uint32_t tmem, bool negate, volatile int *stop) {
  constexpr uint32_t kCols = 128;      // columns of a tile's scores
  constexpr int kChunk = 128 * 128;    // bytes of 64 elements of a tile's rows
  const uint32_t id_qk = tc_idesc(128, kPrBlock, F16, negate, false), id_pv = tc_idesc(128, D, F16, false, true);
  constexpr uint32_t kStep = (128 * D * 2) >> 4;  // a tile or block on, in a descriptor
  const uint32_t q_desc = tc_desc(smem_addr(sm.q), 16), k_desc = tc_desc(smem_addr(sm.kv), 16),
                 v_desc = tc_desc(smem_addr(sm.kv), kChunk);
  constexpr uint32_t kStages = Smem::kStages;
  uint32_t q_phase = 0, p_phase = 0;  // bit k of tile k
  // the stages of block j's values and block j + 1's keys and values, and their phases
  RingAt v0{0, 0}, k1{0, 0}, v1{0, 0}, k0{0, 0};  // k0: of an item's first keys
  auto ring = [&](const RingAt &at) { bar_wait(&sm.kv_full[at.st], at.phase, stop); };
  auto release = [&](const RingAt &at) { tc_commit(&sm.kv_empty[at.st]); };
  // scores of tile k on the block at `at`, n steps of 16 keys
  auto qk = [&](int k, const RingAt &at, uint32_t id) {
    const uint32_t qd = q_desc + k * kStep, kd = k_desc + at.st * kStep;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const int off = ((c / 4) * kChunk + (c % 4) * 32) >> 4;
      tc_mma(tmem + k * kCols, qd + off, kd + off, id, c > 0);
    }
    tc_commit(&sm.s_full[k]);
  };
  for (int n = 0;; ++n) {
    bar_wait(&sm.item_full[n & 1], (n >> 1) & 1, stop);
    const PromptItem &it = sm.item[n & 1];
    const int head = __shfl_sync(~0u, it.head, 0), n0 = __shfl_sync(~0u, it.n[0], 0), n1 = __shfl_sync(~0u, it.n[1], 0);
    const int tail0 = __shfl_sync(~0u, it.tail[0], 0), tail1 = __shfl_sync(~0u, it.tail[1], 0);
    if (__any_sync(~0u, head < 0 || *stop)) break;
    if (elect_one()) bar_arrive(&sm.item_empty[n & 1]);
    const int most = max(n0, n1);
    if (most == 0) continue;
    // the scores of a last block only as far as the tile sees it
    auto qk_any = [&](int k, int j, const RingAt &at) {
      const bool last = j + 1 == (k ? n1 : n0);
      const uint32_t id = last ? tc_idesc(128, 0, F16, negate, false) | (uint32_t)((k ? tail1 : tail0) * 2) << 17 : id_qk;
      if (elect_one()) {
        qk(k, at, id);
        if (last) tc_commit(&sm.q_empty[k]);
      }
    };
    // first scores of both tiles
    v0 = k0.next(kStages);
    k1 = v0.next(kStages);
    v1 = k1.next(kStages);
    ring(k0);
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
      if (!(k ? n1 : n0)) continue;
      bar_wait(&sm.q_full[k], q_phase >> k & 1, stop);
      q_phase ^= 1u << k;
      qk_any(k, 0, k0);
    }
    if (elect_one()) release(k0);
    ring(v0);
    int j = 0;
    for (; j + 2 < min(n0, n1); ++j) {
      const uint32_t vd = v_desc + v0.st * kStep;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // half of the weights at a time: the first half's products run while the second is formed
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          bar_wait(half ? &sm.p_full[k] : &sm.p_half[k], p_phase >> k & 1, stop);
          tc_after_sync();
          if (elect_one()) {
#pragma unroll
            for (int c = 4 * half; c < 4 * half + 4; ++c)
              tc_mma_ta(tmem + 256 + k * D, tmem + k * kCols + c * 8, vd + c * (2048 >> 4), id_pv, j > 0 || c > 0);
            if (half && k == 1) release(v0);
          }
        }
        ring(k == 0 ? k1 : v1);  // these keys; the next values, for the next turn
        if (elect_one()) {
          qk(k, k1, id_qk);
          if (k == 1) release(k1);
        }
      }
      p_phase ^= 3;
      v0 = v1;
      k1 = v0.next(kStages);
      v1 = k1.next(kStages);
    }
#pragma unroll 1
    for (; j < most; ++j) {
      const uint32_t vd = v_desc + v0.st * kStep;
      ring(v0);
      if (j + 1 < most) ring(k1);
#pragma unroll 1
      for (int k = 0; k < 2; ++k) {
        const int blocks = k ? n1 : n0;
        if (j >= blocks) continue;
        bar_wait(&sm.p_full[k], p_phase >> k & 1, stop);
        p_phase ^= 1u << k;
        tc_after_sync();
        const int steps = j + 1 == blocks ? (k ? tail1 : tail0) : kPrBlock / 16;
        if (elect_one()) {
#pragma unroll 1
          for (int c = 0; c < steps; ++c)
            tc_mma_ta(tmem + 256 + k * D, tmem + k * kCols + c * 8, vd + c * (2048 >> 4), id_pv, j > 0 || c > 0);
          if (j + 1 == blocks) tc_commit(&sm.o_full[k]);
        }
        if (j + 1 < blocks) qk_any(k, j + 1, k1);
      }
      if (elect_one()) {
        release(v0);
        if (j + 1 < most) release(k1);
      }
      k0 = k1;  // the next item's, after the last block
      v0 = v1;
      k1 = v0.next(kStages);
      v1 = k1.next(kStages);
    }
  }
}

template <int D, bool F16>
__global__ void __launch_bounds__(kPrThreads, 1)
    k_prompt(const __grid_constant__ PromptArgs p, const __grid_constant__ CUtensorMap map_q,
             const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  extern __shared__ unsigned char raw_prompt[];
  using Smem = PromptSmem<D>;
  Smem &sm = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(raw_prompt) + 1023) & ~(uintptr_t)1023);
  const AttendArgs &a = p.a;
  const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, G = a.hq / a.hkv;
  constexpr int kChunk = 128 * 128;  // bytes of 64 elements of a tile's rows
  if (warp == 8) tmem_alloc(&sm.tmem, 512);
  if (threadIdx.x == 9 * 32) {
    map_ahead(&map_q);
    map_ahead(&map_k);
    map_ahead(&map_v);
  }
  if (threadIdx.x == 0) {
    sm.stop[0] = sm.stop[1] = sm.stop[2] = 0;
    sm.item[0].head = sm.item[1].head = -1;
    for (int k = 0; k < 2; ++k) {
      bar_init(&sm.q_full[k], 1);
      bar_init(&sm.q_empty[k], 1);
      bar_init(&sm.s_full[k], 1);
      bar_init(&sm.p_half[k], 4);
      bar_init(&sm.p_full[k], 4);
      bar_init(&sm.o_full[k], 1);
      bar_init(&sm.item_full[k], 1);
      bar_init(&sm.item_empty[k], 9);
    }
    for (int k = 0; k < Smem::kStages; ++k) {
      bar_init(&sm.kv_full[k], 1);
      bar_init(&sm.kv_empty[k], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  bool bad = false;
  const int64_t *sums = p.prefix;
  int64_t items;
  if (p.given) {
    items = sums[a.n_req];
  } else {
    const int n = (int)a.n_req;
    if (n <= kSort) {
      // longest first: a long item begun late would be the call's end.  Each sequence
      // counts those before it
      for (int i = threadIdx.x; i < n; i += kPrThreads) sm.length[i] = (int)min((int64_t)INT32_MAX, prompt_items(p, i, &bad));
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += kPrThreads) {
        const int mine = sm.length[i];
        int at = 0;
        for (int j = 0; j < n; ++j) at += sm.length[j] > mine || (sm.length[j] == mine && j < i) ? 1 : 0;
        sm.order[at] = i;
      }
      __syncthreads();
      items = scan_units<kPrThreads>(n, sm.sums, 0, [&](int k) { return (int64_t)sm.length[sm.order[k]]; });
    } else {
      items = scan_units<kPrThreads>(n, sm.sums, 0, [&](int k) { return prompt_items(p, k, &bad); });
    }
    sums = sm.sums;
  }
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(~0u, sm.tmem, 0);
  volatile int *stop = sm.stop;
  // columns: scores of tile 0, of tile 1, outputs of tile 0, of tile 1
  constexpr uint32_t kCols = 128;
  constexpr float kExp = F16 ? kPrExp : 0.f;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 9 && lane == 0) {
      int64_t u = blockIdx.x;
      int q_used[2] = {0, 0};
      uint32_t kv = 0;
      for (int n = 0;; ++n) {
        if (n >= 2) bar_wait(&sm.item_empty[n & 1], ((n >> 1) - 1) & 1, stop);
        PromptItem &it = sm.item[n & 1];
        if (u >= items || *stop) {
          it.head = -1;
          bar_arrive(&sm.item_full[n & 1]);
          break;
        }
        const int64_t at = find_unit(sums, a.n_req, u), local = u - sums[at], i = a.n_req <= kSort ? sm.order[at] : at;
        const int64_t x0 = a.offsets[i], len = a.offsets[i + 1] - x0, pairs = (len + 2 * p.tile - 1) / (2 * p.tile);
        const int head = (int)(local % a.hkv);
        const int64_t t0 = (pairs - 1 - local / a.hkv) * 2 * p.tile;
        it.first = (int)x0;
        it.t0 = (int)t0;
        it.len = (int)len;
        it.head = head;
        int blocks[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int64_t from = t0 + k * p.tile;
          const int64_t keys = min(len, from + p.tile);
          blocks[k] = from >= len ? 0 : (int)((keys + kPrBlock - 1) / kPrBlock);
          it.n[k] = blocks[k];
          it.tail[k] = (int)(keys - (int64_t)(blocks[k] - 1) * kPrBlock + 15) >> 4;
        }
        bar_arrive(&sm.item_full[n & 1]);
        u = (int64_t)gridDim.x + (int64_t)atomicAdd(&p.counter[0], 1ull);
        const int most = max(blocks[0], blocks[1]);
        for (int j = 0; j < most; ++j) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            // the block's keys, then its values
            if (j == 0 && blocks[k] > 0) {
              // the tiles' queries: tile 0's before the first keys, tile 1's after them
              if (q_used[k] > 0) bar_wait(&sm.q_empty[k], (q_used[k] - 1) & 1, stop);
              ++q_used[k];
              bar_expect(&sm.q_full[k], (uint32_t)(p.tile * G * D * 2));
              for (int c = 0; c < D / 64; ++c)
                tma_load3(sm.q[k] + c * kChunk, &map_q, c * 64, head * G, (int)(x0 + t0 + k * p.tile), &sm.q_full[k]);
            }
            const uint32_t st = kv % Smem::kStages;
            if (kv >= Smem::kStages) bar_wait(&sm.kv_empty[st], (kv / Smem::kStages - 1) & 1, stop);
            if (*stop) break;
            ++kv;
            bar_expect(&sm.kv_full[st], Smem::kTile);
            for (int c = 0; c < D / 64; ++c)
              tma_load3(sm.kv[st] + c * kChunk, k == 0 ? &map_k : &map_v, c * 64, head, (int)(x0 + (int64_t)j * kPrBlock),
                        &sm.kv_full[st]);
          }
        }
      }
      // no load is in flight when the block ends: what was asked for is waited for
      for (uint32_t st = 0; st < Smem::kStages; ++st)
        if (kv > st) bar_wait(&sm.kv_full[st], ((kv - st + Smem::kStages - 1) / Smem::kStages - 1) & 1, stop);
    } else if (warp == 8) {
      issue_products<D, F16>(sm, tmem, a.scale < 0.f, stop);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int k = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane0 = (uint32_t)(warp & 3) * 32 << 16;
    const uint32_t ts = tmem + lane0 + k * kCols, to = tmem + lane0 + 256 + k * D;
    int ss = 0, os = 0;
    for (int n = 0;; ++n) {
      bar_wait(&sm.item_full[n & 1], (n >> 1) & 1, stop);
      const PromptItem it = sm.item[n & 1];
      __syncwarp();
      if (lane == 0) bar_arrive(&sm.item_empty[n & 1]);
      if (__any_sync(~0u, it.head < 0 || *stop)) break;
      const int blocks = k ? it.n[1] : it.n[0];
      if (blocks == 0) continue;
      const int tok = it.t0 + k * p.tile + row / G;  // the row's token in the sequence
      const bool valid = row < p.tile * G && tok < it.len;
      const int lim = valid ? tok + 1 : 0;           // keys that it sees
      const int all = it.t0 + k * p.tile + 1;        // keys that every row of the tile sees
      // A row without a query holds what shared memory held or another sequence's query: its
      // scores count as zero, so that it has no say in when the warp's maxima move
      const float sl = valid ? fabsf(a.scale) : 0.f;
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < blocks; ++j) {
        bar_wait(&sm.s_full[k], ss & 1, stop);
        __syncwarp();
        ++ss;
        tc_after_sync();
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_load32(s + 32 * c, ts + 32 * c);
        tmem_wait_load();
        if ((j + 1) * kPrBlock > all) {
          const int rel = lim - j * kPrBlock;
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (c >= rel) s[c] = 0xff800000u;
        }
        float tops[4] = {m, m, m, m};
#pragma unroll
        for (int c = 0; c < 128; c += 8)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            tops[x] = fmaxf(tops[x], fmaxf(__uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1])));
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        if (j == 0) {
          m = top;
        } else if (__any_sync(~0u, (top - m) * sl > kPrLazy)) {
          const float up = m == -INFINITY ? 1.f : exp2_fast((m - top) * sl);
          m = top;
          l *= up;
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tmem_load16(o, to + c);
            tmem_wait_load();
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * up);
            tmem_store16(to + c, o);
          }
        }
        const float base = m == -INFINITY ? 0.f : m * sl - kExp;
        const uint64_t sl2 = pair(sl, sl), base2 = pair(-base, -base);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          uint32_t w[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            float p0, p1;
            unpair(fma2(pair(__uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1])), sl2, base2), &p0, &p1);
            p0 = exp2_fast(p0);
            p1 = exp2_fast(p1);
            sum[x & 1] = add2(sum[x & 1], pair(p0, p1));
            w[x] = pack_out<F16>(p0, p1);
          }
          tmem_store16(ts + c / 2, w);
          if (c == 32) {
            tmem_wait_store();
            tc_before_sync();
            __syncwarp();
            if (lane == 0) bar_arrive(&sm.p_half[k]);
          }
        }
        float l0, l1;
        unpair(add2(sum[0], sum[1]), &l0, &l1);
        l += l0 + l1;
        tmem_wait_store();
        tc_before_sync();
        __syncwarp();
        if (lane == 0) bar_arrive(&sm.p_full[k]);
      }
      bar_wait(&sm.o_full[k], os & 1, stop);
      __syncwarp();
      ++os;
      tc_after_sync();
      const int64_t t = (int64_t)it.first + tok, h = (int64_t)it.head * G + row % G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bool nan = false;
      uint16_t *const op = (uint16_t *)a.o + (t * a.hq + h) * D;
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        tmem_load32(o, to + c);
        tmem_wait_load();
        if (valid) {
          uint32_t w[16];
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            const float v0 = __uint_as_float(o[2 * y]) * inv, v1 = __uint_as_float(o[2 * y + 1]) * inv;
            nan |= isnan(v0) || isnan(v1);
            w[y] = pack_out<F16>(v0, v1);
          }
          store64(op + c, w, p.wide);
        }
      }
      if (valid && a.lse) a.lse[t * a.hq + h] = l == 0.f ? -INFINITY : (m * sl - kExp + log2f(l)) * 0.6931471805599453f;
      // the outputs are read: the next item's first product may write them (p_full says so, after this)
      unsigned again = __ballot_sync(~0u, nan);
      __syncwarp();
      if (again) redo_rows<D, F16, false>(a, it.first, 0, tok, (int)h, tok + 1, a.n_tok - it.first, again, false, stop);
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  if (sm.stop[0] && threadIdx.x == 0) {
    flag(a.status, kStatusTimeout);
    for (int k = 0; k < 1000; ++k) __nanosleep(1000);  // what was issued may still be at work on shared memory
  }
  if (bad) flag(a.status, kStatusData);
  if (threadIdx.x == 0) {
    // the last CTA out sets the counters back
    if (atomicAdd(&p.counter[1], 1ull) == gridDim.x - 1) {
      p.counter[0] = 0;
      p.counter[1] = 0;
      __threadfence();
    }
  }
  __syncthreads();
  if (warp == 8) tmem_free(tmem, 512);
}

}  // namespace lv
