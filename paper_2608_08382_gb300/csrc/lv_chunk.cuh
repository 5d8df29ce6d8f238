// Attention of many query rows over the 8-bit cache (lv_kv_attend): chunks of a
// prompt on the context before them, and single tokens of wide head groups.
//
// As in lv_prompt.cuh two tiles of up to 128 rows (whole tokens with their G query
// heads) alternate on the tensor core and in softmax.  The products are fp16:
// four warps turn a block of 128 keys' codes into fp16 (exact) in the layout that
// TMA would leave, the softmax warps bring their own query rows to fp16 (bf16
// ones scaled by a power of two to a largest element of 2^14).  A strip of 16 keys
// lies in one block of the cache; its key scale goes into the factor of its
// scores, its value scale vs, as vs / ref, to its weights.  ref follows the
// largest vs of the strips that the row sees, once that is past 2^3 ref, as the
// weights' maximum follows the true one past 2^8: a weight is at most 2^(8 + 4 + 3)
// then.  Rows of an item whose value scales differ by more than 2^14 are done again
// in fp32, each by a warp (kChThin).
//
// The blocks of keys of all items stand in one line and every CTA takes an even
// share of it, so a few long contexts keep every SM busy; an item that several
// CTAs share leaves a part for each, and k_chunk_join adds them in the line's order.
//
// Warps: 0-3 and 4-7 softmax of the two tiles; 8-11 and 12-15 conversion of keys and
// of values; 16 issues the products; 17 hands out the items; 18 copies the codes,
// two blocks ahead, and brings the scales.
//
// Measured: six chunks of 512 tokens on contexts of up to 32,256, 20/4 heads of 128,
// 497 GFLOP: 520 us with the join, 955 TFLOP/s, 0.50 of the measured rate.  A block
// of both tiles takes 4,000 clocks, the products 2,048 of them; shared memory moves
// 320 KB in that time (2,500 clocks at its rate), and a tile's softmax has the
// converting warps beside it on the SM.
#pragma once

#include "lv_decode.cuh"
#include "lv_prompt.cuh"

namespace lv {

constexpr int kChThreads = 640;
constexpr int kChScales = 8;       // blocks whose scales are kept: more than the copies run ahead
constexpr float kChExp = 4.f;      // weights are 2^4 at the maximum they refer to
constexpr float kChRef = 8.f;      // largest vs / ref
constexpr float kChThin = 0x1p-14f;  // least vs / ref under which fp16 holds 2^kChExp to 2^-15 of it (its least step is 2^-24)

struct ChunkArgs {
  AttendArgs a;
  int tile;            // tokens of a tile
  int least_rows;      // requests of fewer rows are k_attend_decode's
  int64_t *prefix;     // [n_req + 1] units before each request
  bool given;
  float *part;         // [CTAs][2][256][D], then m and l [CTAs][2][256][2]
  float *part_ml;
};

template <int D>
struct ChunkSmem {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kStages = 3;   // blocks of keys or values in fp16
  static constexpr int kCodes = 4;    // blocks of them as codes, on their way
  unsigned char q[2][kTile];
  unsigned char kv[kStages][kTile];
  unsigned char code[kCodes][128 * D];  // at the start: the requests' running sums
  uint64_t code_full[kCodes], code_empty[kCodes];
  uint64_t q_full[2], q_empty[2], kv_full[kStages], kv_empty[kStages], s_full[2], p_half[2], p_full[2], o_full[2];
  uint64_t item_full[2], item_empty[2], scale_full[kChScales];
  PromptItem item[2];
  alignas(16) float ks[kChScales][8], vs[kChScales][8];  // of a block's strips
  float top_vs[kChScales];          // the largest |vs| of a block
  int thin[kChScales];              // the value scales of the item so far lie further apart than kChThin
  uint32_t hidden[kChScales];       // its strips whose block is hidden, a bit each
  uint32_t state[kCodes][8];  // of a block's strips: keys that are there, bit 8: their sign is changed
  int64_t req[2], from[2];  // of each item: its request, its first block
  int whole[2], slot[2];    // no other CTA has a share of it; where its part goes
  uint32_t tmem;
  int stop[3];  // see bar_wait
};

// Pairs of tiles of a request, and blocks of keys of each, counted alike.
__device__ __forceinline__ int64_t chunk_pairs(const ChunkArgs &c, const Span &s) {
  const int G = c.a.hq / c.a.hkv;
  return (int64_t)s.p * G < c.least_rows ? 0 : (s.p + 2 * c.tile - 1) / (2 * c.tile);
}
__device__ __forceinline__ int64_t chunk_blocks(const ChunkArgs &c, const Span &s) {
  return max((int64_t)1, (row_limit(c.a, s, s.p - 1) + kPrBlock - 1) / kPrBlock);
}
__device__ __forceinline__ int64_t chunk_units(const ChunkArgs &c, int64_t i, bool *bad) {
  const Span s = request_span(c.a, i, bad);
  return s.p == 0 ? 0 : chunk_pairs(c, s) * c.a.hkv * chunk_blocks(c, s);
}

__global__ void __launch_bounds__(kScan) k_chunk_prefix(ChunkArgs c) {
  bool bad = false;
  int64_t base = 0;
  for (int64_t i0 = 0; i0 < c.a.n_req; i0 += kScan) {
    const int n = (int)min((int64_t)kScan, c.a.n_req - i0);
    base = scan_units<kScan>(n, c.prefix + i0, base, [&](int k) { return chunk_units(c, i0 + k, &bad); });
  }
  if (bad) flag(c.a.status, kStatusData);
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <int D, bool F16>
__global__ void __launch_bounds__(kChThreads, 1) k_chunk(const __grid_constant__ ChunkArgs c) {
  extern __shared__ unsigned char raw_prompt[];
  using Smem = ChunkSmem<D>;
  Smem &sm = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(raw_prompt) + 1023) & ~(uintptr_t)1023);
  const AttendArgs &a = c.a;
  const CacheView &cv = a.cache;
  const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, G = a.hq / a.hkv;
  constexpr int kChunk = 128 * 128;  // bytes of 64 elements of a tile's rows
  wait_previous();
  if (warp == 16) tmem_alloc(&sm.tmem, 512);
  if (threadIdx.x == 0) {
    sm.stop[0] = sm.stop[1] = sm.stop[2] = 0;
    sm.item[0].head = sm.item[1].head = -1;
    for (int k = 0; k < 2; ++k) {
      bar_init(&sm.q_full[k], 4);
      bar_init(&sm.q_empty[k], 1);
      bar_init(&sm.s_full[k], 1);
      bar_init(&sm.p_half[k], 4);
      bar_init(&sm.p_full[k], 4);
      bar_init(&sm.o_full[k], 1);
      bar_init(&sm.item_full[k], 1);
      bar_init(&sm.item_empty[k], 18);
    }
    for (int k = 0; k < Smem::kStages; ++k) {
      bar_init(&sm.kv_full[k], 4);
      bar_init(&sm.kv_empty[k], 1);
    }
    for (int k = 0; k < Smem::kCodes; ++k) {
      bar_init(&sm.code_full[k], 8);
      bar_init(&sm.code_empty[k], 4);
    }
    for (int k = 0; k < kChScales; ++k) bar_init(&sm.scale_full[k], 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  bool bad = false;
  const int64_t *sums = c.prefix;
  int64_t units;
  if (c.given) {
    units = sums[a.n_req];
  } else {
    int64_t *const S = reinterpret_cast<int64_t *>(sm.code);  // before any copy arrives there
    static_assert(sizeof(sm.code) >= 8 * (kScan + 1), "room for the sums");
    units = scan_units<kChThreads>((int)a.n_req, S, 0, [&](int k) { return chunk_units(c, k, &bad); });
    sums = S;
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i <= a.n_req; i += kChThreads) c.prefix[i] = S[i];
  }
  // the CTA's share of the line and the request it begins in
  const int64_t end = warp_start(blockIdx.x + 1, gridDim.x, units), begin = warp_start(blockIdx.x, gridDim.x, units);
  const int64_t first_req = find_unit(sums, a.n_req, begin), first_sum = sums[first_req];
  let_next();
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the copies will write where the sums were
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = __shfl_sync(~0u, sm.tmem, 0);
  volatile int *stop = sm.stop;
  constexpr uint32_t kCols = 128;

  if (warp >= 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 16) {
      issue_products<D, true>(sm, tmem, a.scale < 0.f, stop);
    } else if (warp == 17 && lane == 0) {
      // the share, an item or a part of one at a time
      int64_t u = begin, i = first_req, before = first_sum;  // units before request i
      for (int n = 0;; ++n) {
        if (n >= 2) bar_wait(&sm.item_empty[n & 1], ((n >> 1) - 1) & 1, stop);
        PromptItem &it = sm.item[n & 1];
        if (u >= end || *stop) {
          it.head = -1;
          bar_arrive(&sm.item_full[n & 1]);
          break;
        }
        bool ignore = false;
        if (c.given) {  // among many requests looked for, not walked to: the others' waits are bounded
          if (u >= sums[i + 1]) i = find_unit(sums, a.n_req, u), before = sums[i];
        } else {
          for (int64_t more; u >= before + (more = chunk_units(c, i, &ignore)); ++i) before += more;
        }
        const Span sp = request_span(a, i, &ignore);
        const int64_t blocks = chunk_blocks(c, sp), local = u - before, seg = local / blocks;
        const int64_t b0 = local % blocks, b1 = min(blocks, b0 + end - u);
        const int t0 = (int)(seg / a.hkv) * 2 * c.tile;
        it.first = (int)sp.first;
        it.t0 = t0;
        it.len = sp.p;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int from = t0 + k * c.tile, last = min(sp.p, from + c.tile) - 1;
          int64_t n_all = 0, keys = 0;
          if (from < sp.p) {
            keys = row_limit(a, sp, last);
            n_all = max((int64_t)1, (keys + kPrBlock - 1) / kPrBlock);
          }
          const int64_t top = min(n_all, b1);
          it.n[k] = (int)max((int64_t)0, top - b0);
          it.tail[k] = top == n_all ? (int)max((int64_t)1, (keys - (n_all - 1) * kPrBlock + 15) >> 4) : kPrBlock / 16;
        }
        sm.req[n & 1] = i;
        sm.from[n & 1] = b0;
        sm.whole[n & 1] = b0 == 0 && b1 == blocks;
        sm.slot[n & 1] = (int)blockIdx.x * 2 + (u == begin ? 0 : 1);
        it.head = (int)(seg % a.hkv);
        bar_arrive(&sm.item_full[n & 1]);
        u += b1 - b0;
      }
    } else if (warp == 18) {
      // The codes' copies, a strip a lane: 16 keys of one block and head are 16 D bytes
      // in a row.  Eight lanes a block; ids and scales of 32 strips (four blocks) at a
      // time, the next 32 ahead.
      RingAt code{0, 1};  // the first turn's slots are free
      uint32_t block = 0;
      for (int n = 0;; ++n) {
        bar_wait(&sm.item_full[n & 1], (n >> 1) & 1, stop);
        const int head = sm.item[n & 1].head, most = max(sm.item[n & 1].n[0], sm.item[n & 1].n[1]);
        const int64_t i = sm.req[n & 1], from = sm.from[n & 1];
        __syncwarp();
        if (lane == 0) bar_arrive(&sm.item_empty[n & 1]);
        if (__any_sync(~0u, head < 0 || *stop)) break;
        bool ignore = false;
        const Span sp = request_span(a, i, &ignore);
        const int64_t keys = row_limit(a, sp, sp.p - 1);
        float most_vs = 0.f, least_vs = INFINITY;  // of the item's blocks
        int32_t id[2];
        float ks[2], vs[2];
        auto look_up = [&](int set, int group) {
          const int64_t strip = (from + 4 * group) * 8 + lane;
          id[set] = -1;
          ks[set] = vs[set] = 0.f;
          if (4 * group + (lane >> 3) < most && strip * 16 < keys) {
            int32_t b = a.table[i * a.width + ((strip * 16) >> cv.log_b)];
            if (b < -1 || b >= cv.n_blocks) {
              bad = true;
              b = -1;
            }
            id[set] = b;
            if (b >= 0) {
              ks[set] = cv.k_scale[(int64_t)b * cv.heads + head];
              vs[set] = cv.v_scale[(int64_t)b * cv.heads + head];
            }
          }
        };
        if (most > 0) look_up(0, 0);
        for (int j = 0; j < most; ++j) {
          if ((j & 3) == 0) {
            if (j > 0) id[0] = id[1], ks[0] = ks[1], vs[0] = vs[1];
            look_up(1, j / 4 + 1);
          }
          const bool mine = (lane >> 3) == (j & 3);
          const int strip = lane & 7;
          const int64_t pos = (from + j) * kPrBlock + strip * 16;
          const int there = id[0] < 0 ? 0 : (int)max((int64_t)0, min((int64_t)16, keys - pos));
          float top = fabsf(vs[0]), low = top > kLeastScale ? top : INFINITY;
#pragma unroll
          for (int x = 1; x < 8; x <<= 1) {
            top = fmaxf(top, __shfl_xor_sync(~0u, top, x));
            low = fminf(low, __shfl_xor_sync(~0u, low, x));
          }
          most_vs = fmaxf(most_vs, __shfl_sync(~0u, top, (j & 3) * 8));
          least_vs = fminf(least_vs, __shfl_sync(~0u, low, (j & 3) * 8));
          const uint32_t gone = __ballot_sync(~0u, id[0] < 0) >> (lane & 24) & 255;
          if (mine) {
            const uint32_t at = (block + j) % kChScales;
            sm.ks[at][strip] = fabsf(ks[0]);
            sm.vs[at][strip] = vs[0];
            if (strip == 0) sm.top_vs[at] = top, sm.thin[at] = least_vs < kChThin * most_vs, sm.hidden[at] = gone;
            bar_arrive(&sm.scale_full[at]);
          }
          const int64_t off = ((((int64_t)max(id[0], 0) * cv.heads + head) << cv.log_b) + (pos & ((1 << cv.log_b) - 1))) * D;
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            bar_wait(&sm.code_empty[code.st], code.phase, stop);
            if (mine) {
              sm.state[code.st][strip] = (uint32_t)there | (v == 0 && ks[0] < 0.f ? 256u : 0u);
              if (there > 0 && !*stop) {
                bar_expect(&sm.code_full[code.st], there * D);
                copy_bytes(sm.code[code.st] + strip * 16 * D, (v ? cv.v : cv.k) + off, there * D, &sm.code_full[code.st]);
              } else {
                bar_arrive(&sm.code_full[code.st]);
              }
            }
            __syncwarp();
            code = code.next(Smem::kCodes);
          }
        }
        block += most;
      }
    }
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    // Codes to fp16, 32 keys of each block a warp: a lane takes 8 codes of a key, which
    // become one piece of 16 bytes; a quarter warp stores eight pieces of one row of
    // 128 bytes, wherever the swizzle puts them, and no two of them meet in a bank.
    constexpr int kLanes = D / 8, kKeys = 32 / kLanes, kSteps = 32 / kKeys;  // lanes a key, keys a load, loads
    const int w = warp & 3, sub = lane % kLanes, key_of = lane / kLanes;
    // warps 8 to 11 the keys, 12 to 15 the values, which take turns in both rings
    RingAt code{0, 0}, to{0, 1};  // the first turn's stages are free
    if (warp >= 12) code = code.next(Smem::kCodes), to = to.next(Smem::kStages);
    for (int n = 0;; ++n) {
      bar_wait(&sm.item_full[n & 1], (n >> 1) & 1, stop);
      const int head = sm.item[n & 1].head, most = max(sm.item[n & 1].n[0], sm.item[n & 1].n[1]);
      __syncwarp();
      if (lane == 0) bar_arrive(&sm.item_empty[n & 1]);
      if (__any_sync(~0u, head < 0 || *stop)) break;
      for (int j = 0; j < most; ++j) {
        bar_wait(&sm.code_full[code.st], code.phase, stop);
        bar_wait(&sm.kv_empty[to.st], to.phase, stop);
        __syncwarp();
        const uint32_t state0 = sm.state[code.st][2 * w], state1 = sm.state[code.st][2 * w + 1];
        const unsigned char *from = sm.code[code.st] + 32 * w * D + key_of * D + sub * 8;
        unsigned char *const at = sm.kv[to.st] + (sub / 8) * kChunk + (32 * w + key_of) * 128;
        if (state0 == 16 && state1 == 16) {
#pragma unroll
          for (int x = 0; x < kSteps; ++x) {
            const uint2 q = *reinterpret_cast<const uint2 *>(from + x * kKeys * D);
            *reinterpret_cast<uint4 *>(at + x * kKeys * 128 + ((sub % 8 ^ (x * kKeys + key_of) % 8) << 4)) =
                make_uint4(lo_half2(q.x), hi_half2(q.x), lo_half2(q.y), hi_half2(q.y));
          }
        } else {  // keys that are not there, or signs to change
#pragma unroll 1
          for (int x = 0; x < kSteps; ++x) {
            const int key = x * kKeys + key_of;
            const uint32_t st = key >= 16 ? state1 : state0, flip = st & 256 ? 0x80808080u : 0u;
            uint2 q = *reinterpret_cast<const uint2 *>(from + x * kKeys * D);
            q = (uint32_t)(key & 15) < (st & 31) ? make_uint2(q.x ^ flip, q.y ^ flip) : make_uint2(0, 0);
            *reinterpret_cast<uint4 *>(at + x * kKeys * 128 + ((sub % 8 ^ key % 8) << 4)) =
                make_uint4(lo_half2(q.x), hi_half2(q.x), lo_half2(q.y), hi_half2(q.y));
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          bar_arrive(&sm.kv_full[to.st]);
          bar_arrive(&sm.code_empty[code.st]);
        }
        code = code.next(Smem::kCodes).next(Smem::kCodes);
        to = to.next(Smem::kStages).next(Smem::kStages);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    const int k = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane0 = (uint32_t)(warp & 3) * 32 << 16;
    const uint32_t ts = tmem + lane0 + k * kCols, to = tmem + lane0 + 256 + k * D;
    uint32_t ss = 0, qs = 0, os = 0, block = 0;
    for (int n = 0;; ++n) {
      bar_wait(&sm.item_full[n & 1], (n >> 1) & 1, stop);
      const PromptItem it = sm.item[n & 1];
      const int64_t i = sm.req[n & 1], from = sm.from[n & 1];
      const bool whole = sm.whole[n & 1];
      const int slot = sm.slot[n & 1];
      __syncwarp();
      if (lane == 0) bar_arrive(&sm.item_empty[n & 1]);
      if (__any_sync(~0u, it.head < 0 || *stop)) break;
      const int blocks = k ? it.n[1] : it.n[0], most = max(it.n[0], it.n[1]);
      const uint32_t block0 = block;
      block += most;
      const int tok = it.t0 + k * c.tile + row / G, h = it.head * G + row % G;
      const bool valid = row < c.tile * G && tok < it.len;
      float m = -INFINITY, l = 0.f, ref = 0.f, inv_ref = 0.f;
      int thin = 0;                // value scales so far apart that a weight may have lost too many bits
      int64_t lim = 0, bound = 0;  // keys that the row sees, that the request has
      if (blocks > 0) {
        bool ignore = false;
        const Span sp = request_span(a, i, &ignore);
        lim = valid ? row_limit(a, sp, tok) : 0;
        bound = row_limit(a, sp, sp.p - 1);
        const int64_t all = row_limit(a, sp, it.t0 + k * c.tile);  // what every row of the tile sees
        // the row's query
        float sl = fabsf(a.scale);
        if (qs > 0) bar_wait(&sm.q_empty[k], (qs - 1) & 1, stop);
        __syncwarp();
        {
          const uint16_t *qp = (const uint16_t *)a.q + ((int64_t)it.first + tok) * a.q_stride + (int64_t)h * D;
          const uint4 *qv = reinterpret_cast<const uint4 *>(qp);
          float up = 1.f;
          if (!F16) {
            uint32_t top = 0;
#pragma unroll 4
            for (int y = 0; y < D / 8; ++y) {
              const uint4 x = valid ? qv[y] : make_uint4(0, 0, 0, 0);
              const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int z = 0; z < 4; ++z) top = max(top, max(v[z] & 0x7fff0000u, (v[z] & 0x7fffu) << 16));
            }
            const int e = top ? min(max((int)(top >> 23) - 127, -100), 127) : 14;  // 2^e <= largest < 2^(e+1)
            up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
            sl *= __uint_as_float((uint32_t)(127 - 14 + e) << 23);
          }
#pragma unroll 4
          for (int y = 0; y < D / 8; ++y) {
            uint4 x = valid ? qv[y] : make_uint4(0, 0, 0, 0);
            if (!F16) {
              uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                const float2 f = unpack2<false>(v[z]);
                v[z] = pack_half2(f.x * up, f.y * up);
              }
              x = make_uint4(v[0], v[1], v[2], v[3]);
            }
            *reinterpret_cast<uint4 *>(sm.q[k] + (y / 8) * kChunk + row * 128 + (((y % 8) ^ (row & 7)) << 4)) = x;
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(&sm.q_full[k]);
          ++qs;
        }
        // in keys from the item's first on: what the row sees, what every row of the tile sees
        const int sees = (int)max((int64_t)0, min((int64_t)INT32_MAX, lim - from * kPrBlock));
        const int all_see = (int)max((int64_t)0, min((int64_t)INT32_MAX, all - from * kPrBlock));
        float f[8], r[8];  // a strip's factor of scores, its value scale
        float top_vs = 0.f;
        uint32_t hidden = 0;
        auto scales = [&](uint32_t b) {
          bar_wait(&sm.scale_full[b % kChScales], (b / kChScales) & 1, stop);
          const float4 *kp = reinterpret_cast<const float4 *>(sm.ks[b % kChScales]);
          const float4 *vp = reinterpret_cast<const float4 *>(sm.vs[b % kChScales]);
          const float4 k0 = kp[0], k1 = kp[1], v0 = vp[0], v1 = vp[1];
          top_vs = sm.top_vs[b % kChScales];
          hidden = sm.hidden[b % kChScales];
          f[0] = k0.x * sl, f[1] = k0.y * sl, f[2] = k0.z * sl, f[3] = k0.w * sl;
          f[4] = k1.x * sl, f[5] = k1.y * sl, f[6] = k1.z * sl, f[7] = k1.w * sl;
          r[0] = v0.x, r[1] = v0.y, r[2] = v0.z, r[3] = v0.w;
          r[4] = v1.x, r[5] = v1.y, r[6] = v1.z, r[7] = v1.w;
        };
        for (int j = 0; j < blocks; ++j) {
          // A block's scales are there before its scores.  Of the first block they are
          // looked at after the scores: earlier an older phase of their barrier could be
          // taken for this one.
          if (j > 0) scales(block0 + j);
          bar_wait(&sm.s_full[k], ss & 1, stop);
          ++ss;
          if (j == 0) scales(block0);
          __syncwarp();
          tc_after_sync();
          // what the row does not see goes to -infinity where it stands
          if (hidden || (j + 1) * kPrBlock > all_see) {
            const int rel = sees - j * kPrBlock;
#pragma unroll 1
            for (int x = 0; x < 128; x += 16) {
              uint32_t v[16];
              tmem_load16(v, ts + x);
              tmem_wait_load();
              const bool no = hidden >> (x / 16) & 1;
#pragma unroll
              for (int y = 0; y < 16; ++y)
                if (no || x + y >= rel) v[y] = 0xff800000u;
              tmem_store16(ts + x, v);
            }
            tmem_wait_store();
            // A value scale is the row's from the first key of its strip on that the row sees: one
            // of later keys would raise ref and take the weights' bits.
            top_vs = 0.f;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              const bool no = (hidden >> x & 1) || 16 * x >= rel;  // nothing of the strip is seen
              if (no) r[x] = 0.f;
              if (no || f[x] == 0.f) f[x] = 1e-37f;  // it must stay there, under a NaN scale too
              top_vs = fmaxf(top_vs, fabsf(r[x]));
            }
          }
          // The scores are read from tensor memory twice, for the maximum and for the
          // weights: a thread that keeps its 128 has no registers left for the rest.
          float top = m;
          uint32_t s[2][32];
          tmem_load32(s[0], ts);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            tmem_wait_load();
            tmem_load32(s[(x + 1) & 1], ts + 32 * ((x + 1) & 3));  // after the last the first again
            const uint32_t *v = s[x & 1];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
              for (int z = 0; z < 16; z += 4) {
                t0 = fmaxf(t0, fmaxf(__uint_as_float(v[16 * y + z]), __uint_as_float(v[16 * y + z + 1])));
                t1 = fmaxf(t1, fmaxf(__uint_as_float(v[16 * y + z + 2]), __uint_as_float(v[16 * y + z + 3])));
              }
              top = fmaxf(top, fmaxf(t0, t1) * f[2 * x + y]);
            }
          }
          const bool grow_ref = !(top_vs <= kChRef * ref);
          if (j == 0) {
            m = top;
            ref = fmaxf(top_vs, kLeastRef);
            inv_ref = 1.f / ref;
          } else if (__any_sync(~0u, top - m > kPrLazy || grow_ref)) {
            const float up = m == -INFINITY ? 1.f : exp2_fast(m - top);
            m = top;
            l *= up;
            const float nref = fmaxf(ref, top_vs), shrink = up * (ref / nref);
            ref = nref;
            inv_ref = 1.f / ref;
#pragma unroll 1
            for (int x = 0; x < D; x += 16) {
              uint32_t o[16];
              tmem_load16(o, to + x);
              tmem_wait_load();
#pragma unroll
              for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * shrink);
              tmem_store16(to + x, o);
            }
          }
          const float base = m == -INFINITY ? -kChExp : m - kChExp;
          const uint64_t base2 = pair(-base, -base);
          uint64_t sum[2] = {0, 0};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            tmem_wait_load();
            if (x < 3) tmem_load32(s[(x + 1) & 1], ts + 32 * (x + 1));
            const uint32_t *v = s[x & 1];
            uint32_t w[16];
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              const float fs = f[2 * x + y / 8], rs = r[2 * x + y / 8] * inv_ref;
              float p0, p1;
              unpair(fma2(pair(__uint_as_float(v[2 * y]), __uint_as_float(v[2 * y + 1])), pair(fs, fs), base2), &p0, &p1);
              const uint64_t pp = pair(exp2_fast(p0), exp2_fast(p1));
              sum[y & 1] = add2(sum[y & 1], pp);
              unpair(mul2(pp, pair(rs, rs)), &p0, &p1);
              w[y] = pack_half2(p0, p1);
            }
            tmem_store16(ts + 16 * x, w);  // over columns that were read
            if (x == 1) {
              tmem_wait_store();
              tc_before_sync();
              __syncwarp();
              if (lane == 0) bar_arrive(&sm.p_half[k]);
            }
          }
          float l0, l1;
          unpair(add2(sum[0], sum[1]), &l0, &l1);
          l += l0 + l1;
          thin = sm.thin[(block0 + j) % kChScales];
          tmem_wait_store();
          tc_before_sync();
          __syncwarp();
          if (lane == 0) bar_arrive(&sm.p_full[k]);
        }
        bar_wait(&sm.o_full[k], os & 1, stop);
        ++os;
        __syncwarp();
        tc_after_sync();
      }
      const int64_t t = (int64_t)it.first + tok;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t at = (int64_t)slot * 256 + k * 128 + row;
      bool nan = false;
      if (blocks > 0) {
#pragma unroll 1
        for (int x = 0; x < D; x += 16) {
          uint32_t o[16];
          tmem_load16(o, to + x);
          tmem_wait_load();
          if (!valid) continue;
          if (whole) {
            uint4 *op = reinterpret_cast<uint4 *>((uint16_t *)a.o + (t * a.hq + h) * D + x);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              uint32_t w[4];
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                const float v0 = __uint_as_float(o[8 * y + 2 * z]) * inv * ref, v1 = __uint_as_float(o[8 * y + 2 * z + 1]) * inv * ref;
                nan |= isnan(v0) || isnan(v1);
                w[z] = pack_out<F16>(v0, v1);
              }
              op[y] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          } else {
            float4 *pp = reinterpret_cast<float4 *>(c.part + at * D + x);
#pragma unroll
            for (int y = 0; y < 4; ++y)
              pp[y] = make_float4(__uint_as_float(o[4 * y]) * ref, __uint_as_float(o[4 * y + 1]) * ref,
                                  __uint_as_float(o[4 * y + 2]) * ref, __uint_as_float(o[4 * y + 3]) * ref);
          }
        }
      }
      if (valid && whole && a.lse)
        a.lse[t * a.hq + h] = l == 0.f ? -INFINITY : (m - kChExp + log2f(l)) * 0.6931471805599453f;
      if (!whole) *reinterpret_cast<float2 *>(c.part_ml + 2 * at) = make_float2(m, thin ? -l : l);  // the join does it again
      unsigned again = __ballot_sync(~0u, nan || (thin && whole && valid));
      __syncwarp();
      if (again) redo_rows<D, F16, true>(a, it.first, i, tok, h, lim, bound, again, thin != 0, stop);
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  if (sm.stop[0] && threadIdx.x == 0) flag(a.status, kStatusTimeout);
  if (sm.stop[0])
    for (int k = 0; k < 1000; ++k) __nanosleep(1000);  // products that were issued may still read shared memory
  if (bad) flag(a.status, kStatusData);
  __syncthreads();
  if (warp == 16) tmem_free(tmem, 512);
}

// The items that several CTAs shared: a warp a row adds its parts in the line's
// order.  A part whose keys the row does not see has l = 0 and no sums; one whose
// weights lost bits has its l negative, and its row is done again.
template <int D, bool F16>
__global__ void __launch_bounds__(256) k_chunk_join(ChunkArgs c, int ctas) {
  constexpr int E = D / 32, kBatch = 4;
  const AttendArgs &a = c.a;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, G = a.hq / a.hkv;
  wait_previous();
  const int64_t units = c.prefix[a.n_req], i = blockIdx.x;
  if (c.prefix[i + 1] == c.prefix[i]) return;
  bool ignore = false;
  const Span sp = request_span(a, i, &ignore);
  const int64_t blocks = chunk_blocks(c, sp), items = chunk_pairs(c, sp) * a.hkv;
  // a CTA takes a quarter of an item's rows, its warps eight each
  for (int64_t y = blockIdx.y; y < items * 4; y += gridDim.y) {
    const int64_t seg = y >> 2, u0 = c.prefix[i] + seg * blocks;
    const int64_t w0 = warp_of(u0, ctas, units), w1 = warp_of(u0 + blocks - 1, ctas, units);
    if (w0 == w1) continue;
    const int64_t slot0 = w0 * 2 + (warp_start(w0, ctas, units) < u0 ? 1 : 0);
    for (int r = (int)(y & 3) * 64 + w; r < ((int)(y & 3) + 1) * 64; r += 8) {
      const int row = r & 127, k = r >> 7;
      const int tok = (int)seg / a.hkv * 2 * c.tile + k * c.tile + row / G, h = (int)seg % a.hkv * G + row % G;
      if (row >= c.tile * G || tok >= sp.p) continue;
      float top = -INFINITY, l = 0.f, o[E];
      bool thin = false;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
      for (int64_t x0 = w0; x0 <= w1; x0 += kBatch) {
        float pm[kBatch], pl[kBatch], po[kBatch][E], nm = top;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int64_t x = x0 + b;
          pm[b] = -INFINITY, pl[b] = 0.f;
          if (x <= w1) {
            const int64_t at = (x == w0 ? slot0 : x * 2) * 256 + r;
            const float2 ml = *reinterpret_cast<const float2 *>(c.part_ml + 2 * at);
            pm[b] = ml.x, pl[b] = ml.y;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              const float2 v = *reinterpret_cast<const float2 *>(c.part + at * D + lane * E + e);
              po[b][e] = v.x, po[b][e + 1] = v.y;
            }
          }
          nm = fmaxf(nm, pm[b]);
        }
        const float base = nm == -INFINITY ? 0.f : nm, up = top == -INFINITY ? 1.f : exp2_fast(top - base);
        l *= up;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= up;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          if (pl[b] == 0.f) continue;
          const float f = pm[b] == -INFINITY ? 1.f : exp2_fast(pm[b] - base);
          l += fabsf(pl[b]) * f;
          thin |= pl[b] < 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] += po[b][e] * f;
        }
        top = nm;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t t = sp.first + tok;
      bool nan = false;
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        *reinterpret_cast<uint32_t *>((uint16_t *)a.o + (t * a.hq + h) * D + lane * E + e) = pack_out<F16>(o[e] * inv, o[e + 1] * inv);
        nan |= isnan(o[e]) || isnan(o[e + 1]);
      }
      if (a.lse && lane == 0) a.lse[t * a.hq + h] = l == 0.f ? -INFINITY : (top - kChExp + log2f(l)) * 0.6931471805599453f;
      if (__any_sync(~0u, nan || thin)) redo_row<D, F16, true>(a, sp.first, i, t, h, row_limit(a, sp, tok), row_limit(a, sp, sp.p - 1), thin);
    }
  }
}

}  // namespace lv
