// Products of a step's tokens with a layer's weights (lv_linear, lv_gated_linear) on
// the tensor cores.
//
// D = W X^T: the weights' rows stand along the accumulator's 128 lanes and the tokens
// along its columns, so that a call of any number of tokens, from one up, fills the
// lanes and pays columns for the tokens it has (in steps of 16).  Both operands come
// by TMA in pieces of 64 along the sum, 128 bytes a row, swizzled; what a piece has
// past a row's end or past the last row is zero in both.  The gated form puts 64 rows
// of each weight array into the lanes of one accumulator, so that it is the same
// product: its two halves meet in shared memory on the way out.  There the bias is
// added, the activation applied and the residual added in fp32, and what comes is
// rounded once.
//
// Two kernels: k_product for few tokens, where the weights' bytes bound the call, and
// k_product_pair for many, where the products do.
#pragma once

#include "lv_attend.cuh"
#include "lv_cut.h"
#include "lv_tc.cuh"

namespace lv {

struct LinearArgs {
  const void *bias[2];       // [1]: of the gated form's second weights
  const void *residual;
  void *y;
  int64_t r_stride, y_stride;
  int64_t n_tok;
  int d_out, act;
  int chunks;                // pieces of 64 along the sum
  int tokens;                // columns of a tile, a multiple of 16
  int stages, room;          // of the stages, and the bytes that they or the sums take (k_product)
  int split;                 // CTAs that share a tile's sum (k_product)
  int64_t token_tiles, tiles;
  int *status;
};

template <bool F16>
__device__ __forceinline__ float value_of(uint16_t b) {
  return F16 ? __half2float(__ushort_as_half(b)) : __uint_as_float((uint32_t)b << 16);
}

// 1 / (1 + exp(-x)), of whichever sign the exponential is small: nothing overflows, and
// far to the left what is left is exp(x) and not the reciprocal of an infinity.
__device__ __forceinline__ float logistic(float x) {
  const float e = __expf(-fabsf(x));
  return __fdividef(x < 0.f ? e : 1.f, 1.f + e);
}
// The activation in fp32.  The two forms of GELU are written without the difference of
// nearly equal numbers that 1 + erf and 1 + tanh have at the left: erfc, and 1 + tanh u =
// 2 / (1 + exp(-2u)).
template <int ACT>
__device__ __forceinline__ float activated(float x) {
  if (ACT == LV_ACT_SILU) return x * logistic(x);
  if (ACT == LV_ACT_GELU) return 0.5f * x * erfcf(x * -0.70710678118654752f);
  if (ACT == LV_ACT_GELU_TANH) return x * logistic(1.5957691216057308f * (x + 0.044715f * x * x * x));
  return ACT == LV_ACT_RELU && x < 0.f ? 0.f : x;
}
template <int ACT, int N>
__device__ __forceinline__ void activate_all(float *v) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = activated<ACT>(v[k]);
}
// Of a whole array: one decision.
template <class A>
__device__ __forceinline__ void activate(A &array, int act) {
  constexpr int kN = sizeof(A) / sizeof(float);
  float *const v = reinterpret_cast<float *>(&array);
  if (act == LV_ACT_NONE) return;
  switch (act) {
    case LV_ACT_SILU: activate_all<LV_ACT_SILU, kN>(v); break;
    case LV_ACT_GELU: activate_all<LV_ACT_GELU, kN>(v); break;
    case LV_ACT_GELU_TANH: activate_all<LV_ACT_GELU_TANH, kN>(v); break;
    default: activate_all<LV_ACT_RELU, kN>(v);
  }
}

// Outputs of a CTA's tile.
template <bool GATED>
__host__ __device__ constexpr int tile_outputs() { return GATED ? kRows / 2 : kRows; }

template <bool F16>
__device__ __forceinline__ void unpack8(const uint4 &b, float *v) {
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = value_of<F16>((uint16_t)(w[k >> 1] >> (k & 1) * 16));
}

// Two fp32 products in one instruction, and eight 16-bit values as pairs of floats.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
template <bool F16>
__device__ __forceinline__ void unpack_pairs(const uint4 &b, uint64_t *v) {
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (F16) {
      const float2 f = __half22float2(*(const __half2 *)&w[k]);
      v[k] = pair(f.x, f.y);
    } else {
      v[k] = pair(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
    }
  }
}

// The biases of outputs o .. o + 7.
template <bool GATED, bool F16>
__device__ __forceinline__ void load_bias(const LinearArgs &a, int o, float (*b)[8]) {
#pragma unroll
  for (int k = 0; k < (GATED ? 2 : 1); ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      b[k][e] = a.bias[k] && o + e < a.d_out ? value_of<F16>(((const uint16_t *)a.bias[k])[o + e]) : 0.f;
}

// 16 rows by 16 columns of tensor memory, as four 8 x 8 blocks: r[4 h + 2 g + k] is column
// 8 h + 2 (lane & 3) + k of row 8 g + lane / 4.
__device__ __forceinline__ void tmem_load_blocks(uint32_t *r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(at));
}
// Four 8 x 8 blocks of 16-bit values, a pair of columns of row lane / 4 a register, to
// or from shared memory with their columns as its rows: lane l gives the place of
// column l & 7 of block l / 8.
__device__ __forceinline__ void store_turned(uint32_t at, const uint32_t *w) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]),
               "r"(w[2]), "r"(w[3])
               : "memory");
}
__device__ __forceinline__ void load_turned(uint32_t *w, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
               : "r"(at)
               : "memory");
}

// Eight 16-bit values in a row from memory, to shared memory or to registers with zeros
// for those that are not there, or to memory; n of them are.
__device__ __forceinline__ void copy_some(uint4 *to, const uint16_t *p, int n) {
  const int bytes = min(max(n, 0), 8) * 2;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(to)), "l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 load_some(const uint16_t *p, int n) {
  if (n >= 8) return *(const uint4 *)p;
  uint32_t w[4] = {};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) w[e >> 1] |= (uint32_t)p[e] << (e & 1) * 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_some(uint16_t *p, const uint4 &v, int n) {
  if (n >= 8) {
    *(uint4 *)p = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) p[e] = (uint16_t)(w[e >> 1] >> (e & 1) * 16);
}

// An accumulator on its way out, by eight warps: warp w has a quarter of the lanes,
// 32 (w & 3) on, and the 16 columns of every second turn.  It reads them in 8 x 8
// blocks, which hold a row's neighbouring columns; turned on their way through shared
// memory as 16-bit values they become a token's neighbouring outputs, 16 bytes a
// thread, 64 a token.  The residual comes in the other way round.  A token's 64 bytes
// stand at 64 times its number there, their four pieces exchanged by half the number,
// so that no access meets a bank twice.  Plain: a warp's rows are its own outputs, and
// no other warp is waited for.  Gated: the rows 64 on are the second sums of a warp
// two on; the two exchange eight columns each, in fp32.  The next columns are on their
// way meanwhile, and what is added to them two turns ahead, from before the sums are
// ready on.  (In fp32 through shared memory, a row a thread: 160 instructions and 1,200
// clocks for 16 columns.)
//
// An exchange is written, the two warps meet, and it is read.  Its place is free again
// when they have met once more, since each has then read what it got: turn after turn a
// place is not the one before's, nor is it from a tile's last turn to the next tile's
// first, which nothing else puts in order (`slot` runs on through all of a warp's tiles).
constexpr int kOutCols = 16;
constexpr int kAhead = 3;    // turns whose residual, or exchange, has a place
static_assert(kAhead >= 2, "a turn's place is not the one before's");
struct OutRoom {             // of a warp
  uint4 out[kOutCols * 4];
  uint4 add[kAhead][kOutCols * 4];  // the residual, or the other warp's sums
};
template <bool GATED, bool F16, class R, class F>
__device__ __forceinline__ void drain(const LinearArgs &a, uint32_t tmem, OutRoom *rooms, int warp, int lane, int64_t t0, int o0,
                                      int &slot, R ready, F all_read) {
  constexpr int kHalves = GATED ? 1 : 2;  // eights of columns that a warp finishes
  constexpr int kTurn = 2 * kOutCols;     // from a warp's columns to its next
  const int four = warp >> 2, quarter = warp & 3;
  const int row0 = o0 + (GATED ? quarter & 1 : quarter) * 32;  // the output of the warp's first row
  const int own = GATED ? quarter >> 1 : 0;                    // its first eight
  const uint32_t at = tmem + ((uint32_t)quarter * 32 << 16);
  OutRoom &room = rooms[warp], &other = rooms[warp ^ 2];
  // in shared memory: this lane's place among the blocks, and its token and piece
  const int bt = lane & 7, bp = (lane >> 3) ^ (bt >> 1 & 3), block = bt * 4 + bp;
  const int mt = lane >> 2, piece = mt * 4 + ((lane & 3) ^ (mt >> 1 & 3));
  // in memory
  int c0 = four * kOutCols;
  const int o = row0 + (lane & 3) * 8, n = a.d_out - o;
  const int64_t first = t0 + c0 + own * 8 + mt;
  int left = n > 0 ? (int)(min(a.n_tok, t0 + a.tokens) - first) : 0;  // of the tile's tokens, from this lane's on
  uint16_t *y = (uint16_t *)a.y + first * a.y_stride + o;
  const uint16_t *rp = (const uint16_t *)a.residual + first * a.r_stride + o;
  const bool adds = !GATED && a.residual;
  float b[2][4] = {};
#pragma unroll
  for (int k = 0; k < (GATED ? 2 : 1); ++k)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int f = row0 + g * 8 + (lane >> 2);
      if (a.bias[k] && f < a.d_out) b[k][g] = value_of<F16>(((const uint16_t *)a.bias[k])[f]);
    }
  uint32_t r[16];
  auto read = [&](int c) {
    tmem_load_blocks(r, at + c);
    tmem_load_blocks(r + 8, at + (16u << 16) + c);
  };
  int ask_left = left, ask_at = slot;  // of the turn whose residual is asked for next
  auto ask = [&] {
#pragma unroll
    for (int h = 0; h < 2; ++h) copy_some(&room.add[ask_at][h * 32 + piece], rp + h * 8 * a.r_stride, h * 8 < ask_left ? n : 0);
    asm volatile("cp.async.commit_group;" ::: "memory");
    rp += kTurn * a.r_stride;
    ask_left -= kTurn;
    ask_at = ask_at + 1 == kAhead ? 0 : ask_at + 1;
  };
  if (adds) {
    __syncwarp();  // the tile before has been read
    for (int k = 0; k + 1 < kAhead; ++k) ask();
  }
  ready();
  if (c0 < a.tokens)
    read(c0);
  else
    all_read();
  for (; c0 < a.tokens; c0 += kTurn, slot = slot + 1 == kAhead ? 0 : slot + 1) {
    __syncwarp();
    if (adds) {
      ask();
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      __syncwarp();
    }
    tmem_wait_load();
    const bool last = c0 + kTurn >= a.tokens;
    if (last) all_read();
    float v[kHalves][4][2], u[4][2];
    if (GATED) {
      float *const to = (float *)room.add[slot], *const from = (float *)other.add[slot];
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t mine = (g >> 1) * 8 + (g & 1) * 2 + k;  // in r, of the first eight columns
          const float p = __uint_as_float(r[mine]), q = __uint_as_float(r[mine + 4]);
          v[0][g][k] = own ? q : p;
          to[(g * 2 + k) * 32 + lane] = own ? p : q;
        }
      asm volatile("bar.sync %0, 64;" ::"r"(1 + four * 2 + (quarter & 1)) : "memory");
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          u[g][k] = from[(g * 2 + k) * 32 + lane];
          if (own) {  // these rows are the second sums
            const float x = v[0][g][k];
            v[0][g][k] = u[g][k];
            u[g][k] = x;
          }
        }
    } else {
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int k = 0; k < 2; ++k) v[h][g][k] = __uint_as_float(r[(g >> 1) * 8 + h * 4 + (g & 1) * 2 + k]);
    }
    if (!last) read(c0 + kTurn);
    if (a.bias[0])
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int k = 0; k < 2; ++k) v[h][g][k] += b[0][g];
    activate(v, a.act);
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      uint32_t w[4];
      if (GATED)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int k = 0; k < 2; ++k) v[h][g][k] *= u[g][k] + b[1][g];
      if (adds) {
        load_turned(w, smem_addr(&room.add[slot][h * 32 + block]));
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int k = 0; k < 2; ++k) v[h][g][k] += value_of<F16>((uint16_t)(w[g] >> k * 16));
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) w[g] = pack_out<F16>(v[h][g][0], v[h][g][1]);
      store_turned(smem_addr(&room.out[h * 32 + block]), w);
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
      if (h * 8 < left) store_some(y + h * 8 * a.y_stride, room.out[h * 32 + piece], n);
    y += kTurn * a.y_stride;
    left -= kTurn;
  }
  // what was asked for past the tile's end (zeros, of no memory) does not come after the next tile's
  if (adds) asm volatile("cp.async.wait_all;" ::: "memory");
}

__device__ __forceinline__ void tma_load2(void *to, const CUtensorMap *map, int x, int y, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_addr(to)),
      "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar))
      : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// All threads of the cluster; what they wrote to shared memory is seen after it.
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of a place in this block's shared memory in another block of the cluster.
__device__ __forceinline__ uint32_t peer_addr(const void *p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
  return r;
}
// n bytes in a row from this block's shared memory to that of another one, counted by a
// barrier there: addresses and n multiples of 16.
__device__ __forceinline__ void send_bytes(uint32_t to, const void *from, uint32_t n, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to),
               "r"(smem_addr(from)), "r"(n), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void store_peer(uint32_t at, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}

__host__ __device__ constexpr uint32_t columns_for(int n) { return n <= 32 ? 32 : n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512; }

// Few tokens: the weights' bytes bound the call.  A CTA forms a tile of 128 rows by
// `tokens` columns, and `split` CTAs of a cluster share its sum, each a stretch of it,
// so that there are CTAs for every SM and, two to an SM, one's beginning and end lie
// in the other's loads.  The parts are joined through the cluster's shared memory, in
// the stretches' order: each CTA takes the columns that are its to finish.
//
// Measured: 16 tokens, gated, 4096 -> 14336 in bf16 37.5 us, 6.3 TB/s (0.92 of the
// measured rate); 96 tokens 6912 -> 5120 with a residual 17.4 us (10.9 of bytes; the 40 row
// tiles in clusters of three are 120 CTAs, so 32 SMs load nothing), one token 5120 -> 3584
// 9.1 us (5.4): the rest is the first loads' latency, the join (1.5 us) and a kernel's
// beginning and end, of which the setup lies beside the kernel before.  1,100 tokens
// 1280 -> 5120 with a residual 15.4 us (7.5 of operations): 280 CTAs come to their way out
// together (4 us by the cut's model), and ask for the residual only then.
constexpr int kSpThreads = 256;

struct SplitSmem {
  uint64_t full[kSpStages], empty[kSpStages], done, joined;
  uint32_t tmem;
  int stop[3];  // see bar_wait
};
// The stages stand first, from a 1,024-byte boundary on, and later a tile's sums in
// their place: a CTA's own and those that it gets, or the way out's rooms.  Then this.
static_assert(kOutRooms == 8 * sizeof(OutRoom), "what a cut counts with");

// The parts of a tile's sums to the CTAs that finish them, and out from there.  The
// columns that CTA r finishes begin at r tokens / split.  A CTA puts its accumulator into
// its own shared memory, a column of 132 floats after the other, and sends each other
// CTA its columns by one bulk copy; what it gets stands behind, by the sender.  (By
// stores of four bytes a lane into the others' shared memory: 2 to 5 us longer for 96
// tokens.)
template <bool GATED, bool F16>
__device__ __forceinline__ void join(const LinearArgs &a, SplitSmem &sm, uint32_t tmem, float *sums, int warp, int lane,
                                     uint32_t rank, int64_t t0, int o0, volatile int *stop) {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // this CTA's stages are free
  auto first = [&](int r) { return a.tokens * r / a.split; };
  const int most = (a.tokens + a.split - 1) / a.split;
  float *const got = sums + a.tokens * kColFloats;
  // Warps 0-3 and 4-7 take turns of 16 columns; a warp reads its quarter of the lanes.
  const int row = (warp & 3) * 32 + lane;
  const uint32_t lane0 = tmem + ((uint32_t)(warp & 3) * 32 << 16);
  for (int c0 = (warp >> 2) * 16; c0 < a.tokens; c0 += 32) {
    uint32_t r[16];
    tmem_load16(r, lane0 + c0);
    tmem_wait_load();
#pragma unroll
    for (int k = 0; k < 16; ++k) sums[(c0 + k) * kColFloats + row] = __uint_as_float(r[k]);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (threadIdx.x < a.split && threadIdx.x != rank) {
    const int to = threadIdx.x, begin = first(to);
    send_bytes(peer_addr(got + (rank < to ? rank : rank - 1) * most * kColFloats, to), sums + begin * kColFloats,
               (uint32_t)((first(to + 1) - begin) * kColFloats * sizeof(float)), peer_addr(&sm.joined, to));
  }
  constexpr int kGroups = tile_outputs<GATED>() / 8;
  const int group = threadIdx.x % kGroups, o = o0 + group * 8;
  float b[2][8];
  load_bias<GATED, F16>(a, o, b);
  const int begin = first(rank), mine = first(rank + 1) - begin;
  constexpr int kStep = kSpThreads / kGroups;
  int c = threadIdx.x / kGroups;
  const int n = a.d_out - o, end = n > 0 ? (int)min((int64_t)mine, a.n_tok - (t0 + begin)) : 0;
  const bool adds = !GATED && a.residual;
  uint4 next = make_uint4(0, 0, 0, 0);  // what is added to the next token's outputs
  auto ask = [&](int at) {
    if (adds && at < end) next = load_some((const uint16_t *)a.residual + (t0 + begin + at) * a.r_stride + o, n);
  };
  ask(c);
  bar_wait(&sm.joined, 0, stop);
  for (; c < end; c += kStep) {
    float v[8] = {}, u[8] = {};
    for (int s = 0; s < a.split; ++s) {
      const float *const at =
          (s == rank ? sums + (begin + c) * kColFloats : got + ((s < rank ? s : s - 1) * most + c) * kColFloats) + group * 8;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 q = *(const float4 *)(at + e);
        v[e] += q.x, v[e + 1] += q.y, v[e + 2] += q.z, v[e + 3] += q.w;
        if (GATED) {
          const float4 w = *(const float4 *)(at + kRows / 2 + e);
          u[e] += w.x, u[e + 1] += w.y, u[e + 2] += w.z, u[e + 3] += w.w;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[0][e];
    activate(v, a.act);
    float add[8];
    unpack8<F16>(next, add);
    ask(c + kStep);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (GATED) v[e] *= u[e] + b[1][e];
      if (adds) v[e] += add[e];
    }
    store_some((uint16_t *)a.y + (t0 + begin + c) * a.y_stride + o,
               make_uint4(pack_out<F16>(v[0], v[1]), pack_out<F16>(v[2], v[3]), pack_out<F16>(v[4], v[5]),
                          pack_out<F16>(v[6], v[7])),
               n);
  }
  __syncwarp();
  cluster_sync();  // what this CTA sent has arrived
}

template <bool GATED, bool F16>
__global__ void __launch_bounds__(kSpThreads)
    k_product(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap map_w,
              const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_x) {
  extern __shared__ unsigned char raw_product[];
  unsigned char *const stage0 = (unsigned char *)((reinterpret_cast<uintptr_t>(raw_product) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage_bytes = kWBytes + a.tokens * kPiece * 2;
  SplitSmem &sm = *reinterpret_cast<SplitSmem *>(stage0 + a.room);
  const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t columns = columns_for(a.tokens);
  if (warp == 0) tmem_alloc(&sm.tmem, columns);
  if (threadIdx.x == 32) {
    map_ahead(&map_w);
    if (GATED) map_ahead(&map_u);
    map_ahead(&map_x);
    sm.stop[0] = sm.stop[1] = sm.stop[2] = 0;
    for (int k = 0; k < a.stages; ++k) {
      bar_init(&sm.full[k], 1);
      bar_init(&sm.empty[k], 1);
    }
    bar_init(&sm.done, 1);
    bar_init(&sm.joined, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  let_next();
  const uint32_t tmem = __shfl_sync(~0u, sm.tmem, 0);
  volatile int *stop = sm.stop;
  const uint32_t rank = blockIdx.x % a.split;
  const int64_t tile = blockIdx.x / a.split;
  const int64_t t0 = tile % a.token_tiles * a.tokens;
  const int o0 = (int)(tile / a.token_tiles) * tile_outputs<GATED>();
  const int from = (int)((int64_t)a.chunks * rank / a.split), to = (int)((int64_t)a.chunks * (rank + 1) / a.split);
  const int n = to - from;
  if (threadIdx.x == 0 && a.split > 1)
    bar_expect(&sm.joined, (uint32_t)((a.split - 1) * (a.tokens * (rank + 1) / a.split - a.tokens * rank / a.split) * kColFloats * 4));
  wait_previous();

  // Both loops are the whole warp's, with one lane that issues: what they count is then
  // the same in all lanes and stays in uniform registers.  (A loop of one lane, with its
  // stage by a division: 540 clocks a turn, whatever it loaded.)
  if (warp == 1) {
    int st = 0, x = from * kPiece;
    uint32_t round = 0;  // of the ring
    for (int i = 0; i < n; ++i, x += kPiece) {
      if (round > 0) bar_wait(&sm.empty[st], (round - 1) & 1, stop);
      if (elect_one()) {
        unsigned char *const at = stage0 + st * stage_bytes;
        bar_expect(&sm.full[st], stage_bytes);
        tma_load2(at, &map_w, x, o0, &sm.full[st]);
        if (GATED) tma_load2(at + kWBytes / 2, &map_u, x, o0, &sm.full[st]);
        tma_load2(at + kWBytes, &map_x, x, (int)t0, &sm.full[st]);
      }
      if (++st == a.stages) st = 0, ++round;
    }
  } else if (warp == 0) {
    const uint32_t idesc = tc_idesc(kRows, a.tokens, F16, false, false);
    const uint32_t base = tc_desc(smem_addr(stage0), 16);
    int st = 0;
    uint32_t phase = 0;
    for (int i = 0; i < n; ++i) {
      bar_wait(&sm.full[st], phase, stop);
      tc_after_sync();
      if (elect_one()) {
        const uint32_t w = base + (st * stage_bytes >> 4), x = w + (kWBytes >> 4);
#pragma unroll
        for (int k = 0; k < kPiece / 16; ++k) tc_mma(tmem, w + k * 2, x + k * 2, idesc, i > 0 || k > 0);
        tc_commit(i + 1 == n ? &sm.done : &sm.empty[st]);
      }
      if (++st == a.stages) st = 0, phase ^= 1;
    }
  }
  __syncwarp();
  bar_wait(&sm.done, 0, stop);
  __syncwarp();
  tc_after_sync();
  // every CTA's products are done: the stages may hold sums
  float *const sums = reinterpret_cast<float *>(stage0);
  if (a.split == 1) {
    __syncthreads();
    int slot = 0;
    drain<GATED, F16>(a, tmem, reinterpret_cast<OutRoom *>(stage0), warp, lane, t0, o0, slot, [] {}, [] {});
  } else {
    join<GATED, F16>(a, sm, tmem, sums, warp, lane, rank, t0, o0, stop);
  }
  tc_before_sync();
  if (threadIdx.x == 0 && *stop) {
    flag(a.status, kStatusTimeout);
    for (int k = 0; k < 1000; ++k) __nanosleep(1000);  // what was issued may still be at work on shared memory
  }
  __syncthreads();
  if (warp == 0) tmem_free(tmem, columns);
}

// Many tokens: the products bound the call.  A pair of CTAs on neighbouring SMs forms
// a tile of 256 rows by `tokens` columns with instructions that take both SMs'
// operands: each CTA loads its 128 weight rows and half of the tokens, so that a term
// of the sum costs half the shared-memory reads of two CTAs on their own.  The pairs
// stay and take tiles in turn; two accumulators let a tile's products run while the
// one before is on its way out.
//
// Measured: 8,192 tokens, 4096 -> 6144 in bf16, 212 us in a burst, 1,945 TFLOP/s (1.01 of the
// measured rate: a library's product of these sizes takes 212), 239 us kept up under the
// power limit (238); 4,001 tokens, gated, 5120 -> 6912 in fp16 315 to 331 us, 1,710 to 1,800
// TFLOP/s, kept up 357; 333 tokens 43 to 45 us: 108 tiles on 76 pairs are two rounds, and a
// tile's way out (4 us) stands behind the last.
//   warps 0-7  a tile's way out (drain);
//   warp 8     loads; warp 9 of the first CTA issues the products of both.
constexpr int kPaThreads = 320;

struct PairSmem {
  unsigned char stage[kPaRoom];
  OutRoom out[8];
  uint64_t full[kPaStages], empty[kPaStages], sums_full[2], sums_empty[2];
  uint32_t tmem;
  int stop[3];  // see bar_wait
};

// Loads into this CTA's shared memory whose bytes are counted by a barrier of the
// pair's first CTA.
__device__ __forceinline__ void tma_load2_pair(void *to, const CUtensorMap *map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_addr(to)),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t *to, int columns) {  // one whole warp of each CTA
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t at, int columns) {  // one whole warp of each CTA
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
// One arrival at the barrier at this place in both CTAs when all that this thread has
// issued is done.
__device__ __forceinline__ void tc_commit_pair(uint64_t *bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)),
      "h"((uint16_t)3)
      : "memory");
}
__device__ __forceinline__ void tc_mma_pair(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n.reg .pred p;\n.reg .b64 da, db;\nsetp.ne.b32 p, %4, 0;\nmov.b64 da, {%1, %5};\nmov.b64 db, {%2, %5};\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kDescHigh)
      : "memory");
}
// An arrival that says no more than that tensor memory has been read (the loads were
// waited for); one that released the thread's stores would wait for them.
__device__ __forceinline__ void bar_arrive_peer(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// First outputs and tokens of a tile: bands of twelve row tiles, row tile after row tile
// and then token tile after token tile, so that the tiles at work at a time share their
// operands in L2 (us kept up of 8,192 tokens, 4096 -> 6144, whose 24 row tiles they divide:
// bands of 4 248, 8 245, 12 241, 24 246; other numbers of row tiles, and the gated form,
// were not measured).
__device__ __forceinline__ void pair_tile(const LinearArgs &a, int64_t tile, int64_t *row_tile, int64_t *token_tile) {
  constexpr int64_t kBand = 12;
  const int64_t rows = quotient(a.tiles, a.token_tiles), of_band = kBand * a.token_tiles;
  const int64_t band = quotient(tile, of_band), in = tile - band * of_band;
  const int64_t wide = min(kBand, rows - band * kBand), t = quotient(in, wide);
  *token_tile = t;
  *row_tile = band * kBand + in - t * wide;
}

template <bool GATED, bool F16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPaThreads, 1)
    k_product_pair(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_x) {
  extern __shared__ unsigned char raw_pair[];
  PairSmem &sm = *reinterpret_cast<PairSmem *>((reinterpret_cast<uintptr_t>(raw_pair) + 1023) & ~(uintptr_t)1023);
  const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  if (warp == 9) tmem_alloc_pair(&sm.tmem, 512);
  if (threadIdx.x == 8 * 32) {
    map_ahead(&map_w);
    if (GATED) map_ahead(&map_u);
    map_ahead(&map_x);
    sm.stop[0] = sm.stop[1] = sm.stop[2] = 0;
    for (int k = 0; k < a.stages; ++k) {
      bar_init(&sm.full[k], 1);
      bar_init(&sm.empty[k], 1);
    }
    for (int k = 0; k < 2; ++k) {
      bar_init(&sm.sums_full[k], 1);
      bar_init(&sm.sums_empty[k], 16);  // the eight warps of both CTAs
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  tc_before_sync();
  __syncthreads();
  cluster_sync();
  tc_after_sync();
  let_next();
  wait_previous();
  const uint32_t tmem = __shfl_sync(~0u, sm.tmem, 0);
  volatile int *stop = sm.stop;
  const int64_t pairs = gridDim.x / 2, first = blockIdx.x / 2;
  const int half = a.tokens / 2;
  const uint32_t stage_bytes = kWBytes + half * kPiece * 2;
  constexpr int kOut = tile_outputs<GATED>();
  constexpr uint32_t kCols = 256;  // of an accumulator

  if (warp == 8) {
    const uint32_t bytes = 2 * stage_bytes;
    int st = 0;
    uint32_t round = 0;  // of the ring
    for (int64_t tile = first; tile < a.tiles; tile += pairs) {
      int64_t row_tile, token_tile;
      pair_tile(a, tile, &row_tile, &token_tile);
      const int o = (int)(row_tile * 2 + rank) * kOut, t = (int)(token_tile * a.tokens) + (int)rank * half;
      for (int i = 0; i < a.chunks; ++i) {
        if (round > 0) bar_wait(&sm.empty[st], (round - 1) & 1, stop);
        if (elect_one()) {
          unsigned char *const at = sm.stage + st * stage_bytes;
          const uint32_t bar = peer_addr(&sm.full[st], 0);
          if (rank == 0) bar_expect(&sm.full[st], bytes);
          tma_load2_pair(at, &map_w, i * kPiece, o, bar);
          if (GATED) tma_load2_pair(at + kWBytes / 2, &map_u, i * kPiece, o, bar);
          tma_load2_pair(at + kWBytes, &map_x, i * kPiece, t, bar);
        }
        if (++st == a.stages) st = 0, ++round;
      }
      if (__any_sync(~0u, *stop)) break;
    }
    // the products have read, and their arrivals reached, every stage before the CTA ends
    for (int k = 0; k < a.stages; ++k)
      if (round > 0 || k < st) bar_wait(&sm.empty[k], (k < st ? round : round - 1) & 1, stop);
  } else if (warp == 9 && rank == 0) {
    const uint32_t idesc = tc_idesc(256, a.tokens, F16, false, false), base = tc_desc(smem_addr(sm.stage), 16);
    int st = 0;
    uint32_t phase = 0;
    int n = 0;
    for (int64_t tile = first; tile < a.tiles; tile += pairs, ++n) {
      if (n >= 2) bar_wait(&sm.sums_empty[n & 1], ((n >> 1) - 1) & 1, stop);
      tc_after_sync();
      const uint32_t d = tmem + (n & 1) * kCols;
      for (int i = 0; i < a.chunks; ++i) {
        bar_wait(&sm.full[st], phase, stop);
        tc_after_sync();
        if (elect_one()) {
          const uint32_t w = base + (st * stage_bytes >> 4), x = w + (kWBytes >> 4);
#pragma unroll
          for (int k = 0; k < kPiece / 16; ++k) tc_mma_pair(d, w + k * 2, x + k * 2, idesc, i > 0 || k > 0);
          tc_commit_pair(&sm.empty[st]);
          if (i + 1 == a.chunks) tc_commit_pair(&sm.sums_full[n & 1]);
        }
        if (++st == a.stages) st = 0, phase ^= 1;
      }
      if (__any_sync(~0u, *stop)) break;
    }
  } else if (warp < 8) {
    int n = 0, slot = 0;
    for (int64_t tile = first; tile < a.tiles; tile += pairs, ++n) {
      int64_t row_tile, token_tile;
      pair_tile(a, tile, &row_tile, &token_tile);
      auto ready = [&] {
        bar_wait(&sm.sums_full[n & 1], (n >> 1) & 1, stop);
        __syncwarp();
        tc_after_sync();
      };
      auto all_read = [&] {
        tc_before_sync();
        __syncwarp();
        if (lane == 0) bar_arrive_peer(peer_addr(&sm.sums_empty[n & 1], 0));
      };
      drain<GATED, F16>(a, tmem + (n & 1) * kCols, sm.out, warp, lane, token_tile * a.tokens,
                        (int)(row_tile * 2 + rank) * kOut, slot, ready, all_read);
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  if (threadIdx.x == 0 && *stop) {
    flag(a.status, kStatusTimeout);
    for (int k = 0; k < 1000; ++k) __nanosleep(1000);  // what was issued may still be at work on shared memory
  }
  __syncthreads();
  cluster_sync();  // the pair ends together
  if (warp == 9) tmem_free_pair(tmem, 512);
}

}  // namespace lv
