// Host side of the attention calls: argument checks and launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "llmvisor.h"
#include "lv_attend.cuh"
#include "lv_chunk.cuh"
#include "lv_decode.cuh"
#include "lv_kv.h"
#include "lv_kv_plan.cuh"
#include "lv_kv_store.cuh"
#include "lv_prompt.cuh"

using namespace lv;

namespace {

#define LV_CUDA(call)                          \
  do {                                         \
    if ((call) != cudaSuccess) return LV_ECUDA; \
  } while (0)

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int log2_of(int64_t x) { return 63 - __builtin_clzll((unsigned long long)x); }

// The context's scratch, at least `bytes`.  It grows by doubling and what it
// outgrows is kept to the context's end: a call that was captured into a graph
// works there at every replay.
lv_status scratch_for(KvHost *kv, size_t bytes) {
  if (bytes <= kv->cap) return LV_OK;
  const size_t cap = std::max(std::max(bytes, 2 * kv->cap), (size_t)1 << 20);
  if (kv->n_outgrown == 64) return LV_ENOMEM;
  void *p = nullptr;
  if (cudaMalloc(&p, cap) != cudaSuccess) {
    cudaGetLastError();
    return LV_ENOMEM;
  }
  if (kv->scratch) kv->outgrown[kv->n_outgrown++] = kv->scratch;
  kv->scratch = static_cast<unsigned char *>(p);
  kv->cap = cap;
  return LV_OK;
}

// The context's two counters for work that kernels hand out.
lv_status counters_for(KvHost *kv) {
  if (!kv->counter) {
    void *c = nullptr;
    if (cudaMalloc(&c, 2 * sizeof(unsigned long long)) != cudaSuccess) {
      cudaGetLastError();
      return LV_ENOMEM;
    }
    if (cudaMemset(c, 0, 2 * sizeof(unsigned long long)) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
      cudaFree(c);
      return LV_ECUDA;
    }
    kv->counter = static_cast<unsigned long long *>(c);
  }
  return LV_OK;
}

bool cache_ok(const lv_kv_cache *c) {
  if (!c || c->n_blocks < 0 || c->n_blocks > (1ll << 31) || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return false;
  if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->n_blocks == 0) return true;
  return c->k && c->v && c->k_scale && c->v_scale && aligned(c->k, 16) && aligned(c->v, 16) &&
         aligned(c->k_scale, 4) && aligned(c->v_scale, 4);
}

// An array of n_tok tokens of `heads` heads.
bool rows_ok(const void *p, int64_t stride, int64_t n_tok, int64_t heads, int64_t dim) {
  return n_tok == 0 || (p && aligned(p, 16) && stride % 8 == 0 && stride >= heads * dim && stride <= (1ll << 40));
}

bool heads_ok(int32_t dtype, int32_t hq, int32_t hkv) {
  return (dtype == LV_BF16 || dtype == LV_F16) && hkv >= 1 && hkv <= 1024 && hq >= hkv && hq % hkv == 0 &&
         hq / hkv <= LV_MAX_GROUP;
}

constexpr int64_t kMostTokens = 1ll << 30;

// A kernel's shared-memory limit, once for a context; `kind` numbers the kernels.
template <class K>
lv_status limit_smem(KvHost *kv, K kernel, int kind, size_t bytes) {
  if (kv->configured >> kind & 1) return LV_OK;
  LV_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  kv->configured |= 1u << kind;
  return LV_OK;
}

// Launches a kernel that may start while the one before it in the stream runs
// (it calls wait_previous itself).
template <class... P, class... A>
lv_status launch_after(void (*kernel)(P...), dim3 grid, unsigned block, size_t smem, cudaStream_t stream, A... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LV_CUDA(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
  return LV_OK;
}

template <int D, bool F16, int NT>
lv_status run_decode(KvHost *kv, const AttendArgs &a, cudaStream_t stream) {
  DecodeArgs d{};
  d.a = a;
  d.nt = NT;
  d.most_rows = kDecRows;
  const int64_t ctas = (int64_t)kv->sms * (NT == 1 ? kDecCtas1 : kDecCtas2);
  d.warps = ctas * kDecWarps;
  const int G = a.hq / a.hkv, tiles = (G + 8 * NT - 1) / (8 * NT);
  const int64_t segments = a.n_req * a.hkv * tiles;
  // scratch: running sums, the parts
  const size_t o_part = (8 * ((size_t)a.n_req + 1) + 255) & ~(size_t)255;
  const size_t slots = 2 * (size_t)d.warps * 8 * NT;
  const lv_status st = scratch_for(kv, o_part + slots * (D + 2) * sizeof(float));
  if (st != LV_OK) return st;
  d.prefix = reinterpret_cast<int64_t *>(kv->scratch);
  d.part = reinterpret_cast<float *>(kv->scratch + o_part);
  d.part_ml = d.part + slots * D;
  d.given = a.n_req > kScan;
  if (d.given) {
    k_attend_prefix<<<1, kScan, 0, stream>>>(d);
    LV_CUDA(cudaGetLastError());
  }
  k_attend_decode<D, F16, NT><<<(unsigned)ctas, kDecWarps * 32, 0, stream>>>(d);
  LV_CUDA(cudaGetLastError());
  // Warps of a row that is joined, by the parts there are in a segment (us a call, 16
  // decodes of 128 segments, about 19 parts each, and 3 long ones of 6, about 400):
  // one 43.4, four 41.7 and 56.1, eight 43.8 and 52.0, sixteen 51.6 and 51.3
  const int64_t y = (int64_t)a.hkv * tiles * 8 * NT, y1 = (int64_t)a.hkv * tiles * NT;
  const unsigned n = (unsigned)a.n_req;
  if (segments * 64 < d.warps)
    return launch_after(k_attend_join<D, F16, 16>, dim3(n, (unsigned)std::min<int64_t>(y, 4096)), 16 * 32, 0, stream, d);
  if (segments * 8 < d.warps)
    return launch_after(k_attend_join<D, F16, 4>, dim3(n, (unsigned)std::min<int64_t>(y, 4096)), 4 * 32, 0, stream, d);
  return launch_after(k_attend_join<D, F16, 1>, dim3(n, (unsigned)std::min<int64_t>(y1, 4096)), kJoinWarps * 32, 0,
                      stream, d);
}

template <int D, bool F16>
lv_status run_chunk(KvHost *kv, const AttendArgs &a, cudaStream_t stream) {
  ChunkArgs c{};
  c.a = a;
  if (c.a.scale == 0.f) c.a.scale = 1e-37f;  // a masked score is -infinity: its product with the scale must be too
  const int G = a.hq / a.hkv, ctas = kv->sms;
  c.tile = 128 / G;
  c.least_rows = kDecRows + 1;
  const size_t o_part = (8 * ((size_t)a.n_req + 1) + 255) & ~(size_t)255;
  const size_t slots = 2 * (size_t)ctas * 256;
  lv_status st = scratch_for(kv, o_part + slots * (D + 2) * sizeof(float));
  if (st != LV_OK) return st;
  c.prefix = reinterpret_cast<int64_t *>(kv->scratch);
  c.part = reinterpret_cast<float *>(kv->scratch + o_part);
  c.part_ml = c.part + slots * D;
  c.given = a.n_req > kScan;
  if (c.given) {
    k_chunk_prefix<<<1, kScan, 0, stream>>>(c);
    LV_CUDA(cudaGetLastError());
  }
  constexpr size_t smem = sizeof(ChunkSmem<D>) + 1024;
  static_assert(smem <= 227 << 10, "an SM's shared memory");
  st = limit_smem(kv, k_chunk<D, F16>, (D == 128 ? 0 : 2) + (F16 ? 1 : 0), smem);
  if (st != LV_OK) return st;
  k_chunk<D, F16><<<(unsigned)ctas, kChThreads, smem, stream>>>(c);
  LV_CUDA(cudaGetLastError());
  const int64_t y = (a.n_tok / (2 * c.tile) + 1) * a.hkv * 4;  // quarters of the items of the longest request there can be
  return launch_after(k_chunk_join<D, F16>, dim3((unsigned)a.n_req, (unsigned)std::min<int64_t>(y, 2048)), 256, 0, stream,
                      c, ctas);
}

// Requests of up to kDecRows rows (new tokens times query heads of a key/value
// head) by k_attend_decode, others by k_chunk.  Where every request has one token
// all are of one kind; else the device's offsets say, and both go over the
// requests, each taking its own.
template <int D, bool F16>
lv_status run_cached(KvHost *kv, const AttendArgs &a, cudaStream_t stream) {
  const int64_t G = a.hq / a.hkv, most = (a.offsets ? a.n_tok : 1) * G;  // rows of a request, at most
  if (G <= kDecRows) {
    const lv_status st = !a.offsets && G <= 8 ? run_decode<D, F16, 1>(kv, a, stream) : run_decode<D, F16, 2>(kv, a, stream);
    if (st != LV_OK) return st;
  }
  return most > kDecRows ? run_chunk<D, F16>(kv, a, stream) : LV_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder of tensor maps, through the runtime (no link against the
// driver's library); null where it is missing.
EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    const cudaError_t rc = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
    return rc == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(p) : nullptr;
  }();
  return f;
}

// The map of a [token][head][element] array whose boxes are `tokens` tokens of
// `heads` heads and 64 elements.
lv_status map_rows(CUtensorMap *map, const void *at, int32_t dtype, int64_t n_tok, int64_t n_heads, int64_t dim,
                   int64_t stride, int tokens, int heads) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return LV_ECUDA;
  const cuuint64_t size[3] = {(cuuint64_t)dim, (cuuint64_t)n_heads, (cuuint64_t)n_tok};
  const cuuint64_t step[2] = {(cuuint64_t)dim * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)tokens}, one[3] = {1, 1, 1};
  const CUresult rc =
      encode(map, dtype == LV_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
             const_cast<void *>(at), size, step, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return rc == CUDA_SUCCESS ? LV_OK : LV_ECUDA;
}

template <int D, bool F16>
lv_status run_prompt(KvHost *kv, const AttendArgs &a, cudaStream_t stream) {
  PromptArgs p{};
  p.a = a;
  const int G = a.hq / a.hkv;
  p.tile = 128 / G;
  p.wide = aligned(a.o, 32);
  const int32_t dtype = F16 ? LV_F16 : LV_BF16;
  CUtensorMap mq, mk, mv;
  lv_status st = map_rows(&mq, a.q, dtype, a.n_tok, a.hq, D, a.q_stride, p.tile, G);
  if (st == LV_OK) st = map_rows(&mk, a.k, dtype, a.n_tok, a.hkv, D, a.k_stride, kPrBlock, 1);
  if (st == LV_OK) st = map_rows(&mv, a.v, dtype, a.n_tok, a.hkv, D, a.v_stride, kPrBlock, 1);
  if (st != LV_OK) return st;
  st = counters_for(kv);
  if (st != LV_OK) return st;
  p.counter = kv->counter;
  p.given = a.n_req > kScan;
  if (p.given) {
    st = scratch_for(kv, 8 * ((size_t)a.n_req + 1));
    if (st != LV_OK) return st;
    p.prefix = reinterpret_cast<int64_t *>(kv->scratch);
    k_prompt_prefix<<<1, kScan, 0, stream>>>(p);
    LV_CUDA(cudaGetLastError());
  }
  constexpr size_t smem = sizeof(PromptSmem<D>) + 1024;
  static_assert(smem <= 227 << 10, "an SM's shared memory");
  st = limit_smem(kv, k_prompt<D, F16>, 4 + (D == 128 ? 0 : 2) + (F16 ? 1 : 0), smem);
  if (st != LV_OK) return st;
  // a CTA an SM; no more than there can be items
  const int64_t items = (a.n_tok / (2 * p.tile) + std::min(a.n_req, a.n_tok)) * a.hkv;
  const unsigned grid = (unsigned)std::min<int64_t>(items, kv->sms);
  k_prompt<D, F16><<<grid, kPrThreads, smem, stream>>>(p, mq, mk, mv);
  LV_CUDA(cudaGetLastError());
  return LV_OK;
}

}  // namespace

extern "C" {

lv_status lv_kv_plan(lv_ctx *ctx, const int32_t *p, const int32_t *c, int64_t n_req, int32_t block_tokens,
                     const int32_t *free_blocks, int64_t n_free, int32_t *table, int64_t table_width,
                     int64_t *token_offsets, int64_t *slots, int64_t n_slots, int64_t *counts, void *stream_) {
  if (!ctx || n_req < 0 || n_req > (1ll << 24) || n_free < 0 || n_slots < 0 || table_width < 0 ||
      table_width > (1ll << 31))
    return LV_EINVAL;
  if (block_tokens < 1 || block_tokens > (1 << 16) || (block_tokens & (block_tokens - 1))) return LV_EINVAL;
  if (!token_offsets || !counts || (n_req > 0 && (!p || !c)) || (n_free > 0 && !free_blocks) ||
      (n_slots > 0 && !slots) || (n_req > 0 && table_width > 0 && !table))
    return LV_EINVAL;
  if (!aligned(p, 4) || !aligned(c, 4) || !aligned(free_blocks, 4) || !aligned(table, 4) ||
      !aligned(token_offsets, 8) || !aligned(slots, 8) || !aligned(counts, 8))
    return LV_EINVAL;
  cudaStream_t stream = (cudaStream_t)stream_;
  KvHost *kv = kv_host(ctx);
  PlanArgs a{};
  a.p = p;
  a.c = c;
  a.n_req = n_req;
  a.log_b = log2_of(block_tokens);
  a.free = free_blocks;
  a.n_free = n_free;
  a.table = table;
  a.width = table_width;
  a.offsets = token_offsets;
  a.slots = slots;
  a.n_slots = n_slots;
  a.counts = counts;
  a.status = kv->d_status;
  const int64_t tiles = std::max<int64_t>(1, (n_req + kPlanTile - 1) / kPlanTile);
  if (tiles > 1) {
    const lv_status st = scratch_for(kv, 16 * (size_t)tiles);
    if (st != LV_OK) return st;
    a.sums = reinterpret_cast<int64_t *>(kv->scratch);
    k_plan_sums<<<(unsigned)tiles, kPlanThreads, 0, stream>>>(a);
    LV_CUDA(cudaGetLastError());
  }
  // CTAs of a tile: one for each 2,048 slots, up to two an SM in all, which is what fits
  const int64_t per = (std::max(n_slots, n_req) / tiles + 2047) / 2048;
  const int64_t slices = std::max<int64_t>(1, std::min<int64_t>(per, 2 * kv->sms / std::min<int64_t>(tiles, kv->sms)));
  static_assert(sizeof(PlanSmem) <= 48 << 10, "static limit");
  const dim3 grid((unsigned)slices, (unsigned)tiles);
  if (tiles > 1) return launch_after(k_plan, grid, kPlanThreads, sizeof(PlanSmem), stream, a);
  k_plan<<<grid, kPlanThreads, sizeof(PlanSmem), stream>>>(a);
  LV_CUDA(cudaGetLastError());
  return LV_OK;
}

lv_status lv_kv_store(lv_ctx *ctx, const lv_kv_cache *cache, int32_t dtype, const void *k, int64_t k_stride,
                      const void *v, int64_t v_stride, const int64_t *slots, int64_t n_tok, void *stream_) {
  if (!ctx || !cache_ok(cache) || n_tok < 0 || n_tok > kMostTokens || (dtype != LV_BF16 && dtype != LV_F16))
    return LV_EINVAL;
  const int d = cache->head_dim, heads = cache->n_kv_heads;
  if (!rows_ok(k, k_stride, n_tok, heads, d) || !rows_ok(v, v_stride, n_tok, heads, d)) return LV_EINVAL;
  if (n_tok == 0) return LV_OK;
  if (!slots || !aligned(slots, 8)) return LV_EINVAL;
  cudaStream_t stream = (cudaStream_t)stream_;
  KvHost *kv = kv_host(ctx);
  StoreArgs a{};
  a.x[0] = k, a.x[1] = v;
  a.stride[0] = k_stride, a.stride[1] = v_stride;
  a.code[0] = cache->k, a.code[1] = cache->v;
  a.scale[0] = cache->k_scale, a.scale[1] = cache->v_scale;
  a.slots = slots;
  a.n_tok = n_tok;
  a.n_blocks = cache->n_blocks;
  a.log_b = log2_of(cache->block_tokens);
  a.heads = heads;
  a.status = kv->d_status;
  int window = 1;  // four CTAs an SM, where there are tokens for them
  while (window < kStoreWindow && n_tok / (2 * window) >= 4 * kv->sms) window *= 2;
  const unsigned grid = (unsigned)((n_tok + window - 1) / window);
  if (d == 128 && dtype == LV_F16) k_kv_store<128, true><<<grid, kStoreWarps * 32, 0, stream>>>(a, window);
  if (d == 128 && dtype == LV_BF16) k_kv_store<128, false><<<grid, kStoreWarps * 32, 0, stream>>>(a, window);
  if (d == 64 && dtype == LV_F16) k_kv_store<64, true><<<grid, kStoreWarps * 32, 0, stream>>>(a, window);
  if (d == 64 && dtype == LV_BF16) k_kv_store<64, false><<<grid, kStoreWarps * 32, 0, stream>>>(a, window);
  LV_CUDA(cudaGetLastError());
  return LV_OK;
}

lv_status lv_kv_attend(lv_ctx *ctx, const lv_kv_cache *cache, int32_t dtype, int32_t n_q_heads, const void *q,
                       int64_t q_stride, int64_t n_tok, const int64_t *token_offsets, const int32_t *c, int64_t n_req,
                       const int32_t *table, int64_t table_width, float scale, void *o, float *lse, void *stream_) {
  if (!ctx || !cache_ok(cache) || !heads_ok(dtype, n_q_heads, cache->n_kv_heads)) return LV_EINVAL;
  if (n_tok < 0 || n_tok > kMostTokens || n_req < 0 || n_req > (1ll << 24) || table_width < 0 ||
      table_width > (1ll << 31) || !std::isfinite(scale))
    return LV_EINVAL;
  if (!token_offsets && n_tok != n_req) return LV_EINVAL;
  if (!rows_ok(q, q_stride, n_tok, n_q_heads, cache->head_dim)) return LV_EINVAL;
  if (n_tok == 0 || n_req == 0) return LV_OK;
  if (!o || !aligned(o, 16) || !aligned(lse, 4) || !c || !aligned(c, 4) || !aligned(token_offsets, 8) ||
      (table_width > 0 && !table) || !aligned(table, 4))
    return LV_EINVAL;
  AttendArgs a{};
  a.cache = {cache->k, cache->v, cache->k_scale, cache->v_scale, cache->n_blocks, log2_of(cache->block_tokens),
             cache->n_kv_heads};
  a.q = q;
  a.q_stride = q_stride;
  a.n_tok = n_tok;
  a.offsets = token_offsets;
  a.c = c;
  a.n_req = n_req;
  a.table = table;
  a.width = table_width;
  a.hq = n_q_heads;
  a.hkv = cache->n_kv_heads;
  a.scale = scale * 1.4426950408889634f;
  a.o = o;
  a.lse = lse;
  KvHost *kv = kv_host(ctx);
  a.status = kv->d_status;
  cudaStream_t stream = (cudaStream_t)stream_;
  if (cache->head_dim == 128)
    return dtype == LV_F16 ? run_cached<128, true>(kv, a, stream) : run_cached<128, false>(kv, a, stream);
  return dtype == LV_F16 ? run_cached<64, true>(kv, a, stream) : run_cached<64, false>(kv, a, stream);
}

lv_status lv_prompt_attend(lv_ctx *ctx, int32_t dtype, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                           const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                           int64_t v_stride, int64_t n_tok, const int64_t *offsets, int64_t n_seq, float scale,
                           void *o, float *lse, void *stream_) {
  if (!ctx || !heads_ok(dtype, n_q_heads, n_kv_heads) || (head_dim != 64 && head_dim != 128)) return LV_EINVAL;
  if (n_tok < 0 || n_tok > kMostTokens || n_seq < 0 || n_seq > (1ll << 24) || !std::isfinite(scale)) return LV_EINVAL;
  if (!rows_ok(q, q_stride, n_tok, n_q_heads, head_dim) || !rows_ok(k, k_stride, n_tok, n_kv_heads, head_dim) ||
      !rows_ok(v, v_stride, n_tok, n_kv_heads, head_dim))
    return LV_EINVAL;
  if (n_tok == 0 || n_seq == 0) return LV_OK;
  if (!o || !aligned(o, 16) || !aligned(lse, 4) || !offsets || !aligned(offsets, 8)) return LV_EINVAL;
  AttendArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.n_tok = n_tok;
  a.offsets = offsets;
  a.n_req = n_seq;
  a.hq = n_q_heads;
  a.hkv = n_kv_heads;
  a.scale = scale * 1.4426950408889634f;
  a.o = o;
  a.lse = lse;
  KvHost *kv = kv_host(ctx);
  a.status = kv->d_status;
  if (a.scale == 0.f) a.scale = 1e-37f;  // a masked score is -infinity: its product with the scale must be too
  cudaStream_t stream = (cudaStream_t)stream_;
  if (head_dim == 128)
    return dtype == LV_F16 ? run_prompt<128, true>(kv, a, stream) : run_prompt<128, false>(kv, a, stream);
  return dtype == LV_F16 ? run_prompt<64, true>(kv, a, stream) : run_prompt<64, false>(kv, a, stream);
}

}  // extern "C"
