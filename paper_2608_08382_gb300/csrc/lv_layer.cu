// Host side of a step's work for each token: argument checks and launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "llmvisor.h"
#include "lv_kv.h"
#include "lv_linear.cuh"
#include "lv_logprobs.cuh"
#include "lv_rotate.cuh"

using namespace lv;

namespace {

#define LV_CUDA(call)                          \
  do {                                         \
    if ((call) != cudaSuccess) return LV_ECUDA; \
  } while (0)

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMostTokens = 1ll << 30, kMostStride = 1ll << 38;
constexpr int kMostWidth = 1 << 24;

// n rows of `width` 16-bit elements that begin at 16-byte boundaries.
bool rows_ok(const void *p, int64_t stride, int64_t n, int64_t width) {
  return n == 0 || (p && aligned(p, 16) && stride % 8 == 0 && stride >= width && stride <= kMostStride);
}

bool is16(int32_t dtype) { return dtype == LV_BF16 || dtype == LV_F16; }

// The caller's arrays of a product.
struct Operands {
  const void *x, *w[2];
  int64_t x_stride, w_stride;
  int d_in;
};

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

// The map of an array of n rows of `width` elements whose boxes are `rows` rows of 64 elements.
lv_status map_matrix(CUtensorMap *map, const void *at, int32_t dtype, int64_t n, int64_t width, int64_t stride, int rows) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return LV_ECUDA;
  const cuuint64_t size[2] = {(cuuint64_t)width, (cuuint64_t)n}, step[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {kPiece, (cuuint32_t)rows}, one[2] = {1, 1};
  const CUresult rc =
      encode(map, dtype == LV_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
             const_cast<void *>(at), size, step, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return rc == CUDA_SUCCESS ? LV_OK : LV_ECUDA;
}

// Kernels' shared-memory limits, once for a context, at the most that a block can
// have; `kind` numbers the kernels (the attention calls' are below 8).
constexpr int kMostSmem = 227 << 10;
template <class K>
lv_status limit_smem(KvHost *kv, K kernel, int kind) {
  if (kv->configured >> kind & 1) return LV_OK;
  LV_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
  kv->configured |= 1u << kind;
  return LV_OK;
}

// Launches a kernel that may start while the one before it in the stream still runs
// (it calls wait_previous itself, when its setup is done); `cluster` CTAs in a cluster,
// 0 where the kernel says it.
template <class... P, class... A>
lv_status launch_after(void (*kernel)(P...), int64_t grid, unsigned block, size_t smem, int cluster, cudaStream_t stream,
                       const A &...args) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cluster ? 2 : 1;
  LV_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
  return LV_OK;
}

// Clusters of each size that the device holds at a time, a CTA an SM (GB300: 152, 76, 46,
// 36, 28, 23, 15, 15: its groups of SMs hold only whole ones).  Asked for once a device.
struct Clusters {
  std::atomic<bool> known{false};
  std::atomic<int> most[kSpSplit + 1] = {};
};
lv_status clusters_of(const Clusters **out) {
  constexpr int kDevices = 64;
  static Clusters all[kDevices];
  int dev = 0;
  LV_CUDA(cudaGetDevice(&dev));
  if (dev >= kDevices) return LV_EINVAL;
  Clusters &c = all[dev];
  if (!c.known.load(std::memory_order_acquire)) {
    // a kernel that takes more than half of an SM's shared memory
    LV_CUDA(cudaFuncSetAttribute(k_product_pair<false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
    LV_CUDA(cudaFuncSetAttribute(k_product<false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
    for (int n = 1; n <= kSpSplit; ++n) {
      cudaLaunchAttribute attr{};
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = n;
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3(1024 * n);
      cfg.blockDim = dim3(kSpThreads);
      cfg.dynamicSmemBytes = 128 << 10;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      int most = 0;
      LV_CUDA(cudaOccupancyMaxActiveClusters(&most, k_product<false, false>, &cfg));
      c.most[n].store(std::max(most, 1), std::memory_order_relaxed);
    }
    c.known.store(true, std::memory_order_release);
  }
  *out = &c;
  return LV_OK;
}

template <bool GATED, bool F16>
lv_status run_linear(KvHost *kv, LinearArgs &a, const Operands &m, cudaStream_t stream) {
  const int32_t dtype = F16 ? LV_F16 : LV_BF16;
  const int64_t outputs = tile_outputs<GATED>(), row_tiles = (a.d_out + outputs - 1) / outputs;
  a.chunks = (m.d_in + kPiece - 1) / kPiece;
  const Clusters *hold;
  lv_status st = clusters_of(&hold);
  if (st != LV_OK) return st;
  const Shape shape = choose([&](int n) { return (int64_t)hold->most[n].load(std::memory_order_relaxed); }, a.n_tok, row_tiles,
                             a.chunks);
  a.tokens = shape.tokens;
  a.split = shape.split;
  a.token_tiles = (a.n_tok + a.tokens - 1) / a.tokens;
  a.tiles = (shape.pair ? (row_tiles + 1) / 2 : row_tiles) * a.token_tiles;
  CUtensorMap mw, mu, mx;
  st = map_matrix(&mw, m.w[0], dtype, a.d_out, m.d_in, m.w_stride, (int)outputs);
  if (st == LV_OK) st = map_matrix(&mx, m.x, dtype, a.n_tok, m.d_in, m.x_stride, shape.pair ? a.tokens / 2 : a.tokens);
  if (st == LV_OK && GATED) st = map_matrix(&mu, m.w[1], dtype, a.d_out, m.d_in, m.w_stride, (int)outputs);
  if (st != LV_OK) return st;
  if (!GATED) mu = mw;
  const int kind = 8 + (GATED ? 2 : 0) + (F16 ? 1 : 0);
  if (shape.pair) {
    constexpr size_t smem = sizeof(PairSmem) + 1024;
    static_assert(smem <= kMostSmem, "an SM's shared memory");
    st = limit_smem(kv, k_product_pair<GATED, F16>, kind + 4);
    if (st != LV_OK) return st;
    a.stages = pair_stages(a.tokens);
    const int64_t grid = 2 * std::min<int64_t>(a.tiles, hold->most[2].load(std::memory_order_relaxed));
    return launch_after(k_product_pair<GATED, F16>, grid, kPaThreads, smem, 0, stream, a, mw, mu, mx);
  }
  st = limit_smem(kv, k_product<GATED, F16>, kind);
  if (st != LV_OK) return st;
  const bool alone = a.tiles <= hold->most[a.split].load(std::memory_order_relaxed);
  a.stages = split_stages(a.tokens, alone);
  a.room = (int)((std::max(a.stages * split_stage(a.tokens), split_sums(a.tokens, a.split)) + 15) / 16 * 16);
  return launch_after(k_product<GATED, F16>, a.tiles * a.split, kSpThreads, 1024 + a.room + sizeof(SplitSmem), a.split, stream,
                      a, mw, mu, mx);
}

lv_status linear(lv_ctx *ctx, int32_t dtype, LinearArgs &a, const Operands &m, bool gated, cudaStream_t stream) {
  if (!ctx || !is16(dtype) || a.n_tok < 0 || a.n_tok > kMostTokens || m.d_in < 1 || m.d_in > kMostWidth || a.d_out < 1 ||
      a.d_out > kMostWidth || a.act < LV_ACT_NONE || a.act > LV_ACT_RELU)
    return LV_EINVAL;
  if (!rows_ok(m.x, m.x_stride, a.n_tok, m.d_in) || !rows_ok(a.y, a.y_stride, a.n_tok, a.d_out)) return LV_EINVAL;
  for (int k = 0; k < (gated ? 2 : 1); ++k)
    if (!rows_ok(m.w[k], m.w_stride, a.d_out, m.d_in) || !aligned(a.bias[k], 2)) return LV_EINVAL;
  if (a.residual && !rows_ok(a.residual, a.r_stride, a.n_tok, a.d_out)) return LV_EINVAL;
  if (a.residual == a.y && a.residual && a.r_stride != a.y_stride) return LV_EINVAL;
  if (a.n_tok == 0) return LV_OK;
  KvHost *kv = kv_host(ctx);
  a.status = kv->d_status;
  if (gated) return dtype == LV_F16 ? run_linear<true, true>(kv, a, m, stream) : run_linear<true, false>(kv, a, m, stream);
  return dtype == LV_F16 ? run_linear<false, true>(kv, a, m, stream) : run_linear<false, false>(kv, a, m, stream);
}

template <int D, bool F16>
lv_status run_rotate(const KvHost *kv, RotateArgs &a, bool neighbours, cudaStream_t stream) {
  // A token's heads to as many warps as there have to be for one on each of an SM's four
  // schedulers, two or four heads each at least: what a warp does once for its heads (the
  // angles) is half of what eight heads cost it.  (us of 128, 512 and 2,048 tokens, for
  // four warps an SM 4.9, 6.8 and 10.7, for twenty 5.9, 6.1 and 12.2)
  constexpr int kAtOnce = 32 / (D / 8);
  const int heads = a.heads[0] + a.heads[1];
  const int64_t parts = std::min<int64_t>((kv->sms * 4 + a.n_tok - 1) / a.n_tok, (heads + kAtOnce - 1) / kAtOnce);
  a.part = (int)(((heads + parts - 1) / parts + kAtOnce - 1) / kAtOnce * kAtOnce);
  a.parts = (heads + a.part - 1) / a.part;
  const int64_t grid = std::min<int64_t>((a.n_tok * a.parts + kRoWarps - 1) / kRoWarps, kv->sms * kRoCtas);
  constexpr unsigned kThreads = kRoWarps * 32;
  if (a.weight[0] || a.weight[1])
    return neighbours ? launch_after(k_rotate<D, F16, true, true>, grid, kThreads, 0, 0, stream, a)
                      : launch_after(k_rotate<D, F16, true, false>, grid, kThreads, 0, 0, stream, a);
  return neighbours ? launch_after(k_rotate<D, F16, false, true>, grid, kThreads, 0, 0, stream, a)
                    : launch_after(k_rotate<D, F16, false, false>, grid, kThreads, 0, 0, stream, a);
}

template <int TYPE>
lv_status run_logprobs(const KvHost *kv, LogprobArgs &a, cudaStream_t stream) {
  const int64_t vectors = a.vocab / (TYPE == LV_F32 ? 4 : 8);
  // us of 128,000 bf16 logits: one row with 20 alternatives, by a CTA 16.4, two 11.9, four
  // 9.3, eight 8.7; 128 rows with five 19.6, 18.2, 14.1, 18.8.  4,096 rows of 32,000: CTAs
  // of 128 threads 52.8, of 256 63.0; 1,000 rows of 128,000 58.1 and 50.9
  const int threads = a.n_tok >= 16 * kv->sms ? 128 : 256;
  auto pays = [&](int64_t n) {  // n CTAs a row: they fit, and each thread has loads
    return n <= kLpCluster && a.n_tok * n <= 4 * kv->sms && vectors >= n * threads * (a.n_tok * n <= 64 ? 4 : 8);
  };
  while (pays(2 * a.cluster)) a.cluster *= 2;
  const int64_t grid = a.n_tok * a.cluster;
  if (grid > INT32_MAX) return LV_EINVAL;
  return threads == 256 ? launch_after(k_logprobs<TYPE, 256>, grid, 256, 0, a.cluster, stream, a)
                        : launch_after(k_logprobs<TYPE, 128>, grid, 128, 0, a.cluster, stream, a);
}

}  // namespace

extern "C" {

lv_status lv_linear(lv_ctx *ctx, int32_t dtype, const void *x, int64_t x_stride, int64_t n_tok, const void *w,
                    int64_t w_stride, int32_t d_in, int32_t d_out, const void *bias, int32_t act,
                    const void *residual, int64_t residual_stride, void *y, int64_t y_stride, void *stream) {
  LinearArgs a{};
  a.bias[0] = bias, a.residual = residual, a.y = y;
  a.r_stride = residual_stride, a.y_stride = y_stride;
  a.n_tok = n_tok, a.d_out = d_out, a.act = act;
  return linear(ctx, dtype, a, Operands{x, {w, nullptr}, x_stride, w_stride, d_in}, false, (cudaStream_t)stream);
}

lv_status lv_gated_linear(lv_ctx *ctx, int32_t dtype, const void *x, int64_t x_stride, int64_t n_tok,
                          const void *w_gate, const void *w_up, int64_t w_stride, int32_t d_in, int32_t d_out,
                          const void *bias_gate, const void *bias_up, int32_t act, void *y, int64_t y_stride,
                          void *stream) {
  LinearArgs a{};
  a.bias[0] = bias_gate, a.bias[1] = bias_up, a.y = y, a.y_stride = y_stride;
  a.n_tok = n_tok, a.d_out = d_out, a.act = act;
  return linear(ctx, dtype, a, Operands{x, {w_gate, w_up}, x_stride, w_stride, d_in}, true, (cudaStream_t)stream);
}

lv_status lv_qk_rotate(lv_ctx *ctx, int32_t dtype, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                       const void *q, int64_t q_stride, const void *k, int64_t k_stride, int64_t n_tok,
                       const int64_t *token_offsets, const int32_t *c, int64_t n_req, const void *q_weight,
                       const void *k_weight, float eps, const lv_rope *rope, void *q_out, int64_t q_out_stride,
                       void *k_out, int64_t k_out_stride, void *stream_) {
  if (!ctx || !is16(dtype) || (head_dim != 64 && head_dim != 128) || n_kv_heads < 1 || n_kv_heads > 1024 ||
      n_q_heads < n_kv_heads || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > LV_MAX_GROUP)
    return LV_EINVAL;
  if (n_tok < 0 || n_tok > kMostTokens || n_req < 0 || n_req > (1ll << 24) || (!token_offsets && n_tok != n_req) ||
      !(eps >= 0.f) || !std::isfinite(eps))
    return LV_EINVAL;
  if (!rope || rope->dim < 0 || rope->dim > head_dim || rope->dim % 16 ||
      (rope->order != LV_ROPE_HALVES && rope->order != LV_ROPE_NEIGHBOURS))
    return LV_EINVAL;
  RotateArgs a{};
  for (int j = 0; j < rope->dim / 2; ++j) {
    const double f = rope->freq[j];
    if (!(std::fabs(f) <= 8.0)) return LV_EINVAL;
    const double turns = std::fabs(f) / 6.283185307179586476925;  // whole ones do nothing
    const uint64_t turn = (uint64_t)((turns - (double)(int64_t)turns) * 0x1p64);
    a.turn[j] = f < 0.0 ? 0 - turn : turn;
  }
  const int64_t dq = (int64_t)n_q_heads * head_dim, dk = (int64_t)n_kv_heads * head_dim;
  if (!rows_ok(q, q_stride, n_tok, dq) || !rows_ok(k, k_stride, n_tok, dk) || !rows_ok(q_out, q_out_stride, n_tok, dq) ||
      !rows_ok(k_out, k_out_stride, n_tok, dk) || !aligned(q_weight, 2) || !aligned(k_weight, 2))
    return LV_EINVAL;
  if ((q == q_out && q && q_stride != q_out_stride) || (k == k_out && k && k_stride != k_out_stride)) return LV_EINVAL;
  if (n_tok == 0 || n_req == 0) return LV_OK;
  if (!aligned(token_offsets, 8) || !aligned(c, 4)) return LV_EINVAL;
  a.x[0] = q, a.x[1] = k, a.y[0] = q_out, a.y[1] = k_out, a.weight[0] = q_weight, a.weight[1] = k_weight;
  a.x_stride[0] = q_stride, a.x_stride[1] = k_stride, a.y_stride[0] = q_out_stride, a.y_stride[1] = k_out_stride;
  a.n_tok = n_tok, a.offsets = token_offsets, a.c = c, a.n_req = n_req;
  a.heads[0] = n_q_heads, a.heads[1] = n_kv_heads;
  a.dim = rope->dim, a.eps = eps;
  const bool next = rope->order == LV_ROPE_NEIGHBOURS;
  const KvHost *kv = kv_host(ctx);
  a.status = kv->d_status;
  cudaStream_t stream = (cudaStream_t)stream_;
  if (head_dim == 128)
    return dtype == LV_F16 ? run_rotate<128, true>(kv, a, next, stream) : run_rotate<128, false>(kv, a, next, stream);
  return dtype == LV_F16 ? run_rotate<64, true>(kv, a, next, stream) : run_rotate<64, false>(kv, a, next, stream);
}

lv_status lv_token_logprobs(lv_ctx *ctx, int32_t dtype, const void *logits, int64_t stride, int64_t n_tok,
                            int32_t vocab, const int32_t *ids, float *logp, float *entropy, float *lse,
                            int32_t n_top, int32_t *top_ids, float *top_logp, void *stream_) {
  if (!ctx || (!is16(dtype) && dtype != LV_F32) || n_tok < 0 || n_tok > kMostTokens || vocab < 1 || vocab > kMostWidth ||
      n_top < 0 || n_top > LV_MAX_TOP)
    return LV_EINVAL;
  if (n_tok == 0) return LV_OK;
  if (!logits || !aligned(logits, dtype == LV_F32 ? 4 : 2) || stride < vocab || stride > kMostStride || (logp && !ids) ||
      (n_top > 0 && (!top_ids || !top_logp)))
    return LV_EINVAL;
  if (!aligned(ids, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(top_ids, 4) ||
      !aligned(top_logp, 4))
    return LV_EINVAL;
  const KvHost *kv = kv_host(ctx);
  LogprobArgs a{logits, stride, n_tok, vocab, n_top, 1, ids, logp, entropy, lse, top_ids, top_logp, kv->d_status};
  cudaStream_t stream = (cudaStream_t)stream_;
  if (dtype == LV_BF16) return run_logprobs<LV_BF16>(kv, a, stream);
  return dtype == LV_F16 ? run_logprobs<LV_F16>(kv, a, stream) : run_logprobs<LV_F32>(kv, a, stream);
}

}  // extern "C"
