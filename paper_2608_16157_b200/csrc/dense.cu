// Host side of include/ftdense.h: handle, validation, launches.
#include "../../include/ftdense.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <new>

#include "dense_logp.cuh"
#include "dense_norm.cuh"
#include "dense_w4.cuh"
#include "dense_w4_tile.cuh"
#include "host.cuh"

using namespace ftmoe;

struct ft_dense {
  int device = 0, sm_count = 148;
  int clusters[kW4MaxCluster + 1] = {};   // of each size that fit at once, a block an SM
  uint32_t *status_dev = nullptr;
  void *encode = nullptr;          // cuTensorMapEncodeTiled
  uint64_t launches = 0;
};

namespace {

std::atomic<int> g_dense_cuda_error{cudaSuccess};   // the CUDA error behind the latest FT_ERR_CUDA / FT_ERR_OOM

#define FD_CUDA(expr)                                                                       \
  do {                                                                                      \
    cudaError_t e_ = (expr);                                                                \
    if (e_ != cudaSuccess) {                                                                \
      g_dense_cuda_error = e_;                                                              \
      (void)cudaGetLastError();                                                             \
      return e_ == cudaErrorMemoryAllocation ? FT_ERR_OOM : FT_ERR_CUDA;                    \
    }                                                                                       \
  } while (0)

bool type16(int dtype) { return dtype == FT_DENSE_BF16 || dtype == FT_DENSE_FP16; }
bool aligned(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

bool w4_ok(int64_t n, int64_t k, int group) {
  return n >= 1 && n <= (1 << 24) && (group == 32 || group == 64 || group == 128) && k >= group && k <= 65536 && k % group == 0;
}

template <bool BF16, bool RES32, bool POST, bool GATE, int E>
cudaError_t launch_norm_form(const NormArgs &a, bool wide, cudaStream_t st) {
  const int threads = a.lanes > 32 ? a.lanes : 128, rows = threads / a.lanes;
  const unsigned grid = (unsigned)(((long long)a.T + rows - 1) / rows);
  if (!wide) return launch(add_norm_kernel<BF16, RES32, POST, GATE, 1, false, E>, grid, threads, 0, st, a);
  return a.wide == kWideAll ? launch(add_norm_kernel<BF16, RES32, POST, GATE, 8, true, E>, grid, threads, 0, st, a)
                            : launch(add_norm_kernel<BF16, RES32, POST, GATE, 8, false, E>, grid, threads, 0, st, a);
}
template <bool BF16, bool RES32, int E>
cudaError_t launch_norm_elems(NormArgs a, bool wide, cudaStream_t st) {
  a.lanes = 32;
  while (a.lanes * E < a.d) a.lanes *= 2;
  const bool gate = a.y && a.gate && a.gate_step;
  if (a.post) return gate ? launch_norm_form<BF16, RES32, true, true, E>(a, wide, st) : launch_norm_form<BF16, RES32, true, false, E>(a, wide, st);
  return gate ? launch_norm_form<BF16, RES32, false, true, E>(a, wide, st) : launch_norm_form<BF16, RES32, false, false, E>(a, wide, st);
}

template <bool BF16, bool RES32>
cudaError_t launch_norm(const ft_dense *h, const NormArgs &a, bool wide, cudaStream_t st) {
  // 8 elements a thread while that leaves no more threads than the SMs hold at once, then 16 (32, with half of the threads an SM: 68 us for 16384 tokens
  // of 2048 against 61; 8: 79)
  if ((long long)a.T * a.d > 8ll * h->sm_count * 1024 || a.d > 8 * 1024) return launch_norm_elems<BF16, RES32, 16>(a, wide, st);
  return launch_norm_elems<BF16, RES32, 8>(a, wide, st);
}

template <bool BF16, int G, bool ZERO, int NT>
cudaError_t launch_w4_stream(const ft_dense *h, const W4Args &a, cudaStream_t st) {
  W4Stream p;
  w4_stream_share(a.g, h->clusters, kW4Warps<NT>, p);
  const int smem = w4_stream_memory<NT>(a.g, p);
  const int per_block = kW4Warps<NT> / p.wk, want = (a.g.quads + per_block - 1) / per_block, fit = h->clusters[p.cluster];
  return launch_clusters(w4_stream_kernel<BF16, G, ZERO, NT>, dim3((want < fit ? want : fit) * p.cluster, (a.T + 8 * NT - 1) / (8 * NT)), kW4Warps<NT> * 32, smem,
                         p.cluster, st, a, p);
}

template <bool BF16, int G, bool ZERO>
cudaError_t launch_w4_tokens(const ft_dense *h, const W4Args &a, cudaStream_t st) {
  if (a.T <= 8) return launch_w4_stream<BF16, G, ZERO, 1>(h, a, st);
  if (a.T <= 16) return launch_w4_stream<BF16, G, ZERO, 2>(h, a, st);
  return launch_w4_stream<BF16, G, ZERO, 4>(h, a, st);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// x as [T][k]; a box is 64 k of a tile's tokens, rows of 128 bytes with the 128-byte swizzle.
bool make_x_map(const ft_dense *h, CUtensorMap *tm, const W4Args &a, int tokens) {
  const cuuint64_t dims[2] = {(cuuint64_t)a.g.k, (cuuint64_t)a.T}, strides[1] = {(cuuint64_t)a.x_stride * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)tokens}, ones[2] = {1, 1};
  return reinterpret_cast<EncodeTiledFn>(h->encode)(tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<uint16_t *>(a.x), dims, strides, box, ones,
                                                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF16, bool ZERO, bool EXACT>
cudaError_t launch_w4_tile(const ft_dense *h, const W4Args &a, W4Tile p, cudaStream_t st) {
  CUtensorMap tm;
  if (!make_x_map(h, &tm, a, p.bn)) return cudaErrorInvalidValue;
  const int smem = w4_tile_memory<EXACT>(a.g, p), units = p.row_tiles * p.tok_tiles, fit = h->clusters[p.cluster];
  return launch_clusters(w4_tile_kernel<BF16, ZERO, EXACT>, dim3((p.cluster > 1 || units < fit ? units : fit) * p.cluster), W4TileCfg<EXACT>::kThreads, smem, p.cluster, st, tm, a, p, W4Again{a, p});
}

template <bool BF16, bool ZERO>
cudaError_t launch_w4_many(const ft_dense *h, const W4Args &a, cudaStream_t st) {
  const W4Tile p = w4_tile_share(a.g, a.T, a.out32 != 0, h->clusters);
  return a.out32 ? launch_w4_tile<BF16, ZERO, true>(h, a, p, st) : launch_w4_tile<BF16, ZERO, false>(h, a, p, st);
}

template <bool BF16>
cudaError_t launch_w4(const ft_dense *h, const W4Args &a, bool zero, cudaStream_t st) {
  if (a.T > (a.out32 ? 32 : 16)) return zero ? launch_w4_many<BF16, true>(h, a, st) : launch_w4_many<BF16, false>(h, a, st);
  switch (a.g.group) {
    case 32: return zero ? launch_w4_tokens<BF16, 32, true>(h, a, st) : launch_w4_tokens<BF16, 32, false>(h, a, st);
    case 64: return zero ? launch_w4_tokens<BF16, 64, true>(h, a, st) : launch_w4_tokens<BF16, 64, false>(h, a, st);
    default: return zero ? launch_w4_tokens<BF16, 128, true>(h, a, st) : launch_w4_tokens<BF16, 128, false>(h, a, st);
  }
}

// A row to a cluster of blocks of 512 threads while one a SM takes them all, as many as leave a thread some pieces; more rows to blocks of 256,
// four a SM, whose ends overlap with the others' passes (two to a row while all fit at once); short rows to the smallest.
template <int TY>
cudaError_t launch_logprobs(const ft_dense *h, const LogpArgs &a, cudaStream_t st) {
  const long long pieces = a.vocab / LogpType<TY>::kVec, sms = h->sm_count;
  if (pieces <= 1024 && a.T > sms) return launch(logprobs_kernel<TY, 128>, dim3((unsigned)a.T), 128, sizeof(LogpSmem<4>), st, a, 1);
  int cluster = 1;
  if (a.T > sms) {
    if (2ll * a.T <= 4 * sms && pieces >= 2048) cluster = 2;
    return launch_clusters(logprobs_kernel<TY, 256>, dim3((unsigned)a.T * cluster), 256, sizeof(LogpSmem<8>), cluster, st, a, cluster);
  }
  while (cluster < kLogpCluster && 2ll * a.T * cluster <= sms && pieces >= 1024 * cluster) cluster *= 2;
  return launch_clusters(logprobs_kernel<TY, 512>, dim3((unsigned)a.T * cluster), 512, sizeof(LogpSmem<16>), cluster, st, a, cluster);
}

constexpr int kMaxSmem = 227 * 1024;

template <bool BF16, int G, bool ZERO>
cudaError_t allow_smem_stream() {
  cudaError_t e = cudaFuncSetAttribute(w4_stream_kernel<BF16, G, ZERO, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(w4_stream_kernel<BF16, G, ZERO, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(w4_stream_kernel<BF16, G, ZERO, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  return e;
}
template <bool BF16, bool ZERO>
cudaError_t allow_smem() {
  cudaError_t e = allow_smem_stream<BF16, 32, ZERO>();
  if (e == cudaSuccess) e = allow_smem_stream<BF16, 64, ZERO>();
  if (e == cudaSuccess) e = allow_smem_stream<BF16, 128, ZERO>();
  if (e == cudaSuccess) e = cudaFuncSetAttribute(w4_tile_kernel<BF16, ZERO, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(w4_tile_kernel<BF16, ZERO, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  return e;
}

template <int TY>
cudaError_t allow_smem_logprobs() {
  return cudaFuncSetAttribute(logprobs_kernel<TY, 512>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(LogpSmem<16>));
}

// How many clusters of a size run at once when each block takes an SM (the SMs of a cluster stand together, so not all are used).
cudaError_t count_clusters(ft_dense *h) {
  for (int c = 1; c <= kW4MaxCluster; ++c) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(c * h->sm_count);
    cfg.blockDim = dim3(W4TileCfg<false>::kThreads);
    cfg.dynamicSmemBytes = kMaxSmem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = c;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = h->sm_count;
    const cudaError_t e = c == 1 ? cudaSuccess : cudaOccupancyMaxActiveClusters(&n, w4_tile_kernel<true, false, false>, &cfg);
    if (e != cudaSuccess) return e;
    h->clusters[c] = n;
  }
  return cudaSuccess;
}

}  // namespace

extern "C" {

const char *ft_dense_last_cuda_error(void) { return cudaGetErrorString((cudaError_t)g_dense_cuda_error.load()); }

ft_status_t ft_dense_create(int device, ft_dense_t **out) {
  if (!out) return FT_ERR_INVALID_ARG;
  *out = nullptr;
  if (device < 0) return FT_ERR_INVALID_ARG;
  DeviceScope dev(device);
  FD_CUDA(dev.err);
  ft_dense *h = new (std::nothrow) ft_dense();
  if (!h) return FT_ERR_OOM;
  h->device = device;
  cudaError_t e = cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) e = cudaMalloc(&h->status_dev, 256);
  if (e == cudaSuccess) e = cudaMemset(h->status_dev, 0, 256);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
  if (e == cudaSuccess) e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &h->encode, cudaEnableDefault, &found);
  if (e == cudaSuccess) e = allow_smem<true, true>();
  if (e == cudaSuccess) e = allow_smem<true, false>();
  if (e == cudaSuccess) e = allow_smem<false, true>();
  if (e == cudaSuccess) e = allow_smem<false, false>();
  if (e == cudaSuccess) e = allow_smem_logprobs<kLogpBf16>();
  if (e == cudaSuccess) e = allow_smem_logprobs<kLogpFp16>();
  if (e == cudaSuccess) e = allow_smem_logprobs<kLogpFp32>();
  if (e == cudaSuccess) e = count_clusters(h);
  if (e == cudaSuccess && (!h->encode || found != cudaDriverEntryPointSuccess)) e = cudaErrorNotSupported;
  if (e != cudaSuccess) {
    (void)cudaFree(h->status_dev);
    delete h;
    FD_CUDA(e);
  }
  *out = h;
  return FT_OK;
}

ft_status_t ft_dense_destroy(ft_dense_t *h) {
  if (!h) return FT_OK;
  DeviceScope dev(h->device);
  cudaError_t e = cudaDeviceSynchronize();
  (void)cudaFree(h->status_dev);
  delete h;
  FD_CUDA(e);
  return FT_OK;
}

ft_status_t ft_dense_add_norm(ft_dense_t *h, int T, int d, int dtype, int res_dtype, int flags, const void *y, int64_t y_stride,
                              const void *res, int64_t res_stride, const void *gate, int64_t gate_stride, int gate_step,
                              const void *w_post, const void *w_pre, float w_offset, float eps, float res_scale, float y_scale,
                              void *res_out, int64_t res_out_stride, void *out, int64_t out_stride, void *stream) {
  if (!h || T < 0 || d < 1 || !type16(dtype) || (res_dtype != dtype && res_dtype != FT_DENSE_FP32) || (flags & ~FT_DENSE_NORM_POST))
    return FT_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || (gate_step != 0 && gate_step != 1)) return FT_ERR_INVALID_ARG;
  if (d > kNormMaxDim) return FT_ERR_UNSUPPORTED;
  if (T == 0) return FT_OK;
  if ((!y && !res) || (!res_out && !out)) return FT_ERR_INVALID_ARG;
  const bool res32 = res_dtype == FT_DENSE_FP32;
  if (!aligned(y, 2) || !aligned(gate, 2) || !aligned(w_post, 2) || !aligned(w_pre, 2) || !aligned(out, 2) || !aligned(res, res32 ? 4 : 2) ||
      !aligned(res_out, res32 ? 4 : 2))
    return FT_ERR_INVALID_ARG;
  if ((y && T > 1 && y_stride < d) || (res && T > 1 && res_stride < d) || (res_out && T > 1 && res_out_stride < d) || (out && T > 1 && out_stride < d) ||
      (gate && gate_stride < 0))
    return FT_ERR_INVALID_ARG;
  // a row is read whole before it is written, but only by its own threads
  if ((res_out && res_out == res && T > 1 && res_out_stride != res_stride) || (out && out == y && T > 1 && out_stride != y_stride)) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->device);
  FD_CUDA(dev.err);
  NormArgs a;
  a.T = T; a.d = d; a.post = y && (flags & FT_DENSE_NORM_POST) ? 1 : 0; a.gate_step = gate_step;
  a.y = static_cast<const uint16_t *>(y); a.gate = static_cast<const uint16_t *>(gate);
  a.w_post = static_cast<const uint16_t *>(w_post); a.w_pre = static_cast<const uint16_t *>(w_pre);
  a.res = res; a.res_out = res_out; a.out = static_cast<uint16_t *>(out);
  a.y_stride = y_stride; a.res_stride = res_stride; a.gate_stride = gate_stride; a.res_out_stride = res_out_stride; a.out_stride = out_stride;
  a.w_offset = w_offset; a.eps = eps; a.res_scale = res_scale; a.y_scale = y_scale;
  a.mean_low = eps > 1.3e-23f ? 0u : (127u - 100u) << 23;          // (2^-76), 2^-100
  auto rows16 = [&](const void *p, int64_t stride, int bytes) { return aligned(p, 16) && (T == 1 || stride * bytes % 16 == 0); };
  a.wide = (rows16(y, y_stride, 2) ? kWideY : 0u) | (rows16(res, res_stride, res32 ? 4 : 2) ? kWideRes : 0u) | (rows16(gate, gate_stride, 2) ? kWideGate : 0u) |
           (aligned(w_post, 16) ? kWidePost : 0u) | (aligned(w_pre, 16) ? kWidePre : 0u) | (rows16(res_out, res_out_stride, res32 ? 4 : 2) ? kWideResOut : 0u) |
           (rows16(out, out_stride, 2) ? kWideOut : 0u);
  // eight elements at a time, unless hardly an array would have them in one access
  const bool wide = d % 8 == 0 && ((a.wide & kWideY) || (a.wide & kWideRes));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf = dtype == FT_DENSE_BF16;
  FD_CUDA(bf ? (res32 ? launch_norm<true, true>(h, a, wide, st) : launch_norm<true, false>(h, a, wide, st))
             : (res32 ? launch_norm<false, true>(h, a, wide, st) : launch_norm<false, false>(h, a, wide, st)));
  h->launches += 1;
  return FT_OK;
}

size_t ft_dense_w4_bytes(int64_t n, int64_t k, int group, int has_zeros) {
  if (!w4_ok(n, k, group)) return 0;
  return (size_t)w4_geom(n, k, group, has_zeros != 0).bytes();
}

ft_status_t ft_dense_w4_pack(ft_dense_t *h, int64_t n, int64_t k, int group, int dtype, const uint8_t *codes, int64_t codes_stride,
                             const void *scales, const uint8_t *zeros, void *image, void *stream) {
  if (!h || !type16(dtype)) return FT_ERR_INVALID_ARG;
  if (!w4_ok(n, k, group)) return FT_ERR_UNSUPPORTED;
  if (!codes || !scales || !image || (n > 1 && codes_stride < k / 2) || !aligned(scales, 2) || !aligned(image, 16)) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->device);
  FD_CUDA(dev.err);
  const W4Geom g = w4_geom(n, k, group, zeros != nullptr);
  const long long blocks = ((long long)g.quads * g.nb + 7) / 8;
  const unsigned grid = (unsigned)(blocks < 16ll * h->sm_count ? blocks : 16ll * h->sm_count);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint16_t *sc = static_cast<const uint16_t *>(scales);
  FD_CUDA(dtype == FT_DENSE_BF16 ? launch(w4_pack_kernel<true>, grid, 256, 0, st, g, codes, codes_stride, sc, zeros, static_cast<uint8_t *>(image))
                                 : launch(w4_pack_kernel<false>, grid, 256, 0, st, g, codes, codes_stride, sc, zeros, static_cast<uint8_t *>(image)));
  h->launches += 1;
  return FT_OK;
}

ft_status_t ft_dense_w4_forward(ft_dense_t *h, int T, int64_t n, int64_t k, int group, int dtype, int has_zeros, const void *x,
                                int64_t x_stride, const void *image, const void *bias, void *y, int64_t y_stride, int out_dtype,
                                void *stream) {
  if (!h || T < 0 || T > (1 << 20) || !type16(dtype) || (out_dtype != dtype && out_dtype != FT_DENSE_FP32)) return FT_ERR_INVALID_ARG;
  if (!w4_ok(n, k, group)) return FT_ERR_UNSUPPORTED;
  if (T == 0) return FT_OK;
  const bool out32 = out_dtype == FT_DENSE_FP32;
  if (!x || !image || !y || !aligned(x, 16) || !aligned(image, 16) || !aligned(bias, 2) || !aligned(y, out32 ? 4 : 2)) return FT_ERR_INVALID_ARG;
  if (T > 1 && (x_stride < k || x_stride % 8 || x_stride >= (1ll << 38) || y_stride < n)) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->device);
  FD_CUDA(dev.err);
  W4Args a;
  a.g = w4_geom(n, k, group, has_zeros != 0);
  a.T = T; a.out32 = out32 ? 1 : 0;
  a.x = static_cast<const uint16_t *>(x); a.bias = static_cast<const uint16_t *>(bias);
  a.image = static_cast<const uint8_t *>(image); a.y = y;
  a.x_stride = x_stride; a.y_stride = y_stride; a.status = h->status_dev;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  FD_CUDA(dtype == FT_DENSE_BF16 ? launch_w4<true>(h, a, has_zeros != 0, st) : launch_w4<false>(h, a, has_zeros != 0, st));
  h->launches += 1;
  return FT_OK;
}

ft_status_t ft_dense_logprobs(ft_dense_t *h, int T, int64_t vocab, int dtype, const void *logits, int64_t stride, float scale,
                              const int32_t *tokens, int64_t tokens_stride, int n_tokens, float *logprob, float *entropy, int top_k,
                              int32_t *top_ids, float *top_logprobs, void *stream) {
  if (!h || T < 0 || vocab < 1 || vocab > (1 << 30) || (!type16(dtype) && dtype != FT_DENSE_FP32) || !(scale > 0.f) || !(scale <= kLogpMaxScale) ||
      n_tokens < 0 || top_k < 0 || top_k > kLogpTop)
    return FT_ERR_INVALID_ARG;
  if (T == 0) return FT_OK;
  const bool given = tokens && n_tokens > 0;
  if (!logits || (given && !logprob) || (top_k > 0 && (!top_ids || !top_logprobs)) || (n_tokens > 0 && !tokens)) return FT_ERR_INVALID_ARG;
  if (!aligned(logits, dtype == FT_DENSE_FP32 ? 4 : 2) || !aligned(tokens, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(top_ids, 4) ||
      !aligned(top_logprobs, 4) || (T > 1 && (stride < vocab || (given && tokens_stride < n_tokens))))
    return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->device);
  FD_CUDA(dev.err);
  LogpArgs a;
  a.logits = logits; a.stride = stride; a.T = T; a.vocab = (int32_t)vocab; a.n_tokens = given ? n_tokens : 0; a.top_k = top_k;
  logp_scale(a, scale);
  a.tokens = given ? tokens : nullptr; a.tokens_stride = tokens_stride;
  a.logprob = logprob; a.entropy = entropy; a.top_logprobs = top_logprobs; a.top_ids = top_ids;
  a.status = h->status_dev;
  FD_CUDA(dtype == FT_DENSE_BF16   ? launch_logprobs<kLogpBf16>(h, a, static_cast<cudaStream_t>(stream))
          : dtype == FT_DENSE_FP16 ? launch_logprobs<kLogpFp16>(h, a, static_cast<cudaStream_t>(stream))
                                   : launch_logprobs<kLogpFp32>(h, a, static_cast<cudaStream_t>(stream)));
  h->launches += 1;
  return FT_OK;
}

ft_status_t ft_dense_sync_status(ft_dense_t *h) {
  if (!h) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->device);
  FD_CUDA(dev.err);
  FD_CUDA(cudaDeviceSynchronize());
  uint32_t st = 0;
  FD_CUDA(cudaMemcpy(&st, h->status_dev, sizeof(st), cudaMemcpyDeviceToHost));
  if (!st) return FT_OK;
  FD_CUDA(cudaMemset(h->status_dev, 0, sizeof(st)));
  FD_CUDA(cudaDeviceSynchronize());
  return (st & kStatTimeout) ? FT_ERR_TIMEOUT : FT_ERR_INVALID_ARG;
}

ft_status_t ft_dense_debug_inject(ft_dense_t *h, uint32_t withhold_mask, uint32_t wait_polls) {
  if (!h) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->device);
  FD_CUDA(dev.err);
  const uint32_t polls = wait_polls ? wait_polls : kDefaultWaitPolls;
  FD_CUDA(cudaDeviceSynchronize());
  FD_CUDA(cudaMemcpyToSymbol(g_debug_withhold, &withhold_mask, sizeof(withhold_mask)));
  FD_CUDA(cudaMemcpyToSymbol(g_wait_polls, &polls, sizeof(polls)));
  FD_CUDA(cudaDeviceSynchronize());
  return FT_OK;
}

ft_status_t ft_dense_launch_count(ft_dense_t *h, uint64_t *out) {
  if (!h || !out) return FT_ERR_INVALID_ARG;
  *out = h->launches;
  return FT_OK;
}

}  // extern "C"
