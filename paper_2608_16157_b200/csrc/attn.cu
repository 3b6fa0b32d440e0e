// Host side of include/ftattn.h: handle, validation, launches.
#include "../../include/ftattn.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstring>
#include <new>
#include <utility>

#include "attn_plan.cuh"
#include "attn_rope.cuh"
#include "attn_stream.cuh"
#include "attn_tile.cuh"

using namespace ftmoe;

struct ft_attn {
  ft_attn_config_t cfg;
  int sm_count = 148, page_shift = 4;
  uint32_t *status_dev = nullptr;
  uint8_t *work_mem = nullptr;     // the work partition, one allocation
  AttnWork work;
  AttnGeom geom;
  float *part = nullptr;           // partial results of work items that several CTAs share: streaming kernel, tiled kernel
  size_t part_tile = 0;            // floats before the second
  uint32_t *arrive = nullptr;      // arrival counters of the streaming kernel's
  size_t arrive_bytes = 0;
  void *encode = nullptr;          // cuTensorMapEncodeTiled
  bool planned = false;
  int n_req = 0, T = 0, max_new = 0;   // of the latest slots / plan call
  uint64_t launches = 0;
};

namespace {

cudaError_t g_attn_cuda_error = cudaSuccess;   // the CUDA error behind the latest FT_ERR_CUDA / FT_ERR_OOM

#define FA_CUDA(expr)                                                                       \
  do {                                                                                      \
    cudaError_t e_ = (expr);                                                                \
    if (e_ != cudaSuccess) {                                                                \
      g_attn_cuda_error = e_;                                                               \
      (void)cudaGetLastError();                                                             \
      return e_ == cudaErrorMemoryAllocation ? FT_ERR_OOM : FT_ERR_CUDA;                    \
    }                                                                                       \
  } while (0)

ft_status_t check_config(const ft_attn_config_t *c) {
  if (!c || c->struct_size != sizeof(ft_attn_config_t)) return FT_ERR_INVALID_ARG;
  if (c->device < 0 || (c->dtype != FT_ATTN_BF16 && c->dtype != FT_ATTN_FP16)) return FT_ERR_INVALID_ARG;
  if (c->n_kv_heads < 1 || c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads || c->n_q_heads > 1024 ||
      c->n_q_heads / c->n_kv_heads > 64)
    return FT_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->n_pages >= (1 << 22) || c->max_requests < 1 || c->max_requests > kAttnMaxRequests || c->max_tokens < 1 ||
      c->max_tokens > (1 << 20) || c->max_pages < 1 || c->window < 0)
    return FT_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FT_ERR_UNSUPPORTED;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return FT_ERR_UNSUPPORTED;
  if ((long long)c->n_pages * c->page_tokens >= (1ll << 31) || (long long)c->max_pages * c->page_tokens >= (1ll << 31))
    return FT_ERR_INVALID_ARG;
  // work units of a step are counted in 32 bits: key blocks of all requests and of all tiles of a request's rows
  const long long blocks = (long long)c->max_pages * c->page_tokens / kDecKeys + 2 + kTileCost;
  const long long tile_tokens = 2 * (kTileRows / (c->n_q_heads / c->n_kv_heads));
  const long long entries = c->max_tokens / tile_tokens + c->max_requests;
  if (blocks * c->max_requests * c->n_kv_heads >= (1ll << 31) || blocks * entries * c->n_kv_heads >= (1ll << 31)) return FT_ERR_UNSUPPORTED;
  return FT_OK;
}

// Restores the calling thread's current device when the entry point returns.
struct DeviceScope {
  int prev = -1;
  cudaError_t err;
  explicit DeviceScope(int dev) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && prev != dev) err = cudaSetDevice(dev); else prev = -1;
  }
  ~DeviceScope() { if (prev >= 0) (void)cudaSetDevice(prev); }
};

void free_all(ft_attn *h) {
  (void)cudaFree(h->status_dev);
  (void)cudaFree(h->work_mem);
  (void)cudaFree(h->part);
  (void)cudaFree(h->arrive);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// 16-bit elements, 128-byte swizzle: `rank` dimensions from the innermost, strides in elements.
bool make_map(const ft_attn *h, CUtensorMap *tm, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *stride_elems,
              const cuuint32_t *box) {
  cuuint64_t strides[4];
  const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
  for (int i = 0; i + 1 < rank; ++i) strides[i] = stride_elems[i] * 2;
  return reinterpret_cast<EncodeTiledFn>(h->encode)(tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, rank, const_cast<void *>(base), dims, strides, box,
                                                    ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The cache of a layer as [(page, keys or values, head)][tokens of the page][D]; a box is 64 elements of up to 64 tokens.
bool make_cache_map(const ft_attn *h, CUtensorMap *tm, const void *cache) {
  const ft_attn_config_t &c = h->cfg;
  const cuuint64_t dims[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_tokens, (cuuint64_t)c.n_pages * 2 * c.n_kv_heads};
  const cuuint64_t strides[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_tokens * c.head_dim};
  const cuuint32_t box[3] = {64, (cuuint32_t)(c.page_tokens < kDecKeys ? c.page_tokens : kDecKeys), 1};
  return make_map(h, tm, cache, 3, dims, strides, box);
}

// The packed queries as [T][key/value head][head of the group][D]; a box is 64 elements of all heads of a group, of the
// tokens of one 128-row tile.
bool make_query_map(const ft_attn *h, CUtensorMap *tm, const void *q, int64_t q_stride) {
  const ft_attn_config_t &c = h->cfg;
  const cuuint64_t D = c.head_dim, G = h->geom.group;
  const cuuint64_t dims[4] = {D, G, (cuuint64_t)c.n_kv_heads, (cuuint64_t)h->T};
  const cuuint64_t strides[3] = {D, G * D, (cuuint64_t)q_stride};
  const cuuint32_t box[4] = {64, (cuuint32_t)G, 1, (cuuint32_t)(kTileRows / h->geom.group)};
  return make_map(h, tm, q, 4, dims, strides, box);
}

// The same cache as [(page, keys or values, head)][keys, values][chunk of 64 elements][tokens of the page][64 elements]: from the
// place of a head's keys, a box is the keys and values of up to 64 tokens.
bool make_page_map(const ft_attn *h, CUtensorMap *tm, const void *cache) {
  const ft_attn_config_t &c = h->cfg;
  const cuuint64_t D = c.head_dim, page = (cuuint64_t)c.page_tokens * D;
  const cuuint64_t dims[5] = {64, (cuuint64_t)c.page_tokens, D / 64, 2, (cuuint64_t)c.n_pages * 2 * c.n_kv_heads - c.n_kv_heads};
  const cuuint64_t strides[4] = {D, 64, page * c.n_kv_heads, page};
  const cuuint32_t box[5] = {64, (cuuint32_t)(c.page_tokens < kDecKeys ? c.page_tokens : kDecKeys), (cuuint32_t)(D / 64), 2, 1};
  return make_map(h, tm, cache, 5, dims, strides, box);
}

template <int D, bool BF16>
cudaError_t allow_smem() {
  cudaError_t e = cudaFuncSetAttribute(attn_stream_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, StreamCfg<D>::kSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_rope_stream_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448 / kRopeBlocks - 1024);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(attn_tile_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileCfg<D>::kSmem);
  return e;
}

// A launch the stream's next kernel may be scheduled beside: every kernel here waits for all before it (grid_wait) before it
// touches memory that a kernel or a copy of the stream writes, so only launch latency and prologues overlap.
template <typename... P, typename... Args>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, Args &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

template <int D, bool BF16>
ft_status_t launch_forward(ft_attn *h, AttnFwdArgs a, const void *cache, cudaStream_t st) {
  CUtensorMap tm, tm_q;
  if (!make_page_map(h, &tm, cache)) return FT_ERR_CUDA;
  a.part = h->part;
  a.arrive = h->arrive;
  FA_CUDA(launch(attn_stream_kernel<D, BF16>, h->geom.dec_grid, StreamCfg<D>::kThreads, StreamCfg<D>::kSmem, st, tm, a));
  h->launches += 1;
  if (h->max_new * h->geom.group > kDecRows) {
    if (!make_query_map(h, &tm_q, a.q, a.q_stride) || !make_cache_map(h, &tm, cache)) return FT_ERR_CUDA;
    a.part = h->part + h->part_tile;
    FA_CUDA(launch(attn_tile_kernel<D, BF16>, h->geom.tile_grid, kTileThreads, TileCfg<D>::kSmem, st, tm_q, tm, a));
    FA_CUDA(launch(attn_join_kernel<D, BF16>, dim3(h->geom.tile_grid - 1, 2 * (D / 16)), 128, 0, st, a));
    h->launches += 2;
  }
  return FT_OK;
}

template <int D, bool BF16>
cudaError_t launch_rope(const ft_attn *h, RopeArgs &a, bool wide, cudaStream_t st) {
  const int heads = a.n_q + 2 * a.n_kv, lanes = wide ? D / 16 : D / 8;
  // one head per lane group while that does not fill the GPU (2048 threads an SM), more, up to 8, where it fills it several
  // times over: the token's cosines and sines are read once per group
  const long long fill = (long long)a.T * heads * lanes / ((long long)h->sm_count * 2048);
  a.heads_per_group = fill < 1 ? 1 : fill > 8 ? 8 : (int)fill;
  // many tokens: resident blocks (kRopeBlocks an SM), a lane group for every head or every second, third, ... one
  const int stage = rope_stage_bytes(heads, D, 2 * a.rot_half), smem = kRopeStages * stage + 2 * kRopeStages * 8 + 16;
  if (wide && fill >= 1 && smem <= 232448 / kRopeBlocks - 1024) {
    const int passes = (heads * lanes + 511) / 512, consumers = ((heads + passes - 1) / passes * lanes + 31) / 32 * 32;
    const long long blocks = (long long)h->sm_count * kRopeBlocks;
    return launch(attn_rope_stream_kernel<D, BF16>, (unsigned)(a.T < blocks ? a.T : blocks), consumers + 32, smem, st, a);
  }
  const int parts = (heads + a.heads_per_group - 1) / a.heads_per_group;
  const unsigned grid = (unsigned)(((long long)a.T * parts * lanes + 255) / 256);
  return wide ? launch(attn_rope_kernel<D, BF16, 8>, grid, 256, 0, st, a) : launch(attn_rope_kernel<D, BF16, 4>, grid, 256, 0, st, a);
}

ft_status_t allocate(ft_attn *h) {
  const ft_attn_config_t &c = h->cfg;
  FA_CUDA(cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, c.device));
  AttnGeom &g = h->geom;
  g.group = c.n_q_heads / c.n_kv_heads;
  g.n_kv = c.n_kv_heads;
  g.window = c.window;
  g.tile_tokens = 2 * (kTileRows / g.group);
  g.dec_grid = g.tile_grid = h->sm_count < kAttnMaxGrid ? h->sm_count : kAttnMaxGrid;
  g.dec_min_quota = 2;      // one block and its cost (one request of 1000 tokens: 9.1 us with 1, 8.5 with 2, 9.8 with 3)
  g.tile_min_quota = 1;
  g.tile_cap = c.max_tokens / g.tile_tokens + c.max_requests;
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  const size_t n_dec = up(sizeof(AttnEntry) * (size_t)c.max_requests), n_tile = up(sizeof(AttnEntry) * (size_t)g.tile_cap);
  const size_t n_start = up(sizeof(AttnStart) * kAttnMaxGrid), total = 256 + n_dec + n_tile + 2 * n_start;
  FA_CUDA(cudaMalloc(&h->work_mem, total));
  FA_CUDA(cudaMemset(h->work_mem, 0, total));
  FA_CUDA(cudaMalloc(&h->status_dev, 256));
  FA_CUDA(cudaMemset(h->status_dev, 0, 256));
  uint8_t *b = h->work_mem;
  h->work.hdr = reinterpret_cast<AttnPlanHdr *>(b); b += 256;
  h->work.dec = reinterpret_cast<AttnEntry *>(b); b += n_dec;
  h->work.tile = reinterpret_cast<AttnEntry *>(b); b += n_tile;
  h->work.dec_start = reinterpret_cast<AttnStart *>(b); b += n_start;
  h->work.tile_start = reinterpret_cast<AttnStart *>(b);
  h->part_tile = (size_t)g.dec_grid * 2 * (c.head_dim == 128 ? StreamCfg<128>::kPart : StreamCfg<64>::kPart);
  const size_t part = h->part_tile + (size_t)g.tile_grid * 4 * (c.head_dim == 128 ? TileCfg<128>::kPart : TileCfg<64>::kPart);
  FA_CUDA(cudaMalloc(&h->part, part * sizeof(float)));
  h->arrive_bytes = (size_t)c.max_requests * c.n_kv_heads * sizeof(uint32_t);
  FA_CUDA(cudaMalloc(&h->arrive, h->arrive_bytes));
  FA_CUDA(cudaMemset(h->arrive, 0, h->arrive_bytes));
  FA_CUDA((allow_smem<64, true>()));
  FA_CUDA((allow_smem<64, false>()));
  FA_CUDA((allow_smem<128, true>()));
  FA_CUDA((allow_smem<128, false>()));
  cudaDriverEntryPointQueryResult qres;
  FA_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &h->encode, cudaEnableDefault, &qres));
  if (!h->encode || qres != cudaDriverEntryPointSuccess) return FT_ERR_CUDA;
  FA_CUDA(cudaDeviceSynchronize());
  return FT_OK;
}

bool step_ok(const ft_attn *h, int n_req, int T, int max_new) {
  return n_req >= 0 && n_req <= h->cfg.max_requests && T >= 0 && T <= h->cfg.max_tokens && max_new >= 0 && max_new <= T;
}

ft_status_t launch_slots(ft_attn *h, AttnSlotsArgs &a, cudaStream_t st) {
  a.max_pages = h->cfg.max_pages;
  a.n_pages = h->cfg.n_pages;
  a.page_shift = h->page_shift;
  a.w = h->work;
  a.g = h->geom;
  a.status = h->status_dev;
  // block 0 keeps the requests and the work partition; the others share the tokens and pages, a token a thread while there are
  // SMs for that (a token waits for two loads, one after the other)
  const int threads = a.n_req <= 256 ? 256 : 1024;
  const int blocks = 1 + (a.T > 1 ? a.T - 1 : 0) / threads;
  const int grid = a.own_tables ? 1 : 1 + (blocks < h->sm_count - 1 ? blocks : h->sm_count - 1);
  FA_CUDA(threads == 256 ? launch(attn_slots_kernel<256>, grid, 256, 0, st, a) : launch(attn_slots_kernel<1024>, grid, 1024, 0, st, a));
  h->launches += 1;
  h->planned = true;
  h->n_req = a.n_req; h->T = a.T; h->max_new = a.max_new;
  return FT_OK;
}

}  // namespace

extern "C" {

size_t ft_attn_cache_bytes(const ft_attn_config_t *cfg) {
  if (check_config(cfg) != FT_OK) return 0;
  return (size_t)cfg->n_pages * 2 * cfg->n_kv_heads * cfg->page_tokens * cfg->head_dim * 2;
}

const char *ft_attn_last_cuda_error(void) { return cudaGetErrorString(g_attn_cuda_error); }

ft_status_t ft_attn_create(const ft_attn_config_t *cfg, ft_attn_t **out) {
  if (!out) return FT_ERR_INVALID_ARG;
  *out = nullptr;
  ft_status_t rc = check_config(cfg);
  if (rc != FT_OK) return rc;
  DeviceScope dev(cfg->device);
  FA_CUDA(dev.err);
  ft_attn *h = new (std::nothrow) ft_attn();
  if (!h) return FT_ERR_OOM;
  h->cfg = *cfg;
  // a window no request outgrows hides nothing; left as it is, position - window could leave 32 bits
  if (cfg->window >= (long long)cfg->max_pages * cfg->page_tokens) h->cfg.window = 0;
  h->page_shift = cfg->page_tokens == 16 ? 4 : cfg->page_tokens == 32 ? 5 : cfg->page_tokens == 64 ? 6 : 7;
  rc = allocate(h);
  if (rc != FT_OK) {
    free_all(h);
    delete h;
    return rc;
  }
  *out = h;
  return FT_OK;
}

ft_status_t ft_attn_destroy(ft_attn_t *h) {
  if (!h) return FT_OK;
  DeviceScope dev(h->cfg.device);
  cudaError_t e = cudaDeviceSynchronize();
  free_all(h);
  delete h;
  FA_CUDA(e);
  return FT_OK;
}

ft_status_t ft_attn_slots(ft_attn_t *h, int n_req, int T, int max_new, const int32_t *new_len, const int32_t *ctx_len,
                          int32_t *table, int64_t table_stride, int32_t *free_pages, const int32_t *n_free,
                          int32_t *q_start, int32_t *kv_len, int32_t *n_free_out, int32_t *admitted, int32_t *position,
                          int32_t *slot, void *stream) {
  if (!h || !step_ok(h, n_req, T, max_new)) return FT_ERR_INVALID_ARG;
  if (!free_pages || !n_free || !q_start || !n_free_out || (n_req > 0 && (!new_len || !ctx_len || !table || !kv_len || !admitted)) ||
      (T > 0 && (!position || !slot)))
    return FT_ERR_INVALID_ARG;
  if (table_stride < h->cfg.max_pages || n_free_out == n_free || (n_req > 0 && kv_len == ctx_len)) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->cfg.device);
  FA_CUDA(dev.err);
  AttnSlotsArgs a;
  memset(&a, 0, sizeof(a));
  a.n_req = n_req; a.T = T; a.max_new = max_new;
  a.new_len = new_len; a.ctx_len = ctx_len; a.table = table; a.table_stride = table_stride;
  a.free_pages = free_pages; a.n_free = n_free; a.q_start = q_start; a.kv_len = kv_len; a.n_free_out = n_free_out;
  a.admitted = admitted; a.position = position; a.slot = slot;
  return launch_slots(h, a, static_cast<cudaStream_t>(stream));
}

ft_status_t ft_attn_plan(ft_attn_t *h, int n_req, int T, int max_new, const int32_t *q_start, const int32_t *kv_len,
                         void *stream) {
  if (!h || !step_ok(h, n_req, T, max_new) || (n_req > 0 && (!q_start || !kv_len))) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->cfg.device);
  FA_CUDA(dev.err);
  AttnSlotsArgs a;
  memset(&a, 0, sizeof(a));
  a.n_req = n_req; a.T = T; a.max_new = max_new; a.own_tables = 1;
  a.q_start_in = q_start; a.kv_len_in = kv_len;
  return launch_slots(h, a, static_cast<cudaStream_t>(stream));
}

ft_status_t ft_attn_qk_rope(ft_attn_t *h, int T, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                            const void *v, int64_t v_stride, const void *w_q, const void *w_k, float eps,
                            const float *cos_sin, int max_pos, int rot_dim, int interleaved, const int32_t *position,
                            const int32_t *slot, void *q_out, int64_t q_out_stride, void *kv_cache, void *stream) {
  if (!h || T < 0 || T > h->cfg.max_tokens) return FT_ERR_INVALID_ARG;
  if (T == 0) return FT_OK;
  const ft_attn_config_t &c = h->cfg;
  const int D = c.head_dim;
  if (!q || !k || !v || !q_out || !kv_cache || !position || !slot) return FT_ERR_INVALID_ARG;
  if (rot_dim < 0 || rot_dim > D || rot_dim % 8 || (rot_dim > 0 && (!cos_sin || max_pos < 1))) return FT_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)w_q | (uintptr_t)w_k | (uintptr_t)q_out) & 7) return FT_ERR_INVALID_ARG;
  if (((uintptr_t)kv_cache | (uintptr_t)cos_sin) & 15) return FT_ERR_INVALID_ARG;
  if (q_stride < (int64_t)c.n_q_heads * D || q_out_stride < (int64_t)c.n_q_heads * D || k_stride < (int64_t)c.n_kv_heads * D ||
      v_stride < (int64_t)c.n_kv_heads * D || ((q_stride | k_stride | v_stride | q_out_stride) & 3))
    return FT_ERR_INVALID_ARG;
  if (!(eps >= 0.f)) return FT_ERR_INVALID_ARG;
  DeviceScope dev(c.device);
  FA_CUDA(dev.err);
  RopeArgs a;
  a.T = T; a.n_q = c.n_q_heads; a.n_kv = c.n_kv_heads; a.page_shift = h->page_shift; a.n_pages = c.n_pages;
  a.rot_half = rot_dim / 2; a.interleaved = interleaved ? 1 : 0; a.max_pos = max_pos;
  a.q = static_cast<const uint16_t *>(q); a.k = static_cast<const uint16_t *>(k); a.v = static_cast<const uint16_t *>(v);
  a.w_q = static_cast<const uint16_t *>(w_q); a.w_k = static_cast<const uint16_t *>(w_k);
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = q_out_stride;
  a.eps = eps; a.cos_sin = cos_sin; a.position = position; a.slot = slot;
  a.q_out = static_cast<uint16_t *>(q_out); a.cache = static_cast<uint16_t *>(kv_cache);
  a.status = h->status_dev;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf = c.dtype == FT_ATTN_BF16;
  // 16-byte accesses where every address and the halves of the rotated part allow them
  const bool wide = !(((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)w_q | (uintptr_t)w_k | (uintptr_t)q_out) & 15) &&
                    !((q_stride | k_stride | v_stride | q_out_stride) & 7) && rot_dim % 16 == 0;
  FA_CUDA(D == 128 ? (bf ? launch_rope<128, true>(h, a, wide, st) : launch_rope<128, false>(h, a, wide, st))
                   : (bf ? launch_rope<64, true>(h, a, wide, st) : launch_rope<64, false>(h, a, wide, st)));
  h->launches += 1;
  return FT_OK;
}

ft_status_t ft_attn_forward(ft_attn_t *h, const void *q, int64_t q_stride, const void *kv_cache, const int32_t *table,
                            int64_t table_stride, void *out, int64_t out_stride, float *lse, float scale, void *stream) {
  if (!h) return FT_ERR_INVALID_ARG;
  if (!h->planned) return FT_ERR_STATE;
  if (h->n_req == 0 || h->T == 0 || h->max_new == 0) return FT_OK;
  const ft_attn_config_t &c = h->cfg;
  const int D = c.head_dim;
  if (!q || !kv_cache || !table || !out) return FT_ERR_INVALID_ARG;
  if (((uintptr_t)q | (uintptr_t)kv_cache | (uintptr_t)out) & 15) return FT_ERR_INVALID_ARG;
  if (q_stride > (1 << 23) || out_stride > (1 << 23)) return FT_ERR_INVALID_ARG;
  if (q_stride < (int64_t)c.n_q_heads * D || out_stride < (int64_t)c.n_q_heads * D || ((q_stride | out_stride) & 7) ||
      table_stride < c.max_pages || !(scale == scale))
    return FT_ERR_INVALID_ARG;
  DeviceScope dev(c.device);
  FA_CUDA(dev.err);
  AttnFwdArgs a;
  a.w = h->work; a.n_q = c.n_q_heads; a.n_kv = c.n_kv_heads; a.group = h->geom.group; a.page_shift = h->page_shift;
  a.n_pages = c.n_pages; a.window = c.window;
  a.q = static_cast<const uint16_t *>(q); a.cache = static_cast<const uint16_t *>(kv_cache);
  a.q_stride = q_stride; a.out_stride = out_stride; a.table_stride = table_stride; a.table = table;
  a.out = static_cast<uint16_t *>(out); a.lse = lse; a.status = h->status_dev;
  a.scale_log2 = scale * 1.44269504088896f;
  if (a.scale_log2 == 0.f) a.scale_log2 = 1e-30f;   // equal weights without 0 * infinity in masked places
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf = c.dtype == FT_ATTN_BF16;
  if (D == 128) return bf ? launch_forward<128, true>(h, a, kv_cache, st) : launch_forward<128, false>(h, a, kv_cache, st);
  return bf ? launch_forward<64, true>(h, a, kv_cache, st) : launch_forward<64, false>(h, a, kv_cache, st);
}

ft_status_t ft_attn_sync_status(ft_attn_t *h) {
  if (!h) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->cfg.device);
  FA_CUDA(dev.err);
  FA_CUDA(cudaDeviceSynchronize());
  uint32_t st = 0;
  FA_CUDA(cudaMemcpy(&st, h->status_dev, sizeof(st), cudaMemcpyDeviceToHost));
  if (!st) return FT_OK;
  FA_CUDA(cudaMemset(h->status_dev, 0, sizeof(st)));
  FA_CUDA(cudaDeviceSynchronize());
  if (st & kStatTimeout) {      // a call that gave up may have left arrivals behind
    FA_CUDA(cudaMemset(h->arrive, 0, h->arrive_bytes));
    FA_CUDA(cudaDeviceSynchronize());
    return FT_ERR_TIMEOUT;
  }
  return (st & kStatBadIndex) ? FT_ERR_INVALID_ARG : FT_ERR_CUDA;
}

ft_status_t ft_attn_debug_inject(ft_attn_t *h, uint32_t withhold_mask, uint32_t wait_polls) {
  if (!h) return FT_ERR_INVALID_ARG;
  DeviceScope dev(h->cfg.device);
  FA_CUDA(dev.err);
  const uint32_t polls = wait_polls ? wait_polls : kDefaultWaitPolls;
  FA_CUDA(cudaDeviceSynchronize());
  FA_CUDA(cudaMemcpyToSymbol(g_debug_withhold, &withhold_mask, sizeof(withhold_mask)));
  FA_CUDA(cudaMemcpyToSymbol(g_wait_polls, &polls, sizeof(polls)));
  FA_CUDA(cudaDeviceSynchronize());
  return FT_OK;
}

ft_status_t ft_attn_launch_count(ft_attn_t *h, uint64_t *out) {
  if (!h || !out) return FT_ERR_INVALID_ARG;
  *out = h->launches;
  return FT_OK;
}

}  // extern "C"
