// Bookkeeping of a serving step: page allocation and release, block tables, positions and cache slots of the new tokens,
// and the work partition of the attention kernels, from the requests' lengths.
//
// With n_r new tokens, c_r cached ones and p tokens a page: held_r = ceil(c_r/p), need_r = ceil((c_r+n_r)/p) - held_r.
// All of it follows from three prefix sums over the requests (tokens and released pages; needed pages; attention work),
// one request per thread, so every block computes them for itself from 8 bytes a request and no block waits for
// another.  Block 0 writes what belongs to requests and the work partition, the other blocks the per-token arrays, the
// released and the new pages.  Reads are of the step's old state alone: the stack below n_free, columns below held_r;
// writes are of the stack from n_free up and columns from held_r up.
// Bound: latency (a few KB): launch, the lengths, the scans, then block 0's partition.  Measured, launches back to back: 3.5 us for
// 8 requests, 5.5 us for 250 mixed ones with 63 chunks among them or not.
#pragma once
#include "async.cuh"

namespace ftmoe {

constexpr int kAttnMaxRequests = 1024;
constexpr int kUnitCache = 2048;       // entries whose positions a work partition keeps in shared memory while it is made
constexpr int kAttnMaxGrid = 512;      // CTAs a work partition can address
constexpr int kDecRows = 16;           // query rows (tokens x heads of a group) the streaming kernel takes
constexpr int kDecKeys = 64;           // keys of one of its work units
constexpr int kTileRows = 128;         // query rows of one tcgen05 tile; a work item of the tiled kernel is two of them
constexpr int kTileKeys = 128;         // keys of one of its work units
constexpr int kDecCost = 1, kTileCost = 3;   // of a work item besides its blocks, in units

// One entry of the streaming list (a request with few rows) or of the tile list (up to 2 x 128 rows of a request).
// The units of an entry are its key blocks b0 .. b0+nb-1 for each key/value head.  What an item costs besides its blocks
// (queries, first scores, results) counts as `cost` units in front of them, so block b of head h stands at
// unit0*Hkv + h*(nb + cost) + cost + (b - b0), unit0 being the sum of nb + cost of the entries before.  CTA i evaluates the
// blocks that stand at [i*quota, (i+1)*quota).
struct __align__(16) AttnEntry {
  int32_t req, tok0, n_tok, pos0;   // request, first packed row, rows, position of the first row
  int32_t b0, nb, unit0, pad;
};
// Where a CTA's share begins: the first block at or behind its position, and that entry.
struct __align__(16) AttnStart {
  int32_t k, head, blk, pad;
  AttnEntry e;
};
struct __align__(16) AttnPlanHdr {
  int32_t n_req, T;
  int32_t n_dec, dec_units, dec_quota;      // (units times key/value heads)
  int32_t n_tile, tile_units, tile_quota;
};
struct AttnWork {   // device pointers of a handle's work partition
  AttnPlanHdr *hdr;
  AttnEntry *dec, *tile;
  AttnStart *dec_start, *tile_start;        // per CTA
};
struct AttnGeom {
  int32_t group, n_kv, window, tile_tokens;   // tile_tokens: rows of a request per work item of the tiled kernel
  int32_t dec_grid, dec_min_quota, tile_grid, tile_min_quota;
  int32_t tile_cap;                           // entries the tile list holds
};

struct AttnSlotsArgs {
  int32_t n_req, T, max_new, n_pages, max_pages, page_shift, own_tables;
  const int32_t *new_len, *ctx_len, *n_free;
  int32_t *table;
  long long table_stride;
  int32_t *free_pages, *q_start, *kv_len, *n_free_out, *admitted, *position, *slot;
  const int32_t *q_start_in, *kv_len_in;      // own_tables: the lengths come from these two instead
  AttnWork w;
  AttnGeom g;
  uint32_t *status;
};

// Inclusive prefix sum over the block of two packed 32-bit counts; *total gets the sum.
template <int NT>
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long *s_warp,
                                                         unsigned long long *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();             // s_warp may still be read from the scan before
  if (lane == 31) s_warp[warp] = v;
  __syncthreads();
  unsigned long long base = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) {
    const unsigned long long s = s_warp[i];
    if (i < warp) base += s;
    sum += s;
  }
  *total = sum;
  return v + base;
}
__device__ __forceinline__ unsigned long long pack2(uint32_t lo, uint32_t hi) {
  return (unsigned long long)lo | ((unsigned long long)hi << 32);
}

// Number of entries of the ascending array a[0..n) that are <= v.
__device__ __forceinline__ int count_le(const int32_t *a, int n, int v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= v) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// The first block at or behind position u in a list of `n` entries, whose unit0 are also in `units` as far as that goes (null:
// too many).
__device__ __forceinline__ AttnStart locate_unit(const AttnEntry *e, const int32_t *units, int n, int n_kv, int cost, int u) {
  int lo = 0, hi = n;                     // largest entry with unit0 * n_kv <= u
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((units ? units[mid] : e[mid].unit0) * n_kv <= u) lo = mid; else hi = mid;
  }
  AttnStart s;
  s.e = e[lo];
  const int rest = u - s.e.unit0 * n_kv, w = s.e.nb + cost;
  s.k = lo; s.head = rest / w; s.blk = max(0, rest % w - cost); s.pad = 0;
  return s;
}

// A record of whole 16-byte words from L2.
template <typename T>
__device__ __forceinline__ void load_l2(T &out, const T *p) {
  static_assert(sizeof(T) % 16 == 0, "whole words");
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 16; ++i) {
    const int4 v = __ldcg(reinterpret_cast<const int4 *>(p) + i);
    memcpy(reinterpret_cast<char *>(&out) + 16 * i, &v, 16);
  }
}

// A CTA's walk over its share: `take` blocks from block `blk` of (entry k, head).
struct WorkWalk {
  int k, head, blk, take, u;              // u: position of the item's first block
  AttnEntry e, ahead;                     // entry k and, with its last head, the next one
  __device__ __forceinline__ void start(const AttnStart &s) { k = s.k; head = s.head; blk = s.blk; e = s.e; }
  // false: the share is done
  __device__ __forceinline__ bool load(int n, int n_kv, int cost, int end) {
    if (k >= n) return false;
    u = e.unit0 * n_kv + head * (e.nb + cost) + cost;
    take = min(e.nb, end - u) - blk;
    return take > 0;
  }
  // to be called for every item, before `next`: early, for the load to be over by then
  __device__ __forceinline__ void fetch(const AttnEntry *list, int n, int n_kv, int end) {
    if (head == n_kv - 1 && k + 1 < n && u + e.nb < end) load_l2(ahead, list + k + 1);
  }
  // (a share that ends with the item needs no other entry: `load` finds nothing left of this one)
  __device__ __forceinline__ void next(int n_kv, int end) {
    if (u + e.nb >= end) { blk = e.nb; return; }
    blk = 0;
    if (++head == n_kv) { head = 0; ++k; e = ahead; }
  }
};

// Key blocks of `keys` keys that the rows at positions pos0 .. pos0+n-1 attend to: first block and count (at least one
// block, so that rows that attend to nothing are still written).
__device__ __forceinline__ void block_range(int pos0, int n, int window, int keys, int *b0, int *nb) {
  const int hi = max(0, pos0 + n);
  const int lo = window > 0 ? min(hi, max(0, pos0 - window + 1)) : 0;
  *b0 = lo / keys;
  *nb = max(1, (hi + keys - 1) / keys - *b0);
}

// The work partition, by one block; thread r owns request r (n rows from packed row tok0, kv cached tokens).
template <int NT>
__device__ void build_work(const AttnSlotsArgs &a, int n, int tok0, int kv, unsigned long long *s_warp, int32_t *s_tile,
                           const int32_t *s_q, const int32_t *s_kv, int32_t *s_dec, int32_t *s_unit) {
  const int tid = threadIdx.x;
  const AttnGeom &g = a.g;
  const bool dec = n > 0 && n * g.group <= kDecRows;
  int b0 = 0, nb = 0;
  if (dec) block_range(kv - n, n, g.window, kDecKeys, &b0, &nb);
  unsigned long long tot;
  const int w = dec ? nb + kDecCost : 0;
  const unsigned long long inc = block_scan<NT>(pack2(dec ? 1u : 0u, (uint32_t)w), s_warp, &tot);
  const int n_dec = (int)(uint32_t)tot, dec_units = (int)(tot >> 32) * g.n_kv;
  if (dec) {
    AttnEntry e;
    e.req = tid; e.tok0 = tok0; e.n_tok = n; e.pos0 = kv - n; e.b0 = b0; e.nb = nb;
    e.unit0 = (int)(inc >> 32) - w; e.pad = 0;
    a.w.dec[(uint32_t)inc - 1] = e;
    s_dec[(uint32_t)inc - 1] = e.unit0;
  }
  const int tiles = (n > 0 && !dec) ? (n + g.tile_tokens - 1) / g.tile_tokens : 0;
  const unsigned long long tinc = block_scan<NT>((unsigned long long)tiles, s_warp, &tot);
  const int n_tile = min((int)tot, g.tile_cap);
  if (tid < a.n_req) s_tile[tid] = (int)tinc;      // inclusive
  __syncthreads();
  int carry = 0;
  for (int base = 0; base < n_tile; base += NT) {
    const int t = base + tid;
    AttnEntry e;
    if (t < n_tile) {
      const int r = count_le(s_tile, a.n_req, t);
      const int i = t - (r ? s_tile[r - 1] : 0), nr = s_q[r + 1] - s_q[r], first = i * g.tile_tokens;
      e.req = r; e.tok0 = s_q[r] + first; e.n_tok = min(g.tile_tokens, nr - first); e.pos0 = s_kv[r] - nr + first; e.pad = 0;
      block_range(e.pos0, e.n_tok, g.window, kTileKeys, &e.b0, &e.nb);
    }
    const int w = t < n_tile ? e.nb + kTileCost : 0;
    const unsigned long long ui = block_scan<NT>((unsigned long long)w, s_warp, &tot);
    if (t < n_tile) {
      e.unit0 = carry + (int)ui - w;
      a.w.tile[t] = e;
      if (t < kUnitCache) s_unit[t] = e.unit0;
    }
    carry += (int)tot;
  }
  const int tile_units = carry * g.n_kv;
  const int dec_quota = max((dec_units + g.dec_grid - 1) / g.dec_grid, g.dec_min_quota);
  const int tile_quota = max((tile_units + g.tile_grid - 1) / g.tile_grid, g.tile_min_quota);
  if (tid == 0) {
    AttnPlanHdr h;
    h.n_req = a.n_req; h.T = a.T;
    h.n_dec = n_dec; h.dec_units = dec_units; h.dec_quota = dec_quota;
    h.n_tile = n_tile; h.tile_units = tile_units; h.tile_quota = tile_quota;
    *a.w.hdr = h;
  }
  __syncthreads();
  for (int c = tid; c < g.dec_grid; c += NT)
    if ((long long)c * dec_quota < dec_units) a.w.dec_start[c] = locate_unit(a.w.dec, s_dec, n_dec, g.n_kv, kDecCost, c * dec_quota);
  for (int c = tid; c < g.tile_grid; c += NT)
    if ((long long)c * tile_quota < tile_units) a.w.tile_start[c] = locate_unit(a.w.tile, n_tile <= kUnitCache ? s_unit : nullptr, n_tile, g.n_kv, kTileCost, c * tile_quota);
}

// NT >= n_req: 256 threads for up to 256 requests, 1024 above.
template <int NT>
__global__ void __launch_bounds__(NT) attn_slots_kernel(const AttnSlotsArgs a) {
  __shared__ unsigned long long s_warp[NT / 32];
  __shared__ int32_t s_q[NT + 1], s_ctx[NT], s_held[NT], s_freed[NT], s_need[NT], s_kv[NT], s_adm[NT], s_unit[kUnitCache];
  const int tid = threadIdx.x, r = tid;
  unsigned long long tot;
  grid_let_next();
  grid_wait();

  if (a.own_tables) {                       // lengths given: one block, the work partition alone
    int n = 0, q0 = 0, kv = 0;
    if (r < a.n_req) {
      q0 = a.q_start_in[r];
      const int q1 = a.q_start_in[r + 1];
      kv = a.kv_len_in[r];
      n = q1 - q0;
      if (q0 < 0 || q1 > a.T || n < 0 || n > a.max_new || kv < 0 || (long long)kv > ((long long)a.max_pages << a.page_shift)) {
        atomicOr(a.status, kStatBadIndex);  // the request gets no rows
        n = 0; kv = 0;
      }
      s_q[r] = q0;
      s_kv[r] = kv;
      if (r == a.n_req - 1) s_q[a.n_req] = q1;
    }
    build_work<NT>(a, n, q0, kv, s_warp, s_freed, s_q, s_kv, s_need, s_unit);
    return;
  }

  int n = 0, ctx = 0, held = 0, freed = 0;
  bool fin = false, bad = false;
  const int p = 1 << a.page_shift;
  if (r < a.n_req) {
    n = a.new_len[r];
    ctx = a.ctx_len[r];
    fin = n < 0;
    const long long cap = (long long)a.max_pages << a.page_shift;
    if (n > a.max_new) { bad = true; n = 0; }
    if (fin) n = 0;
    if (ctx < 0 || (long long)ctx + n > cap) { bad = true; if (ctx < 0 || ctx > cap) ctx = 0; }
    held = (int)(((long long)ctx + p - 1) >> a.page_shift);
    if (fin && held > a.n_pages) bad = true;         // (nor may the sum of the requests leave 32 bits)
    freed = fin && !bad ? held : 0;
  }
  const unsigned long long inc = block_scan<NT>(pack2((uint32_t)n, (uint32_t)freed), s_warp, &tot);
  const int q1 = (int)(uint32_t)inc, q0 = q1 - n, f1 = (int)(inc >> 32);
  const long long freed_sum = (long long)(tot >> 32);
  if (q1 > a.T) bad = true;
  const int need = (fin || bad) ? 0 : (int)(((long long)ctx + n + p - 1) >> a.page_shift) - held;
  const int need1 = (int)block_scan<NT>((unsigned long long)need, s_warp, &tot);
  int n_free = *a.n_free;
  if (n_free < 0 || n_free > a.n_pages) { bad = true; n_free = 0; }
  if (n_free + freed_sum > a.n_pages) bad = true;      // more pages than there are: nothing is released or taken
  const int total_freed = n_free + freed_sum > a.n_pages ? 0 : (int)freed_sum, avail = n_free + total_freed;
  const bool adm = r < a.n_req && !fin && !bad && (need == 0 || need1 <= avail);
  // taken pages: the admitted requests that need any are a prefix of those that need any
  unsigned long long taken_sum;
  block_scan<NT>((unsigned long long)(adm ? need : 0), s_warp, &taken_sum);
  const int taken = (int)taken_sum;
  const int kv = fin ? 0 : (adm ? ctx + n : ctx);
  s_q[r + 1] = q1;
  if (r == 0) s_q[0] = 0;
  s_ctx[r] = ctx; s_held[r] = held; s_freed[r] = f1; s_need[r] = need1 - need; s_kv[r] = adm ? kv : 0; s_adm[r] = adm;
  __syncthreads();

  if (blockIdx.x == 0) {
    if (bad && (r < a.n_req || r == 0)) atomicOr(a.status, kStatBadIndex);
    if (r < a.n_req) {
      a.kv_len[r] = kv;
      a.admitted[r] = adm ? 1 : 0;
      a.q_start[r + 1] = q1;
    }
    if (r == 0) {
      a.q_start[0] = 0;
      *a.n_free_out = avail - taken;
    }
    // (a request that is not admitted keeps its rows, which attend to nothing; rows past T do not exist)
    build_work<NT>(a, q1 > a.T ? 0 : n, q0, adm ? kv : 0, s_warp, s_freed, s_q, s_kv, s_need, s_unit);
    return;
  }

  // entry i of the stack after the releases
  auto stack_at = [&](int i) -> int {
    if (i < n_free) return a.free_pages[i];
    const int j = i - n_free, rr = count_le(s_freed, a.n_req, j);
    return a.table[rr * a.table_stride + (j - (rr ? s_freed[rr - 1] : 0))];
  };
  const int step = (gridDim.x - 1) * NT, first = (blockIdx.x - 1) * NT + tid;
  for (int t = first; t < a.T; t += step) {
    int pos = -1, slot = -1;
    const int rr = count_le(s_q, a.n_req + 1, t) - 1;       // last request whose rows start at or before t
    if (rr < a.n_req && s_adm[rr]) {
      pos = s_ctx[rr] + t - s_q[rr];
      const int b = pos >> a.page_shift;
      const int page = b < s_held[rr] ? a.table[rr * a.table_stride + b]
                                      : stack_at(avail - 1 - s_need[rr] - (b - s_held[rr]));
      if ((uint32_t)page < (uint32_t)a.n_pages) slot = (page << a.page_shift) + (pos & (p - 1));
      else atomicOr(a.status, kStatBadIndex);
    }
    a.position[t] = pos;
    a.slot[t] = slot;
  }
  for (int j = first; j < total_freed; j += step) {
    const int page = stack_at(n_free + j);
    if (n_free + j < a.n_pages) a.free_pages[n_free + j] = page;
  }
  for (int j = first; j < taken; j += step) {
    const int rr = count_le(s_need, a.n_req, j) - 1;        // last request whose pages start at or before j
    a.table[rr * a.table_stride + s_held[rr] + (j - s_need[rr])] = stack_at(avail - 1 - j);
  }
}

}  // namespace ftmoe
