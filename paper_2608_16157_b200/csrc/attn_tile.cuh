// Attention of requests with many query rows (chunks, whole prompts, wide groups) over the paged cache, on the
// 5th-generation tensor cores.  4*D flops per (query head, key) pair: bound by the tensor pipe and, at the same rate, by the
// exponentials (128 x 128 of either take the tensor pipe 2 x 512 and the special-function units 1024 clocks at D = 128).
//
// A work item is up to 256 query rows (tokens x heads of the group: the keys of a head are read once for all of them) of a
// request, as two tiles of 128 rows; its key blocks of 128 are its work units, cut into equal shares, one CTA per SM (the
// work partition of attn_plan.cuh).  An item with at most 128 rows (short chunks, drafts, single tokens of wide groups: bound by
// HBM) uses both tiles on the same rows, one for the even and one for the odd blocks, and joins them at its end.  Roles of the warps:
//   warp 9     brings Q (4-D TMA boxes: D, heads of the group, head, tokens) and the pages of K and V (128-byte swizzle)
//   warp 8     issues tcgen05.mma: S_t = Q_t K^T into tensor memory, O_t += P_t V with P_t read from there (warp 10: for the second
//              tile of an item with at most 128 rows)
//   warps 0-3, 4-7   softmax of tile 0 and 1: a thread owns a row, so maximum and sum need no exchange
// While one tile is in its softmax the tensor pipe works for the other: one warp issues for both in turn, P_t V of block j and
// then Q_t K^T of block j+1, which keeps the two out of step (two issuing warps fell into step: 4750 against 3860 clocks a
// unit).  P overwrites its scores (tensor memory: 2 x (128 + D) columns) and is handed over in two halves of 64 keys.
// No maximum is taken as a rule: a half block's weights are made with the row's present reference, and their sum tells
// whether any exceeds 2^8; only then (and in a row's first half block) the maximum is taken, O rescaled in tensor memory and the
// half repeated (the maximum is also taken where a mask is applied).  The result is the same, since weights and sum share one
// reference; 16-bit weights up to 2^8 have the same relative rounding.
// Measured, D = 128: a unit of 256 rows x 128 keys 1.88 us (items of 32 and 64 blocks, one a CTA; 3700 clocks at 1965 MHz).  A clock
// trace, of the loop before the issuing warp's steady state had one of its own: 3860 clocks, of them a tile's softmax 2700 and, behind
// it, its two products 1160; pipe and special-function units are busy 2048 each.  D = 64: 1.85 us, the same exponentials.  A prompt
// of 16384 tokens with 32 heads of 128: 1.79 - 1.87 ms in short bursts (1.2 PFLOP/s), 2.11 - 2.17 ms (1.03) in a long run under the
// power limit; of 4096: 159 - 166 us.  Two threads a row (16 softmax warps of 96 registers) made a unit 1.90 us against 1.85 in the same
// run and that prompt 2.09 ms.  168 registers a thread; 68 (D = 128) and 32 (D = 64) bytes spilled.
// P is rounded to the values' type for the second product; scores, maxima, sums and O stay in 32 bits.
#pragma once
#include <type_traits>

#include "attn_stream.cuh"

namespace ftmoe {

constexpr int kTileThreads = 352, kTileHalf = 64;    // keys of half a block
template <int D> struct TileCfg {
  static constexpr int kChunks = D / 64;                    // 64-element pieces of D: 128 rows x 128 bytes each
  static constexpr int kTile = 128 * D * 2;                 // bytes of 128 rows of Q, K or V
  static constexpr int kStages = D == 128 ? 4 : 8;          // ring of K and V tiles
  static constexpr int kStage = 8 * 4096;                   // results on their way out
  static constexpr int kBars = 2 * kStages + 2 + 14;         // (one place of them free)
  static constexpr int kSmem = 1024 + 2 * kTile + kStages * kTile + kStage + kBars * 8 + 64;
  static constexpr int kPart = 128 * (D + 2);               // floats of one tile's partial result: m[128], l[128], O[D][128]
};
static_assert(TileCfg<128>::kSmem <= 232448 && TileCfg<64>::kSmem <= 232448, "shared memory of a CTA");

__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a_tmem), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
// Whether the phase is complete, without waiting for it.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// A value all lanes hold, in a uniform register.
__device__ __forceinline__ int uniform(int v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *tm, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(tm), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// The half blocks a tile takes of the item's range [h0, h1): all, or with `keys` those of the blocks of its parity.
__device__ __forceinline__ int first_half(bool keys, int t, int h0) { return keys && ((h0 >> 1) & 1) != t ? 2 * ((h0 >> 1) + 1) : h0; }
__device__ __forceinline__ int next_half(bool keys, int h) { return keys && (h & 1) ? h + 3 : h + 1; }

__device__ __forceinline__ int count_halves(bool keys, int t, int h0, int h1) {
  auto below = [t](int h) { return 2 * (h >> 2) + max(0, min(2, (h & 3) - 2 * t)); };     // of the blocks of parity t
  return keys ? max(0, below(h1) - below(h0)) : h1 - h0;
}

// What a tile of a work item covers.
struct TileSpan {
  int n, lo, hi, pos0;       // rows' tokens, keys [lo, hi) some row attends to, position of the first token
  // half blocks [first, last) that a part of the item's blocks [kb0, kb1) holds for the tile
  __device__ __forceinline__ void halves(int kb0, int kb1, int *first, int *last) const {
    *first = max(2 * kb0, lo / kTileHalf);
    *last = n > 0 ? min(2 * kb1, (hi + kTileHalf - 1) / kTileHalf) : 0;
    if (*last < *first) *last = *first;
  }
};
__device__ __forceinline__ TileSpan tile_span(const AttnEntry &e, int t, int tokens, int window) {
  TileSpan s;
  s.n = min(tokens, max(0, e.n_tok - t * tokens));
  s.pos0 = e.pos0 + t * tokens;
  s.hi = max(0, s.pos0 + s.n);
  s.lo = window > 0 ? max(0, s.pos0 - window + 1) : 0;
  return s;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kTileThreads, 1)
attn_tile_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm, const AttnFwdArgs a) {
  using Cfg = TileCfg<D>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char *s_stage = smem + (2 + Cfg::kStages) * Cfg::kTile;
  uint64_t *s_bar = reinterpret_cast<uint64_t *>(s_stage + Cfg::kStage);
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(s_bar + Cfg::kBars);
  volatile int *s_abort = reinterpret_cast<volatile int *>(s_tmem + 1);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t q_smem = smem_u32(smem), ring = q_smem + 2 * Cfg::kTile, bars = smem_u32(s_bar);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (Cfg::kStages + s); };
  const uint32_t q_full = bars + 8u * (2 * Cfg::kStages), q_empty = q_full + 8;
  auto s_full = [&](int t) { return q_full + 16 + 8u * t; };
  const uint32_t handed = q_full + 32;
  auto p_full = [&](int t, uint32_t buf) { return q_full + 48 + 16u * t + 8u * buf; };
  // (by the parity of the half's number: a waiter knows the one before the last on each to be complete)
  auto pv_done = [&](int t, uint32_t i) { return q_full + 80 + 16u * t + 8u * (i & 1u); };
  auto o_empty = [&](int t) { return q_full + 112 + 8u * t; };

  const uint32_t limit = g_wait_polls;
  grid_let_next();
  if (tid == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 2);
    mbar_init(handed, 2);
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full(t), 1);
      for (int i = 0; i < 2; ++i) { mbar_init(p_full(t, i), 4); mbar_init(pv_done(t, i), 1); }
      mbar_init(o_empty(t), 4);
    }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  grid_wait();
  AttnPlanHdr hdr;
  AttnStart st;                                        // (stale beyond the shares in use: not looked at)
  load_l2(hdr, a.w.hdr);
  load_l2(st, a.w.tile_start + blockIdx.x);
  const long long u_first = (long long)blockIdx.x * hdr.tile_quota;
  if (u_first >= hdr.tile_units) {
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    return;
  }
  const int u_end = (int)min(u_first + hdr.tile_quota, (long long)hdr.tile_units);
  const uint32_t tm_s = tmem, tm_o = tmem + 256;             // S_t (and P_t) at 128 t, O_t at 256 + D t
  const int tokens = kTileRows / a.group;                    // tokens of a tile
  WorkWalk w;
  w.start(st);

  if (warp >= 8) {
    w.k = uniform(w.k); w.head = uniform(w.head); w.blk = uniform(w.blk);
    uint32_t rs = 0, rph = 0;                 // next entry of the ring and its phase
    auto step = [](uint32_t &s, uint32_t &ph) { if (++s == Cfg::kStages) { s = 0; ph ^= 1u; } };
    uint32_t items = 0;
    if (warp == 9) {
      // ------------------------------ loads ------------------------------
      const bool hook = g_debug_withhold & kWithholdAttnTile;
      const int page_tokens = 1 << a.page_shift;
      const int box_shift = min(a.page_shift, 6), box_rows = 1 << box_shift, boxes = kTileKeys >> box_shift;
      for (; w.load(hdr.n_tile, a.n_kv, kTileCost, u_end) && !*s_abort; w.next(a.n_kv, u_end)) {
        w.fetch(a.w.tile, hdr.n_tile, a.n_kv, u_end);
        AttnEntry e = w.e;
        e.n_tok = uniform(e.n_tok); e.pos0 = uniform(e.pos0); e.b0 = uniform(e.b0); e.tok0 = uniform(e.tok0);
        const int take = uniform(w.take), blk = w.blk, head = w.head;
        const int hi = max(0, e.pos0 + e.n_tok), lo = a.window > 0 ? max(0, e.pos0 - a.window + 1) : 0;
        const int32_t *row = a.table + (long long)e.req * a.table_stride;
        // lane i holds the page of box i of a block; boxes first .. last-1 of a block are loaded
        auto page_of = [&](int b) -> int {
          const int key = (e.b0 + b) * kTileKeys + lane * box_rows;
          return lane < boxes && key < hi && key + box_rows > lo ? __ldcg(row + (key >> a.page_shift)) : 0;
        };
        auto checked = [&](int page) -> int {              // never followed: a box beyond the pool, which is zeros
          if (__builtin_expect((uint32_t)page >= (uint32_t)a.n_pages, 0)) {
            atomicOr(a.status, kStatBadIndex);
            page = a.n_pages;
          }
          return page;
        };
        const bool keys = e.n_tok <= tokens;
        bool withhold = hook && w.k == 0 && head == 0 && blk == 0;
        const int lag = keys ? 2 : 1;             // V of a block comes behind K of the `lag`-th block after it: the order of use
        int page = page_of(blk), page1 = 0, page2 = 0;
        wait_phase(q_empty, (items & 1u) ^ 1u, limit, s_abort, a.status);
        if (*s_abort) break;
        ++items;
        if (elect_one()) {
          const int n_tiles = keys ? 1 : 2;
          mbar_expect_tx(q_full, (uint32_t)(n_tiles * Cfg::kChunks * tokens * a.group * 128));
          for (int t = 0; t < n_tiles; ++t)
            for (int c = 0; c < Cfg::kChunks; ++c)
              tma_load_4d(q_smem + t * Cfg::kTile + c * 16384, &tm_q, c * 64, 0, head, e.tok0 + t * tokens, q_full);
        }
        __syncwarp();
        auto load_tile = [&](int b, int pages, int v) {
          wait_phase(empty_bar(rs), rph ^ 1u, limit, s_abort, a.status);
          if (*s_abort) return;
          const int key0 = (e.b0 + b) * kTileKeys;
          const int first = max(0, lo - key0) >> box_shift, last = min(boxes, (max(0, hi - key0) + box_rows - 1) >> box_shift);
          if (elect_one()) mbar_expect_tx(full_bar(rs), (uint32_t)(max(0, last - first) * box_rows * D * 2));
          __syncwarp();
          const uint32_t dst = ring + rs * Cfg::kTile;
          const bool skip = withhold;                      // test hook: the tile's copies never come
          withhold = false;
          for (int i = first; i < last && !skip; ++i) {
            const int z = (__shfl_sync(0xffffffffu, pages, i) * 2 + v) * a.n_kv + head, y = (key0 + i * box_rows) & (page_tokens - 1);
            if (elect_one()) {
#pragma unroll
              for (int c = 0; c < Cfg::kChunks; ++c)
                tma_load_3d(dst + c * 16384 + i * box_rows * 128, &tm, c * 64, y, z, full_bar(rs));
            }
            __syncwarp();
          }
          step(rs, rph);
        };
#pragma unroll 1
        for (int i = 0; i < take + lag && !*s_abort; ++i) {
          const int next = i + 1 < take ? page_of(blk + i + 1) : 0;     // (used, and waited for, a step later)
          page = checked(page);
          if (i >= lag) load_tile(blk + i - lag, keys ? page2 : page1, 1);
          if (i < take) load_tile(blk + i, page, 0);
          page2 = page1; page1 = page; page = next;
        }
      }
    } else {
      // ------------------------------ tensor core (warps 8 and 10) ------------------------------
      const int mine = warp == 8 ? 0 : 1;
      constexpr uint32_t type = BF16 ? (1u << 7) | (1u << 10) : 0u;
      constexpr uint32_t idesc_qk = (1u << 4) | type | ((uint32_t)(kTileKeys >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
      constexpr uint32_t idesc_pv = (1u << 4) | type | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
      // (little code, the same for both tiles and both halves: what this warp runs is not in the instruction cache for long
      // beside the softmax warps)
      uint32_t cp0 = 0, cp1 = 0, no0 = 0, no1 = 0; // halves of weights consumed, items so far
      uint32_t switches = 0;
      bool issued = false, keys_before = false;
      const uint64_t dq = umma_desc(q_smem, 16, 1024);
      for (; w.load(hdr.n_tile, a.n_kv, kTileCost, u_end); w.next(a.n_kv, u_end)) {
        w.fetch(a.w.tile, hdr.n_tile, a.n_kv, u_end);
        AttnEntry e = w.e;
        e.n_tok = uniform(e.n_tok); e.pos0 = uniform(e.pos0); e.b0 = uniform(e.b0);
        const int take = uniform(w.take), kb0 = e.b0 + w.blk;
        const int hi = max(0, e.pos0 + e.n_tok), lo = a.window > 0 ? max(0, e.pos0 - a.window + 1) : 0;
        const bool keys = e.n_tok <= tokens;
        const int lag = keys ? 2 : 1;
        int h00, h01, h10, h11;
        tile_span(e, 0, tokens, a.window).halves(kb0, kb0 + take, &h00, &h01);
        tile_span(e, keys ? 0 : 1, tokens, a.window).halves(kb0, kb0 + take, &h10, &h11);
        h00 = first_half(keys, 0, h00);
        h10 = first_half(keys, 1, h10);
        // steps [f0, f1): both tiles use all of blocks j - 1 and j, the first half of neither among them
        const int f0 = max(1, ((max(h00, h10) + 2) >> 1) + 1 - kb0), f1 = keys ? 0 : min(take, (min(h01, h11) >> 1) - kb0);
        const uint32_t base0 = cp0, base1 = cp1;
        if (items > 0 && keys != keys_before) {
          // tile 1 changes hands between the two warps, whose instructions are not ordered: both wait until all of both are
          // complete (a commit is for products the thread has issued; without any, it only says so)
          if (elect_one()) { if (issued) umma_commit(handed); else mbar_arrive(handed); }
          __syncwarp();
          wait_phase(handed, switches & 1u, limit, s_abort, a.status);
          ++switches;
        }
        keys_before = keys;
        wait_phase(q_full, items & 1u, limit, s_abort, a.status);
        ++items;
        bool gave_q = false;
        if (!keys && mine == 1) {                             // both tiles are the other warp's
          const uint32_t to = rs + 2 * take;
          rph ^= (to / Cfg::kStages) & 1u;
          rs = to % Cfg::kStages;
        } else
        // step j: P V of block j - lag, Q K^T of block j; the ring holds V and K in this order
#pragma unroll 1
        for (int j = 0; j < take + lag; ++j) {
          if (j == f0 && f0 < f1) {
            // Steps in which both tiles use every half of both blocks.  What bounds a long prompt is this warp's own time (the
            // scalar code around the 32 products of a step), so it holds nothing else, and the ring's next two tiles are looked for
            // where the warp would wait for weights.  Looked for only: waiting there holds this step's last products back when
            // the tiles come late (pages of 16: 515 tokens behind 7000 113 us against 102).
            const uint32_t b0 = cp0 & 1u, b1 = cp1 & 1u;
            const uint32_t pa0 = p_full(0, b0), pb0 = p_full(0, b0 ^ 1u), pa1 = p_full(1, b1), pb1 = p_full(1, b1 ^ 1u);
            const uint32_t va0 = pv_done(0, b0), vb0 = pv_done(0, b0 ^ 1u), va1 = pv_done(1, b1), vb1 = pv_done(1, b1 ^ 1u);
            uint32_t xa0 = (cp0 >> 1) & 1u, xb0 = ((cp0 + 1) >> 1) & 1u, xa1 = (cp1 >> 1) & 1u, xb1 = ((cp1 + 1) >> 1) & 1u;
            uint32_t vs = rs, vph = rph;
            step(rs, rph);
            uint32_t ks = rs, kph = rph;
            step(rs, rph);
            bool ok = wait_phase(full_bar(vs), vph, limit, s_abort, a.status);
            ok = wait_phase(full_bar(ks), kph, limit, s_abort, a.status) && ok;
#pragma unroll 1
            for (; j < f1; ++j) {
              const uint64_t dv = umma_desc(ring + vs * Cfg::kTile, 16384, 1024), dk = umma_desc(ring + ks * Cfg::kTile, 16, 1024);
              const uint32_t give_v = empty_bar(vs), give_k = empty_bar(ks);
              auto pv = [&](int t, int half) {
#pragma unroll
                for (int kk = half * 4; kk < half * 4 + 4; ++kk)
                  umma_ts(tm_o + t * D, tm_s + t * 128 + kk * 8, dv + kk * (2048 >> 4), idesc_pv, 1u);
              };
              auto qk = [&](int t) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                  umma_bf16(tm_s + t * 128, dq + (t * Cfg::kTile + (kk >> 2) * 16384 + (kk & 3) * 32) / 16,
                            dk + ((kk >> 2) * 16384 + (kk & 3) * 32) / 16, idesc_qk, kk != 0 ? 1u : 0u);
              };
              ok = wait_phase(pa0, xa0, limit, s_abort, a.status) && ok;
              tc_fence_after();
              if (elect_one()) {
                if (ok) pv(0, 0);
                umma_commit(va0);
              }
              __syncwarp();
              ok = wait_phase(pb0, xb0, limit, s_abort, a.status) && ok;
              tc_fence_after();
              if (elect_one()) {
                if (ok) { pv(0, 1); }
                umma_commit(vb0);
                if (ok) { qk(0); }
                umma_commit(s_full(0));
              }
              __syncwarp();
              ok = wait_phase(pa1, xa1, limit, s_abort, a.status) && ok;
              tc_fence_after();
              if (elect_one()) {
                if (ok) pv(1, 0);
                umma_commit(va1);
              }
              __syncwarp();
              bool there = true;
              if (j + 1 < f1) {
                vs = rs; vph = rph;
                step(rs, rph);
                ks = rs; kph = rph;
                step(rs, rph);
                there = mbar_test(full_bar(vs), vph) && mbar_test(full_bar(ks), kph);
              }
              ok = wait_phase(pb1, xb1, limit, s_abort, a.status) && ok;
              tc_fence_after();
              if (elect_one()) {
                if (ok) { pv(1, 1); }
                umma_commit(vb1);
                if (ok) { qk(1); }
                umma_commit(s_full(1));
                umma_commit(give_v);
                umma_commit(give_k);
                if (j == take - 1) umma_commit(q_empty);
              }
              __syncwarp();
              if (!there) {
                ok = wait_phase(full_bar(vs), vph, limit, s_abort, a.status) && ok;
                ok = wait_phase(full_bar(ks), kph, limit, s_abort, a.status) && ok;
              }
              xa0 ^= 1u; xb0 ^= 1u; xa1 ^= 1u; xb1 ^= 1u;
            }
            cp0 += 2 * (f1 - f0);
            cp1 += 2 * (f1 - f0);
            issued = true;
            gave_q = f1 == take;
            // (j is the first step behind them)
          }
          const int kb = kb0 + j, kv = kb - lag;
          const bool has_v = j >= lag, has_k = j < take;
          bool ok = true;
          const uint32_t vs = rs, vph = rph;
          if (has_v) step(rs, rph);
          const uint32_t ks = rs, kph = rph;
          if (has_k) step(rs, rph);
          if (keys && (kb & 1) != mine) continue;
          const bool last_k = has_k && j + lag >= take;
          const uint32_t vt = ring + vs * Cfg::kTile;
          if (has_k) ok = wait_phase(full_bar(ks), kph, limit, s_abort, a.status);
          if (has_v) {
            ok = wait_phase(full_bar(vs), vph, limit, s_abort, a.status) && ok;
            const int first = kv * kTileKeys;
            if (__builtin_expect(ok && (first + kTileKeys > hi || first < lo), 0)) {
              // values no row attends to may be anything: their weight is 0, so they have to be finite
#pragma unroll 1
              for (int i = lane; i < kTileKeys * Cfg::kChunks * 8; i += 32) {
                const int r = (i >> 3) % kTileKeys, c = (i >> 3) / kTileKeys;
                if (first + r >= hi || first + r < lo)
                  asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vt + c * 16384 + r * 128 + (i & 7) * 16), "r"(0u) : "memory");
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
            }
          }
          tc_fence_after();
          const uint64_t dv = umma_desc(vt, 16384, 1024), dk = umma_desc(ring + ks * Cfg::kTile, 16, 1024);
#pragma unroll 1
          for (int t = keys ? kb & 1 : 0; t < (keys ? (kb & 1) + 1 : 2); ++t) {
            const int h0 = t ? h10 : h00, h1 = t ? h11 : h01;
            const int hb = has_v ? min(h1, 2 * kv + 2) : h0;
#pragma unroll 1
            for (int h = max(h0, 2 * kv); h < hb; ++h) {
              const uint32_t cp = t ? cp1 : cp0;
              if (h == h0) wait_phase(o_empty(t), ((t ? no1 : no0) & 1u) ^ 1u, limit, s_abort, a.status);
              ok = wait_phase(p_full(t, cp & 1u), (cp >> 1) & 1u, limit, s_abort, a.status) && ok;
              tc_fence_after();
              if (elect_one()) {
                if (ok) {
                  const uint32_t p = tm_s + t * 128 + (h & 1) * 32, o = tm_o + t * D;
                  const uint64_t d = dv + (h & 1) * (8192 >> 4);
                  umma_ts(o, p, d, idesc_pv, h == h0 ? 0u : 1u);
#pragma unroll
                  for (int kk = 1; kk < 4; ++kk) umma_ts(o, p + kk * 8, d + kk * (2048 >> 4), idesc_pv, 1u);
                }
                umma_commit(pv_done(t, cp));
              }
              __syncwarp();
              cp0 += 1 - t; cp1 += t;
            }
            if (elect_one()) {
              if (has_k && 2 * kb < h1 && 2 * kb + 2 > h0) {
                if (ok) {
                  const uint32_t ds = tm_s + t * 128;
                  const uint64_t d = dq + (keys ? 0 : t) * (Cfg::kTile >> 4);
#pragma unroll
                  for (int kk = 0; kk < D / 16; ++kk)
                    umma_bf16(ds, d + ((kk >> 2) * 16384 + (kk & 3) * 32) / 16, dk + ((kk >> 2) * 16384 + (kk & 3) * 32) / 16, idesc_qk,
                              kk != 0 ? 1u : 0u);
                }
                umma_commit(s_full(t));
              }
              if (keys || t == 1) {
                if (has_v) umma_commit(empty_bar(vs));
                if (has_k) umma_commit(empty_bar(ks));
                if (last_k) umma_commit(q_empty);
              }
            }
            __syncwarp();
          }
          gave_q = gave_q || last_k;
          issued = true;
        }
        if (!gave_q) {
          if (elect_one()) mbar_arrive(q_empty);
          __syncwarp();
        }
        cp0 = base0 + count_halves(keys, 0, h00, h01);
        cp1 = base1 + count_halves(keys, 1, h10, h11);
        no0 += h01 > h00 ? 1u : 0u;
        no1 += h11 > h10 ? 1u : 0u;
      }
    }
  } else {
    // ------------------------------ softmax ------------------------------
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t to = tm_o + t * D + lanes;
    const int tok = row / a.group, hq_in = row - tok * a.group;
    const float sl2 = fabsf(a.scale_log2);
    const bool negate = a.scale_log2 < 0.f;
    uint32_t cs = 0, cb = 0;                               // halves and blocks so far
    const uint32_t ts = tm_s + t * 128 + lanes;
    for (; w.load(hdr.n_tile, a.n_kv, kTileCost, u_end); w.next(a.n_kv, u_end)) {
      const AttnEntry &e = w.e;
      const int take = w.take, blk = w.blk, head = w.head;
      const bool keys = e.n_tok <= tokens;
      const TileSpan sp = tile_span(e, keys ? 0 : t, tokens, a.window);
      const bool valid = tok < sp.n;                       // (tok < tokens holds for rows below tokens * group)
      const bool any_row = __any_sync(0xffffffffu, valid);
      const int pos = valid ? sp.pos0 + tok : -1;
      int h0, h1;
      sp.halves(e.b0 + blk, e.b0 + blk + take, &h0, &h1);
      h0 = first_half(keys, t, h0);
      // halves in which every row of the tile attends to every key
      const int f0 = a.window > 0 ? max(h0, (sp.pos0 + sp.n - 1 - a.window + kTileHalf) / kTileHalf) : h0;
      const int f1 = min(h1, (sp.pos0 + 1) / kTileHalf);
      float m = valid ? -INFINITY : 0.f, l = 0.f;          // reference (log2 units) and sum of the row
      uint32_t x[2][32], p[2][16];
      float sum;
      auto weights = [&](float ref) {
        const uint64_t sl2_2 = f2(sl2, sl2), ref_2 = f2(-ref, -ref);
        uint64_t acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p0, p1;
            f2_split(fma2(f2(__uint_as_float(x[c][2 * i]), __uint_as_float(x[c][2 * i + 1])), sl2_2, ref_2), p0, p1);
            p0 = ex2(p0);
            p1 = ex2(p1);
            acc[i & 3] = add2(acc[i & 3], f2(p0, p1));
            p[c][i] = pack_pair<BF16>(p0, p1);
          }
        float l0, l1;
        f2_split(add2(add2(acc[0], acc[1]), add2(acc[2], acc[3])), l0, l1);
        sum = l0 + l1;
      };
      auto hand_over = [&](int half) {
        l += sum;
        tmem_st16(ts + half * 32, p[0]);
        tmem_st16(ts + half * 32 + 16, p[1]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(t, cs & 1u));
        ++cs;
      };
#pragma unroll 1
      for (int h = h0; h < h1; h = next_half(keys, h)) {
        if (h == h0 || (h & 1) == 0) {
          wait_phase(s_full(t), cb & 1u, limit, s_abort, a.status);
          tc_fence_after();
          ++cb;
        }
        if (!any_row) {                                    // nothing of this warp's rows is wanted
          if (lane == 0) mbar_arrive(p_full(t, cs & 1u));
          ++cs;
          continue;
        }
        const uint32_t th = ts + (h & 1) * kTileHalf;
        tmem_ld32(th, x[0]);
        tmem_ld32(th + 32, x[1]);
        tmem_ld_wait();
        const bool clear = h >= f0 && h < f1;              // nothing to mask
        const bool plain = clear && h > h0 && !negate;     // and a reference to begin with
        bool over = true;
        if (plain) {
          weights(m);
          over = valid && !(sum <= 256.f);                 // (true too for a row without a reference: its sum is not a number)
        }
        if (__builtin_expect(__any_sync(0xffffffffu, over), 0)) {
          const int first = h * kTileHalf;
          if (negate) {
#pragma unroll
            for (int i = 0; i < 64; ++i) x[i >> 5][i & 31] ^= 0x80000000u;
          }
          if (!clear) {
            const int c_hi = pos - first, c_lo = a.window > 0 ? pos - a.window + 1 - first : -1;
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (i > c_hi || i < c_lo) x[i >> 5][i & 31] = 0xff800000u;
          }
          float mx[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) mx[i] = fmaxf(__uint_as_float(x[0][i]), __uint_as_float(x[0][8 + i]));
#pragma unroll
          for (int c = 16; c < 64; c += 16)
#pragma unroll
            for (int i = 0; i < 8; ++i) mx[i] = max3(mx[i], __uint_as_float(x[c >> 5][(c & 31) + i]), __uint_as_float(x[c >> 5][(c & 31) + 8 + i]));
          const float bm = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * sl2;
          const bool grow = bm > m + 8.f || (plain && over && bm > m);
          if (h > h0 && __any_sync(0xffffffffu, grow)) {
            // the product of the half before has to be in O (this one's is not asked for yet)
            wait_phase(pv_done(t, cs - 1), ((cs - 1) >> 1) & 1u, limit, s_abort, a.status);
            tc_fence_after();
            const float f = grow ? ex2(m - bm) : 1.f;
            l *= f;
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tmem_ld16(to + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st16(to + c, o);
            }
          }
          if (grow) m = bm;
          weights(m == -INFINITY ? 0.f : m);               // (every score -infinity: weights of 0)
        }
        hand_over(h & 1);
      }
      const bool any = h1 > h0;

      // ------------------------------ result of the item ------------------------------
      w.fetch(a.w.tile, hdr.n_tile, a.n_kv, u_end);
      if (sp.n > 0) {
        if (any) {
          wait_phase(pv_done(t, cs - 1), ((cs - 1) >> 1) & 1u, limit, s_abort, a.status);
          tc_fence_after();
        }
        const int tok_base = e.tok0 + (keys ? 0 : t) * tokens;
        const long long tg = tok_base + tok;
        const int hq = head * a.group + hq_in;
        // this thread's row relative to the tile's first, -1 where there is none; the rows it writes in `emit`
        const int dst = valid ? tok * (int)a.out_stride + hq_in * D : -1;
        uint16_t *out = a.out + (long long)tok_base * a.out_stride + (long long)head * a.group * D + (lane & 7) * 8;
        int rows[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rows[i] = __shfl_sync(0xffffffffu, dst, i * 4 + (lane >> 3));
        unsigned char *stage = s_stage + warp * 4096;         // this warp's 32 rows x 64 columns
        // 64 columns of the rows, one a thread, to memory: through shared memory (16-byte chunks swizzled by the row), so that
        // eight lanes write the 128 bytes of a row
        auto emit = [&](int c, const uint32_t (&o)[2][32], float inv) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint32_t v[4];
#pragma unroll
            for (int z = 0; z < 4; ++z)
              v[z] = pack_pair<BF16>(__uint_as_float(o[i >> 2][(i & 3) * 8 + 2 * z]) * inv, __uint_as_float(o[i >> 2][(i & 3) * 8 + 2 * z + 1]) * inv);
            *reinterpret_cast<uint4 *>(stage + lane * 128 + ((i ^ (lane & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + (lane >> 3);
            const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
            if (rows[i] >= 0) *reinterpret_cast<uint4 *>(out + rows[i] + c) = v;
          }
          __syncwarp();
        };
        auto store_lse = [&](float mm, float ll) {
          if (a.lse && valid) a.lse[tg * a.n_q + hq] = row_lse(mm, ll);
        };
        const bool whole = take == e.nb;
        // (an item that began in the share before leaves its part in the CTA's first place, one that goes on in its second)
        float *part = a.part + (size_t)((blockIdx.x * 2 + (blk == 0 ? 1 : 0)) * 2 + (keys ? 0 : t)) * Cfg::kPart;
        float f_own = 1.f, f_other = 0.f;
        bool any_other = false;
        if (keys) {
          // the other tile has the same rows: its reference and sum through shared memory, its O from tensor memory
          float2 *ml = reinterpret_cast<float2 *>(stage);
          ml[lane] = make_float2(m, l);
          if (lane == 0) ml[32].x = any ? 1.f : 0.f;
          tc_fence_before();
          named_sync(1, 256);
          tc_fence_after();
          const float2 *other = reinterpret_cast<const float2 *>(s_stage + (warp ^ 4) * 4096);
          const float mo = other[lane].x, lo_sum = other[lane].y;
          any_other = other[32].x != 0.f;
          named_sync(1, 256);
          const float mj = fmaxf(m, mo), bm = mj == -INFINITY ? 0.f : mj;
          f_own = ex2(m - bm);
          f_other = ex2(mo - bm);
          l = l * f_own + lo_sum * f_other;
          m = mj;
        }
        const float inv = row_inv(l);
        const uint32_t other_o = tm_o + (1 - t) * D + lanes;
        // with `keys` the tiles share the columns out (D = 64: tile 0 takes them)
        const int c_begin = keys ? t * 64 : 0, c_end = keys ? min(D, (t + 1) * 64) : D;
#pragma unroll 1
        for (int c = c_begin; c < c_end && any_row; c += 64) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (any) {
              tmem_ld32(to + c + i * 32, x[i]);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int z = 0; z < 32; ++z) x[i][z] = 0u;
            }
            if (keys) {
              uint32_t y[32];
              if (any_other) {
                tmem_ld32(other_o + c + i * 32, y);
                tmem_ld_wait();
              } else {
#pragma unroll
                for (int z = 0; z < 32; ++z) y[z] = 0u;
              }
#pragma unroll
              for (int z = 0; z < 32; ++z)
                x[i][z] = __float_as_uint(__uint_as_float(x[i][z]) * f_own + __uint_as_float(y[z]) * f_other);
            }
          }
          if (!keys && any && c + 64 == D) {                  // O_t is free
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_empty(t));
          }
          if (whole) {
            emit(c, x, inv);
          } else if (valid) {
#pragma unroll
            for (int i = 0; i < 64; ++i) part[256 + (c + i) * 128 + row] = __uint_as_float(x[i >> 5][i & 31]);
          }
        }
        if (!keys && any && !any_row && lane == 0) mbar_arrive(o_empty(t));
        if (keys) {                                           // both have read both
          tc_fence_before();
          named_sync(1, 256);
          if (any && lane == 0) mbar_arrive(o_empty(t));
        }
        if (!keys || t == 0) {
          if (whole) {
            store_lse(m, l);
          } else {
            part[row] = m;
            part[128 + row] = l;
          }
        }
      }
    }
  }
  abort_drain(s_abort);
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Joins the parts of the items that several CTAs of the tiled kernel shared, in the order of the CTAs:
//   m = max_c m_c, out = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c.
// Block (c, y): the item that began in CTA c - 1 and goes on in CTA c (none, mostly), tile y / (D/16), 16 of its columns;
// a thread owns a row, so the parts, kept by column, are read in whole lines.  A launch of its own: one CTA joining an item
// that all 148 share (19 MB of parts) took 60 us and more.
template <int D, bool BF16>
__global__ void __launch_bounds__(128) attn_join_kernel(const AttnFwdArgs a) {
  using Cfg = TileCfg<D>;
  grid_let_next();
  grid_wait();
  const AttnPlanHdr hdr = *a.w.hdr;
  const int c = blockIdx.x + 1, t = blockIdx.y / (D / 16), c0 = (blockIdx.y % (D / 16)) * 16, row = threadIdx.x;
  if ((long long)c * hdr.tile_quota >= hdr.tile_units) return;
  const AttnStart st = a.w.tile_start[c];
  const AttnEntry &e = st.e;
  const int u = e.unit0 * a.n_kv + st.head * (e.nb + kTileCost) + kTileCost;
  if (st.blk == 0 || u / hdr.tile_quota != c - 1) return;
  const int tokens = kTileRows / a.group, tok = row / a.group;
  const int last = (u + e.nb - 1) / hdr.tile_quota;
  if (tok >= min(tokens, e.n_tok - t * tokens)) return;
  auto part_of = [&](int i) { return a.part + (size_t)((i * 2 + (i == c - 1 ? 1 : 0)) * 2 + t) * Cfg::kPart; };
  float mm = -INFINITY, ll = 0.f;
#pragma unroll 4
  for (int i = c - 1; i <= last; ++i) {
    const float mc = part_of(i)[row], lc = part_of(i)[128 + row];
    const float mn = fmaxf(mm, mc), bm = mn == -INFINITY ? 0.f : mn;
    ll = ll * ex2(mm - bm) + lc * ex2(mc - bm);
    mm = mn;
  }
  const float bm = mm == -INFINITY ? 0.f : mm, inv = row_inv(ll);
  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll 2
  for (int i = c - 1; i <= last; ++i) {
    const float *pc = part_of(i);
    const float f = ex2(pc[row] - bm);
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[x] = fmaf(f, pc[256 + (c0 + x) * 128 + row], acc[x]);
  }
  const long long tg = e.tok0 + t * tokens + tok;
  const int hq = st.head * a.group + row - tok * a.group;
  uint4 *dst = reinterpret_cast<uint4 *>(a.out + tg * a.out_stride + hq * D + c0);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t v[4];
#pragma unroll
    for (int z = 0; z < 4; ++z) v[z] = pack_pair<BF16>(acc[i * 8 + 2 * z] * inv, acc[i * 8 + 2 * z + 1] * inv);
    dst[i] = make_uint4(v[0], v[1], v[2], v[3]);
  }
  if (a.lse && c0 == 0) a.lse[tg * a.n_q + hq] = row_lse(mm, ll);
}

}  // namespace ftmoe
