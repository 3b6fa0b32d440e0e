// Attention of requests with many query rows (chunks, whole prompts, wide groups) over the paged cache, on the
// 5th-generation tensor cores.  4*D flops per (query head, key) pair: bound by the tensor pipe and, at the same rate, by the
// exponentials (128 x 128 of either take the tensor pipe 2 x 512 and the special-function units 1024 clocks at D = 128).
//
// A work item is up to 256 query rows (tokens x heads of the group: the keys of a head are read once for all of them) of a
// request, as two tiles of 128 rows; its key blocks of 128 are its work units, cut into equal shares, one CTA per SM (the
// work partition of attn_plan.cuh).  Roles of the warps:
//   warp 9     brings Q (4-D TMA boxes: D, heads of the group, head, tokens) and the pages of K and V (128-byte swizzle)
//   warp 8     issues tcgen05.mma: S_t = Q_t K^T into tensor memory, O_t += P_t V with P_t read from tensor memory
//   warps 0-3, 4-7   softmax of tile 0 and 1: a thread owns a row, so maximum and sum need no exchange; P overwrites S
// While one tile is in its softmax the tensor pipe works for the other.  The order of issue (PV_t of block j, then QK_t of
// block j+1) makes the completion of S_t imply that O_t is at rest, so a row's rescaling of O_t in tensor memory needs no
// barrier of its own; it is left out while the maximum grows by less than 2^8 (the result is the same: the sum is taken
// with the same reference; 16-bit weights up to 2^8 have the same relative rounding).
// P is rounded to the values' type for the second product; scores, maxima, sums and O stay in 32 bits.
#pragma once
#include "attn_stream.cuh"

namespace ftmoe {

constexpr int kTileThreads = 320;
template <int D> struct TileCfg {
  static constexpr int kChunks = D / 64;                    // 64-element pieces of D: 128 rows x 128 bytes each
  static constexpr int kTile = 128 * D * 2;                 // bytes of 128 rows of Q, K or V
  static constexpr int kStages = D == 128 ? 5 : 10;         // ring of K and V tiles
  static constexpr int kBars = 2 * kStages + 2 + 8;
  static constexpr int kSmem = 1024 + 2 * kTile + kStages * kTile + kBars * 8 + 64;
  static constexpr int kPart = 128 * (D + 2);               // floats of one tile's partial result: m[128], l[128], O[D][128]
};
static_assert(TileCfg<128>::kSmem <= 232448 && TileCfg<64>::kSmem <= 232448, "shared memory of a CTA");

__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) { umma_bf16(d, a, b, idesc, acc); }
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a_tmem), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
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

// What a tile of a work item covers.
struct TileSpan {
  int n, lo, hi, pos0;       // rows' tokens, keys [lo, hi) some row attends to, position of the first token
  __device__ __forceinline__ bool active(int kb) const { return n > 0 && kb * kTileKeys < hi && (kb + 1) * kTileKeys > lo; }
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
  uint64_t *s_bar = reinterpret_cast<uint64_t *>(smem + (2 + Cfg::kStages) * Cfg::kTile);
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(s_bar + Cfg::kBars);
  volatile int *s_abort = reinterpret_cast<volatile int *>(s_tmem + 1);
  volatile int *s_last = s_abort + 1;                        // [2]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t q_smem = smem_u32(smem), ring = q_smem + 2 * Cfg::kTile, bars = smem_u32(s_bar);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (Cfg::kStages + s); };
  const uint32_t q_full = bars + 8u * (2 * Cfg::kStages), q_empty = q_full + 8;
  auto s_full = [&](int t) { return q_full + 16 + 8u * t; };
  auto p_full = [&](int t) { return q_full + 32 + 8u * t; };
  auto o_full = [&](int t) { return q_full + 48 + 8u * t; };
  auto o_empty = [&](int t) { return q_full + 64 + 8u * t; };

  const AttnPlanHdr hdr = *a.w.hdr;
  const long long u_first = (long long)blockIdx.x * hdr.tile_quota;
  if (u_first >= hdr.tile_units) return;
  int left = (int)min((long long)hdr.tile_quota, hdr.tile_units - u_first);
  const int4 st = a.w.tile_start[blockIdx.x];
  if (tid == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int t = 0; t < 2; ++t) { mbar_init(s_full(t), 1); mbar_init(p_full(t), 4); mbar_init(o_full(t), 1); mbar_init(o_empty(t), 4); }
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
  const uint32_t tm_s = tmem, tm_o = tmem + 256;             // S_t (and P_t) at 128 t, O_t at 256 + D t
  const int tokens = kTileRows / a.group;                    // tokens of a tile
  int k = st.x, head = st.y, blk = st.z;

  if (warp == 9) {
    // ------------------------------ loads ------------------------------
    const int page_tokens = 1 << a.page_shift;
    const int box_rows = min(page_tokens, kDecKeys), boxes = kTileKeys / box_rows;
    const int bx = lane / Cfg::kChunks, ch = lane % Cfg::kChunks;
    const bool owner = bx < boxes;
    uint32_t it = 0, items = 0;
    while (left > 0 && !*s_abort) {
      const AttnEntry e = a.w.tile[k];
      const int take = min(left, e.nb - blk);
      const int hi = max(0, e.pos0 + e.n_tok), lo = a.window > 0 ? max(0, e.pos0 - a.window + 1) : 0;
      const int32_t *row = a.table + (long long)e.req * a.table_stride;
      auto wanted = [&](int b) {
        const int key = (e.b0 + b) * kTileKeys + bx * box_rows;
        return owner && key < hi && key + box_rows > lo;
      };
      auto page_of = [&](int b) -> int { return wanted(b) ? row[((e.b0 + b) * kTileKeys + bx * box_rows) >> a.page_shift] : 0; };
      int page = page_of(blk);
      mbar_wait(q_empty, (items & 1u) ^ 1u, s_abort, a.status);
      if (*s_abort) break;
      if (lane == 0) {
        const int n_tiles = e.n_tok > tokens ? 2 : 1;
        mbar_expect_tx(q_full, (uint32_t)(n_tiles * Cfg::kChunks * tokens * a.group * 128));
        for (int t = 0; t < n_tiles; ++t)
          for (int c = 0; c < Cfg::kChunks; ++c)
            tma_load_4d(q_smem + t * Cfg::kTile + c * 16384, &tm_q, c * 64, 0, head, e.tok0 + t * tokens, q_full);
      }
      ++items;
      for (int b = blk; b < blk + take; ++b) {
        const int next = b + 1 < blk + take ? page_of(b + 1) : 0;
        const bool want = wanted(b);
        if (want && (uint32_t)page >= (uint32_t)a.n_pages) {     // never followed: page 0 instead, and reported
          atomicOr(a.status, kStatBadIndex);
          page = 0;
        }
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, want)) * (uint32_t)(box_rows * 128);
        const int y = ((e.b0 + b) * kTileKeys + bx * box_rows) & (page_tokens - 1);
#pragma unroll
        for (int v = 0; v < 2; ++v, ++it) {
          const int s = it % Cfg::kStages;
          mbar_wait(empty_bar(s), ((it / Cfg::kStages) & 1u) ^ 1u, s_abort, a.status);
          if (*s_abort) break;
          if (lane == 0) mbar_expect_tx(full_bar(s), bytes);
          __syncwarp();
          if (want)
            tma_load_3d(ring + s * Cfg::kTile + ch * 16384 + bx * box_rows * 128, &tm, ch * 64, y, (page * 2 + v) * a.n_kv + head,
                        full_bar(s));
        }
        if (*s_abort) break;
        page = next;
      }
      left -= take;
      blk = 0;
      if (++head == a.n_kv) { head = 0; ++k; }
    }
  } else if (warp == 8) {
    // ------------------------------ tensor core ------------------------------
    constexpr uint32_t type = BF16 ? (1u << 7) | (1u << 10) : 0u;
    constexpr uint32_t idesc_qk = (1u << 4) | type | ((uint32_t)(kTileKeys >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
    constexpr uint32_t idesc_pv = (1u << 4) | type | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
    uint32_t it = 0, items = 0, np[2] = {0, 0}, no[2] = {0, 0};
    while (left > 0) {
      const AttnEntry e = a.w.tile[k];
      const int take = min(left, e.nb - blk);
      const int hi = max(0, e.pos0 + e.n_tok), lo = a.window > 0 ? max(0, e.pos0 - a.window + 1) : 0;
      const TileSpan sp[2] = {tile_span(e, 0, tokens, a.window), tile_span(e, 1, tokens, a.window)};
      bool fresh[2] = {true, true};
      mbar_wait(q_full, items & 1u, s_abort, a.status);
      ++items;
      for (int j = 0; j <= take; ++j) {
        // K of block j is ring entry it + 2j, V of block j-1 entry it + 2j - 1
        const uint32_t ik = it + 2 * j, iv = ik - 1;
        const int kb = e.b0 + blk + j;
        const int sk = ik % Cfg::kStages, sv = iv % Cfg::kStages;
        const uint32_t kt = ring + sk * Cfg::kTile, vt = ring + sv * Cfg::kTile;
        bool ok = true;
        if (j > 0) {
          ok = mbar_wait(full_bar(sv), (iv / Cfg::kStages) & 1u, s_abort, a.status);
          const int first = (kb - 1) * kTileKeys;
          if (ok && (first + kTileKeys > hi || first < lo)) {
            // values no row attends to may be anything: their weight is 0, so they have to be finite
            for (int i = lane; i < kTileKeys * Cfg::kChunks * 8; i += 32) {
              const int r = (i >> 3) % kTileKeys, c = (i >> 3) / kTileKeys;
              if (first + r >= hi || first + r < lo)
                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vt + c * 16384 + r * 128 + (i & 7) * 16), "r"(0u) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (j > 0 && sp[t].active(kb - 1)) {
            if (fresh[t]) mbar_wait(o_empty(t), (no[t] & 1u) ^ 1u, s_abort, a.status);
            ok = mbar_wait(p_full(t), np[t] & 1u, s_abort, a.status) && ok;
            ++np[t];
            tc_fence_after();
            if (lane == 0 && ok) {
              const uint64_t dv = umma_desc(vt, 16384, 1024);      // (an address step is its 16-byte count in the low bits)
#pragma unroll
              for (int kk = 0; kk < kTileKeys / 16; ++kk)
                umma_ts(tm_o + t * D, tm_s + t * 128 + kk * 8, dv + kk * (2048 >> 4), idesc_pv, (fresh[t] && kk == 0) ? 0u : 1u);
            }
            fresh[t] = false;
            if (lane == 0 && (j == take || !sp[t].active(kb))) umma_commit(o_full(t));
            if (j == take || !sp[t].active(kb)) ++no[t];
          }
          if (j < take && sp[t].active(kb)) {
            ok = mbar_wait(full_bar(sk), (ik / Cfg::kStages) & 1u, s_abort, a.status) && ok;
            tc_fence_after();
            if (lane == 0) {
              if (ok) {
                const uint64_t dq = umma_desc(q_smem + t * Cfg::kTile, 16, 1024), dk = umma_desc(kt, 16, 1024);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                  umma_ss(tm_s + t * 128, dq + ((kk >> 2) * 16384 + (kk & 3) * 32) / 16, dk + ((kk >> 2) * 16384 + (kk & 3) * 32) / 16,
                          idesc_qk, kk != 0 ? 1u : 0u);
              }
              umma_commit(s_full(t));
            }
          }
        }
        if (lane == 0) {
          if (j > 0) umma_commit(empty_bar(sv));
          if (j < take) {
            // a block that no tile attends to is still waited for: its copies have to land before the stage is reused
            if (!sp[0].active(kb) && !sp[1].active(kb)) mbar_wait(full_bar(sk), (ik / Cfg::kStages) & 1u, s_abort, a.status);
            umma_commit(empty_bar(sk));
          }
          if (j == take - 1) umma_commit(q_empty);
        }
        __syncwarp();
      }
      it += 2 * take;
      left -= take;
      blk = 0;
      if (++head == a.n_kv) { head = 0; ++k; }
    }
  } else {
    // ------------------------------ softmax ------------------------------
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tm_s + t * 128 + lanes, to = tm_o + t * D + lanes;
    const int tok = row / a.group, hq_in = row - tok * a.group;
    const float sl2 = fabsf(a.scale_log2);
    const bool negate = a.scale_log2 < 0.f;
    uint32_t ns = 0, no = 0;
    while (left > 0) {
      const AttnEntry e = a.w.tile[k];
      const int take = min(left, e.nb - blk);
      const TileSpan sp = tile_span(e, t, tokens, a.window);
      const bool valid = tok < sp.n;                       // (tok < tokens holds for rows below tokens * group)
      const int pos = valid ? sp.pos0 + tok : -1;
      float m = -INFINITY, l = 0.f;
      bool any = false;
      for (int b = blk; b < blk + take; ++b) {
        const int kb = e.b0 + b;
        if (!sp.active(kb)) continue;
        const bool ok = mbar_wait(s_full(t), ns & 1u, s_abort, a.status);
        ++ns;
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(ts + c * 32, s[c]);
        tmem_ld_wait();
        if (negate) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) s[c][i] ^= 0x80000000u;
        }
        const int first = kb * kTileKeys;
        if (first + kTileKeys - 1 > sp.pos0 || (a.window > 0 && first <= sp.pos0 + sp.n - 1 - a.window)) {
          const int c_hi = pos - first, c_lo = a.window > 0 ? pos - a.window + 1 - first : -1;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c * 32 + i > c_hi || c * 32 + i < c_lo) s[c][i] = 0xff800000u;
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          mx[c] = __uint_as_float(s[c][0]);
#pragma unroll
          for (int i = 1; i < 32; ++i) mx[c] = fmaxf(mx[c], __uint_as_float(s[c][i]));
        }
        const float bm = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2;
        // keep the old reference while the maximum is at most 2^8 above it
        const bool grow = bm > m + 8.f;
        if (any) {
          if (__any_sync(0xffffffffu, grow)) {
            const float f = grow ? ex2(m - bm) : 1.f;
            l *= f;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t o[32];
              tmem_ld32(to + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(to + c, o);
            }
            if (grow) m = bm;
          }
        } else if (bm > m) {
          m = bm;
        }
        any = true;
        const float base = m == -INFINITY ? 0.f : m;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float p0 = ex2(fmaf(__uint_as_float(s[q4][2 * i]), sl2, -base));
            const float p1 = ex2(fmaf(__uint_as_float(s[q4][2 * i + 1]), sl2, -base));
            sum[(2 * i) & 2] += p0;
            sum[((2 * i) & 2) + 1] += p1;
            p[i] = pack_pair<BF16>(p0, p1);
          }
          tmem_st16(ts + q4 * 16, p);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(t));
        (void)ok;
      }

      // ------------------------------ result of the item ------------------------------
      if (sp.n > 0) {
        if (any) {
          mbar_wait(o_full(t), no & 1u, s_abort, a.status);
          ++no;
          tc_fence_after();
        }
        const int u0 = e.unit0 * a.n_kv + head * e.nb;
        const int c_first = u0 / hdr.tile_quota, c_last = (u0 + e.nb - 1) / hdr.tile_quota;
        const long long tg = e.tok0 + t * tokens + tok;
        const int hq = head * a.group + hq_in;
        uint16_t *dst = a.out + tg * a.out_stride + hq * D;
        auto store = [&](int c, const uint32_t (&o)[32], float inv) {
          uint4 *d4 = reinterpret_cast<uint4 *>(dst + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
              w[x] = pack_pair<BF16>(__uint_as_float(o[i * 8 + 2 * x]) * inv, __uint_as_float(o[i * 8 + 2 * x + 1]) * inv);
            d4[i] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        };
        auto store_lse = [&](float mm, float ll) {
          if (a.lse && valid) a.lse[tg * a.n_q + hq] = ll > 0.f ? (mm + log2f(ll)) * 0.693147180559945f : -INFINITY;
        };
        if (c_first == c_last) {
          const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            if (any) {
              tmem_ld32(to + c, o);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = 0u;
            }
            if (valid) store(c, o, inv);
          }
          store_lse(m, l);
        } else {
          float *part = a.part + (size_t)((blockIdx.x * 2 + ((int)blockIdx.x == c_first ? 1 : 0)) * 2 + t) * Cfg::kPart;
          part[row] = m;
          part[128 + row] = l;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            if (any) {
              tmem_ld32(to + c, o);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = 0u;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) part[256 + (c + i) * 128 + row] = __uint_as_float(o[i]);
          }
          __threadfence();
          named_sync(1 + t, 128);
          if (row == 0) {
            uint32_t *cnt = a.arrive + ((size_t)k * a.n_kv + head) * 2 + t;
            const bool last = atomicAdd(cnt, 1u) == (uint32_t)(c_last - c_first);
            if (last) *cnt = 0u;
            s_last[t] = last;
            __threadfence();
          }
          named_sync(1 + t, 128);
          if (s_last[t]) {
            float mm = -INFINITY, ll = 0.f;
            for (int c = c_first; c <= c_last; ++c) {
              const float *pc = a.part + (size_t)((c * 2 + (c == c_first ? 1 : 0)) * 2 + t) * Cfg::kPart;
              const float mc = __ldcg(pc + row), lc = __ldcg(pc + 128 + row);
              const float mn = fmaxf(mm, mc), bm = mn == -INFINITY ? 0.f : mn;
              ll = ll * ex2(mm - bm) + lc * ex2(mc - bm);
              mm = mn;
            }
            const float bm = mm == -INFINITY ? 0.f : mm, inv = ll > 0.f ? 1.f / ll : 0.f;
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 32) {
              float acc[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) acc[i] = 0.f;
              for (int c = c_first; c <= c_last; ++c) {
                const float *pc = a.part + (size_t)((c * 2 + (c == c_first ? 1 : 0)) * 2 + t) * Cfg::kPart;
                const float f = ex2(__ldcg(pc + row) - bm);
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[i] = fmaf(f, __ldcg(pc + 256 + (c0 + i) * 128 + row), acc[i]);
              }
              uint32_t o[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(acc[i]);
              if (valid) store(c0, o, inv);
            }
            store_lse(mm, ll);
          }
          named_sync(1 + t, 128);        // s_last is free again
        }
        if (any) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(o_empty(t));
        }
      }
      left -= take;
      blk = 0;
      if (++head == a.n_kv) { head = 0; ++k; }
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

}  // namespace ftmoe
