// Products with 4-bit weights for many tokens, on the 5th-generation tensor cores.  Image and formula: dense_w4.cuh.
//
// A block takes 128 rows (two quads) x up to 192 tokens and walks along k.  Bound: the tensor cores for many tokens (2 T N K flops), HBM and the
// expansion of the codes for few.
//   raw warp      brings the records of 128 k (bulk copies)
//   x warp        brings x (TMA, 64 k of the tokens a box, 128-byte swizzle)
//   expanding     turn codes into 16-bit numbers and leave them in tensor memory
//   mma warp      rows on M = 128 (A from tensor memory), tokens on N (B from shared memory)
// Two forms.  For 16-bit results the operands are the weights s (q - z), rounded once to the type (8 or 11 bits of scale times 4 of code do
// not fit it): an error of the size of the result's own rounding, 0.0014 of the result in bf16 where that is 0.0017.  The tensor core adds
// over all of k, and four warps take the sums out while it works on the next unit.  For float results (EXACT) the operands are the exact q - z,
// a group of k has an accumulator of its own (two in turn), and eight warps add its sums times the row's scale to float sums in registers;
// that takes 1.3 to 2.3 times as long (reading an accumulator beside the tensor core costs 70 clocks for 16 tokens of 32 rows): 22 against 17 us for 24
// tokens through 7168 x 7168, 26 against 18.5 for 64, 448 against 310 for 4096; 144 against 62 for 64 tokens through 2048 x 150001 in groups of 64.
// A weight that the type cannot hold (a scale above a fifteenth of its largest value may give one) makes every sum of its row infinite or NaN, whatever
// the token: a block that has seen one computes the results of those rows again in the end, a warp each, in the exact form.  Right, and slow.
// Measured: 310 us for 4096 tokens through 7168 x 7168 (1.36 PFLOP/s, 0.82 of a library product's rate for as short a run; 365 in a long one, 0.83 of the rate
// that holds there), 88 us for 1024 tokens with groups of 32, 18.5 us for 64 tokens.  With 17 tokens it passes the streaming kernel (24 tokens 17 against 22 us).
// With a cluster of c blocks each takes 1/c of k, and the sums are added over distributed shared memory, in the blocks' order.
#pragma once
#include "dense_w4.cuh"
#include "tcgen.cuh"

namespace ftmoe {

constexpr int kW4Ops = 2;                                       // operands of 128 k in tensor memory
constexpr int kW4Acc = 192, kW4OpAt = 2 * kW4Acc;               // columns of an accumulator; where the operands stand (64 columns each)
static_assert(kW4OpAt + kW4Ops * 64 <= 512, "tensor memory");

struct W4Tile {
  int32_t bn, cluster, row_tiles, tok_tiles;     // tokens of a tile (a multiple of 16)
  int32_t raw_bytes;                             // of a slot: two records
  int32_t ring_bytes;                            // of the tokens' stages, where the sums of a cluster's blocks go in the end
};

template <bool EXACT>
struct W4TileCfg {
  static constexpr int kThreads = EXACT ? 512 : 768, kAdd = EXACT ? 8 : 4, kExpand = EXACT ? 4 : 16;     // of its warps: the last ones, those from 4 on
  static constexpr int kTilesEach = EXACT ? 2 : 1, kHalvesEach = EXACT ? 2 : 1;  // tiles, and halves of 64 k, of an expanding warp
  static constexpr int kCols = kW4Acc / (kAdd / 4);                              // tokens of an adding warp
  static constexpr int kStage = kW4Acc * 256, kStages = 3;                       // 128 k of the tokens: two boxes of 64
  static constexpr int kRaw = EXACT ? 3 : 6;                                     // slots of records
  static constexpr int kBars = 2 * kRaw + 2 * kStages + 2 * kW4Ops + 4;
};
// Fills in the sizes; returns the bytes of dynamic shared memory.
template <bool EXACT>
inline int w4_tile_memory(const W4Geom &g, W4Tile &p) {
  const int stages = W4TileCfg<EXACT>::kStages * W4TileCfg<EXACT>::kStage, join = p.cluster > 1 ? (p.bn + p.cluster - 1) / p.cluster * p.cluster * 512 : 0;
  p.raw_bytes = (2 * g.record(4) + 127) / 128 * 128;
  p.ring_bytes = stages > join ? stages : join;
  return 1024 + p.ring_bytes + W4TileCfg<EXACT>::kRaw * p.raw_bytes + W4TileCfg<EXACT>::kBars * 8 + 32;
}

// Tokens of a tile and blocks that share k (`clusters`: how many clusters of a size the GPU holds at once): the split with the least clocks of the SM with the most to do.  A block of 128 k takes 4 clocks a
// token in the tensor cores, not less than its codes take to expand, nor than its groups' sums to be added; a unit 4000 more, and 2000 over a cluster.
inline W4Tile w4_tile_share(const W4Geom &g, int T, bool exact, const int *clusters) {
  W4Tile best{};
  double least = 1e30;
  const int row_tiles = (g.quads + 1) / 2, per = kW4Block / g.group;
  for (int bn = 32; bn <= kW4Acc; bn += 16) {
    if (bn > 32 && bn - 16 >= T) break;
    for (int cluster = 1; cluster <= kW4MaxCluster && (cluster == 1 || g.nb >= 2 * cluster); ++cluster) {
      const int tok_tiles = (T + bn - 1) / bn;
      const long long units = (long long)row_tiles * tok_tiles, fit = clusters[cluster];
      if (fit == 0 || (cluster > 1 && units > fit)) continue;
      double block = 4. * bn;
      const double expand = exact ? 850 : 750, add = exact ? per * (300 + 4. * bn) : 0.;
      if (block < expand) block = expand;
      if (block < add) block = add;
      const double cost = (double)((units + fit - 1) / fit) * ((double)((g.nb + cluster - 1) / cluster) * block + 4000 + (cluster > 1 ? 2000 : 0));
      if (cost < least) {
        least = cost;
        best.bn = bn; best.cluster = cluster; best.row_tiles = row_tiles; best.tok_tiles = tok_tiles;
      }
    }
  }
  return best;
}

// Whether a weight of row n may be beyond the type's largest value.
template <bool BF16>
__device__ __forceinline__ bool w4_row_over(const W4Args &a, int n) {
  const W4Geom &g = a.g;
  const int quad = n >> 6, m = g.tiles_of(quad), per = kW4Block / g.group;
  const uint8_t *sc = a.image + g.quad_at(quad) + m * 2 * kW4TileBytes + (n & 7) * 16 + (n >> 4 & 3) * 4 + (n >> 3 & 1) * 2;
  bool over = false;
  for (int b = 0; b < g.nb; ++b, sc += g.record(m))
    for (int i = 0; i < per; ++i) over |= fabsf(to_float<BF16>(*reinterpret_cast<const uint16_t *>(sc + i * 128))) > (BF16 ? 3.3895313892515355e38f : 65504.f) / 15.f;
  return over;
}
// The sum of row n and token t in the exact form, by a warp: a lane has 4 of 128 k, their products with q - z, then the scale, in float.
template <bool BF16>
__device__ __forceinline__ float w4_one(const W4Args &a, long long t, int n) {
  const W4Geom &g = a.g;
  const int lane = threadIdx.x & 31, quad = n >> 6, m = g.tiles_of(quad), tile = n >> 4 & 3, gr = n & 7, high = n >> 3 & 1, s = lane * 4 / g.group;
  const uint8_t *rec = a.image + g.quad_at(quad), *sc = rec + m * 2 * kW4TileBytes + s * 128 + gr * 16 + tile * 4 + high * 2;
  const uint8_t *word = rec + ((lane >> 4) * m + tile) * kW4TileBytes + (gr * 4 + (lane & 3)) * 16 + (lane >> 2 & 3) * 4;
  const uint8_t *zero = rec + m * 2 * kW4TileBytes + kW4Block / g.group * 128 + s * 64 + gr * 8 + tile * 2 + high;
  const uint16_t *x = a.x + t * a.x_stride;
  float sum = 0.f;
  for (int k = lane * 4; k < g.k; k += kW4Block) {
    const uint2 v = *reinterpret_cast<const uint2 *>(x + k);
    const uint32_t w = *reinterpret_cast<const uint32_t *>(word), pair[2] = {v.x, v.y};
    const float z = g.zeros ? (float)*zero : 8.f;
    float part = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b) {                  // (of a word, pairs `high` and 2 + high are the row's)
      const uint32_t c = rotl32(w, 32 - (high ? w4_bit<BF16>(2 * b + 1) : w4_bit<BF16>(2 * b)));
      float x0, x1;
      to_float2<BF16>(pair[b], x0, x1);
      part = fmaf(x0, (float)(c & 15u) - z, part);
      part = fmaf(x1, (float)(c >> 16 & 15u) - z, part);
    }
    sum = fmaf(to_float<BF16>(*reinterpret_cast<const uint16_t *>(sc)), part, sum);
    word += g.record(m);
    sc += g.record(m);
    zero += g.record(m);
  }
  return warp_sum(sum);
}

// A block's results in rows whose weights may be beyond the type's largest value, a warp each.  Not inlined and with arguments of its own: an address of the
// kernel's own ones costs it 2 us of 14 (512 tokens x 2048 x 5120), a copy of them 30 of 310 (4096 tokens x 7168 x 7168).
struct W4Again { W4Args a; W4Tile p; };
template <bool BF16>
__device__ __noinline__ void w4_again(const W4Again &args, int threads) {
  const W4Args &a = args.a;
  const W4Tile &p = args.p;
  const int rank = blockIdx.x % p.cluster, n_cl = gridDim.x / p.cluster, share = (p.bn + p.cluster - 1) / p.cluster, lane = threadIdx.x & 31;
  for (int u = blockIdx.x / p.cluster; u < p.row_tiles * p.tok_tiles; u += n_cl) {
    const int tok0 = u / p.row_tiles * p.bn + rank * share, row0 = u % p.row_tiles * 128;
    const int n_tok = min(min(share, p.bn - rank * share), a.T - tok0);
    for (int r = 0; r < 128; r += 32) {
      uint32_t rows = __ballot_sync(0xffffffffu, row0 + r + lane < a.g.n && w4_row_over<BF16>(a, row0 + r + lane));
      for (; rows; rows &= rows - 1) {
        const int n = row0 + r + __ffs(rows) - 1;
        for (int t = threadIdx.x >> 5; t < n_tok; t += threads / 32) {
          const float v = w4_one<BF16>(a, tok0 + t, n);
          if (lane == 0) w4_store<BF16>(a, tok0 + t, n, v);
        }
      }
    }
  }
}

template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

template <bool BF16, bool ZERO, bool EXACT>
__global__ void __launch_bounds__(W4TileCfg<EXACT>::kThreads, 1) w4_tile_kernel(const __grid_constant__ CUtensorMap tm_x, const W4Args a, const W4Tile p,
                                                                                   const __grid_constant__ W4Again args) {
  using Cfg = W4TileCfg<EXACT>;
  constexpr int kRaw = Cfg::kRaw;
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char *s_rec = smem + p.ring_bytes;
  uint64_t *s_bar = reinterpret_cast<uint64_t *>(s_rec + kRaw * p.raw_bytes);
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(s_bar + Cfg::kBars);
  volatile int *s_abort = reinterpret_cast<volatile int *>(s_tmem + 2);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t stage0 = smem_u32(smem), rec0 = smem_u32(s_rec), bars = smem_u32(s_bar);
  auto raw_full = [&](int i) { return bars + 8u * i; };
  auto raw_empty = [&](int i) { return bars + 8u * (kRaw + i); };
  constexpr int kX = 2 * kRaw, kW = kX + 2 * Cfg::kStages, kD = kW + 2 * kW4Ops;
  auto x_full = [&](int i) { return bars + 8u * (kX + i); };
  auto x_empty = [&](int i) { return bars + 8u * (kX + Cfg::kStages + i); };
  auto w_full = [&](int i) { return bars + 8u * (kW + i); };
  auto w_empty = [&](int i) { return bars + 8u * (kW + kW4Ops + i); };
  auto d_full = [&](int i) { return bars + 8u * (kD + i); };
  auto d_empty = [&](int i) { return bars + 8u * (kD + 2 + i); };
  auto wait = [&](uint32_t bar, uint32_t phase) { return mbar_try_wait(bar, phase) || mbar_wait(bar, phase, s_abort, a.status); };

  auto given_up = [&]() { return __any_sync(0xffffffffu, *s_abort) != 0; };      // (the same for all lanes: what follows elects one of all)

  grid_let_next();
  if (tid == 0) {
    for (int i = 0; i < kRaw; ++i) { mbar_init(raw_full(i), 1); mbar_init(raw_empty(i), EXACT ? Cfg::kAdd + Cfg::kExpand : Cfg::kExpand); }
    for (int i = 0; i < Cfg::kStages; ++i) { mbar_init(x_full(i), 1); mbar_init(x_empty(i), 1); }
    for (int i = 0; i < kW4Ops; ++i) { mbar_init(w_full(i), Cfg::kExpand); mbar_init(w_empty(i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(d_full(i), 1); mbar_init(d_empty(i), Cfg::kAdd); }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  grid_wait();

  const W4Geom &g = a.g;
  const int cluster = p.cluster, rank = blockIdx.x % cluster, units = p.row_tiles * p.tok_tiles, n_cl = gridDim.x / cluster, cl = blockIdx.x / cluster;
  const int b0 = (int)((long long)g.nb * rank / cluster), b1 = (int)((long long)g.nb * (rank + 1) / cluster);
  const int per = kW4Block / g.group, rec4 = g.record(4);       // groups of a record
  float odd = 0.f;                                              // NaN once a row's sum (of any token) is not finite
  constexpr int kFirstAdd = Cfg::kThreads / 32 - Cfg::kAdd, kFirstExpand = 4;

  if (warp < 4) {
    if constexpr (EXACT) regs_down<80>();
    // (whole warps walk through the loops, so that what a copy or a product is given stands in uniform registers; one lane issues)
    if (warp == 0) {
      // ------------------------------ x ------------------------------
      int s = 0;
      uint32_t ph = 1;
      for (int u = cl; u < units; u += n_cl) {
        const int tok0 = u / p.row_tiles * p.bn;
        for (int b = b0; b < b1; ++b) {
          wait(x_empty(s), ph);
          if (given_up()) break;        // (a barrier may still expect its bytes: it must not be armed again)
          if (elect_one()) {
            const uint32_t to = stage0 + s * Cfg::kStage;
            mbar_expect_tx(x_full(s), 2 * p.bn * 128);
            tma_load_2d(to, &tm_x, b * kW4Block, tok0, x_full(s));
            tma_load_2d(to + kW4Acc * 128, &tm_x, b * kW4Block + 64, tok0, x_full(s));
          }
          if (++s == Cfg::kStages) { s = 0; ph ^= 1; }
        }
      }
    } else if (warp == 2) {
      // ------------------------------ records ------------------------------
      bool withhold = blockIdx.x == 0 && (g_debug_withhold & kWithholdW4Tile);
      int s = 0;
      uint32_t ph = 1;
      for (int u = cl; u < units; u += n_cl) {
        const int quad = u % p.row_tiles * 2;
        const bool two = quad + 1 < g.quads;
        const int r0 = g.record(g.tiles_of(quad)), r1 = two ? g.record(g.tiles_of(quad + 1)) : 0;
        const uint8_t *src0 = a.image + g.quad_at(quad) + (long long)b0 * r0, *src1 = a.image + g.quad_at(quad + 1) + (long long)b0 * r1;
        for (int b = b0; b < b1; ++b, src0 += r0, src1 += r1) {
          wait(raw_empty(s), ph);
          if (given_up()) break;
          if (elect_one()) {
            mbar_expect_tx(raw_full(s), r0 + r1);
            if (!withhold) bulk_g2s(rec0 + s * p.raw_bytes, src0, r0, raw_full(s));      // (withheld: test hook)
            if (two) bulk_g2s(rec0 + s * p.raw_bytes + rec4, src1, r1, raw_full(s));
          }
          withhold = false;
          if (++s == kRaw) { s = 0; ph ^= 1; }
        }
      }
    } else if (warp == 1) {
      // ------------------------------ mma ------------------------------
      const uint32_t idesc = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(p.bn >> 3) << 17) | ((128u >> 4) << 24);
      const uint32_t tmem_u = uniform(tmem), stage_u = uniform(stage0);
      int s = 0, o = 0, d = 0;
      uint32_t ph = 0, oph = 0, dph = 1;
      auto run = [&](auto steps) {                   // EXACT: instructions of a group of k
        constexpr int kSteps = decltype(steps)::value;
        for (int u = cl; u < units; u += n_cl) {
          if (!EXACT) wait(d_empty(d), dph);
          for (int b = b0, dead = 0; b < b1 && !dead; ++b) {
            dead = given_up();
            wait(x_full(s), ph);
            const bool ok = wait(w_full(o), oph);
            const uint64_t x_desc = umma_desc(stage_u + s * Cfg::kStage, 16, 1024);
            const uint32_t w_at = tmem_u + kW4OpAt + o * 64;
#pragma unroll
            for (int k0 = 0; k0 < 8; k0 += kSteps) {
              if (EXACT) wait(d_empty(d), dph);
              tc_fence_after();
              if (elect_one()) {
                if (ok)
#pragma unroll
                  for (int k16 = k0; k16 < k0 + kSteps; ++k16)
                    umma_ts(tmem_u + d * kW4Acc, w_at + 8 * k16, x_desc + (k16 / 4 * kW4Acc * 128 + k16 % 4 * 32) / 16, idesc,
                            k16 != k0 || (!EXACT && b != b0));
                if (EXACT) umma_commit(d_full(d));
              }
              __syncwarp();
              if (EXACT) {
                d ^= 1;
                if (d == 0) dph ^= 1;
              }
            }
            if (elect_one()) {
              umma_commit(w_empty(o));
              umma_commit(x_empty(s));
            }
            __syncwarp();
            if (++s == Cfg::kStages) { s = 0; ph ^= 1; }
            if (++o == kW4Ops) { o = 0; oph ^= 1; }
          }
          if (!EXACT) {
            if (elect_one()) umma_commit(d_full(d));
            __syncwarp();
            d ^= 1;
            if (d == 0) dph ^= 1;
          }
        }
      };
      if (!EXACT || per == 1) run(std::integral_constant<int, 8>());
      else if (per == 2) run(std::integral_constant<int, 4>());
      else run(std::integral_constant<int, 2>());
    }
  } else if (warp < kFirstExpand + Cfg::kExpand) {
    // ------------------------------ expansion ------------------------------
    // A warp has the tiles of its quarter of tensor memory, both or one of them, with both halves of the 128 k or one; what is not there (rows
    // past the last) is expanded from whatever the slot holds: its operands reach no other row.
    if constexpr (EXACT) regs_down<96>();
    constexpr int kMine = Cfg::kTilesEach, kHalves = Cfg::kHalvesEach;
    const int tile0 = 2 * (warp & 3) + (kMine == 1 ? (warp - kFirstExpand) >> 2 & 1 : 0), half0 = kHalves == 1 ? (warp - kFirstExpand) >> 3 : 0, gr = lane >> 2;
    const W4Const<BF16> con;
    const uint32_t dst = tmem + kW4OpAt + ((uint32_t)(tile0 * 16) << 16);
    int s = 0, rs = 0;
    uint32_t ph = 1, rph = 0;
    for (int u = cl; u < units; u += n_cl) {
      const int quad0 = u % p.row_tiles * 2;
      uint32_t src[kMine], sc_at[kMine], z_at[kMine], next[kMine];           // codes, scales, zero points, from half to half
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const int t = tile0 + j, quad = t >> 2, m = quad0 + quad < g.quads ? g.tiles_of(quad0 + quad) : 1;
        const uint32_t rec = rec0 + quad * rec4;
        src[j] = rec + min(t & 3, m - 1) * kW4TileBytes + lane * 16;
        next[j] = m * kW4TileBytes;
        sc_at[j] = rec + m * 2 * kW4TileBytes + gr * 16 + (t & 3) * 4;
        z_at[j] = rec + m * 2 * kW4TileBytes + per * 128 + gr * 8 + (t & 3) * 2;
      }
      struct Rec {
        uint4 w[kHalves][kMine];
        uint32_t z[kHalves][2][kMine], sc[kHalves][2][kMine];    // per half and 32 k of it
      };
      auto take = [&](Rec &r) {
        wait(raw_full(rs), rph);
        const uint32_t at = rs * p.raw_bytes;
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
          for (int j = 0; j < kMine; ++j) {
            r.w[half][j] = lds_v4(src[j] + at + (half0 + half) * next[j]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (!EXACT) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r.sc[half][h][j]) : "r"(sc_at[j] + at + ((half0 + half) * 2 + h) * per / 4 * 128));
              if (ZERO) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(r.z[half][h][j]) : "r"(z_at[j] + at + ((half0 + half) * 2 + h) * per / 4 * 64));
            }
          }
      };
      auto give_back = [&]() {                       // (the record has been read)
        __syncwarp();
        if (lane == 0) mbar_arrive(raw_empty(rs));
        if (++rs == kRaw) { rs = 0; rph ^= 1; }
      };
      auto expand = [&](const Rec &rec) {
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
          for (int j = 0; j < kMine; ++j) {
            const uint32_t words[4] = {rec.w[half][j].x, rec.w[half][j].y, rec.w[half][j].z, rec.w[half][j].w};
            uint32_t r[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t lo = BF16 ? 0x41c041c0u : 0x4e004e00u, hi = lo;      // 16 + 8
              if (ZERO) w4_zero_pairs<BF16>(rec.z[half][i / 2][j], lo, hi);
              uint32_t c[4];
              w4_expand<BF16>(con, words[i], c);
              r[4 * i] = sub_pair<BF16>(c[0], lo); r[4 * i + 1] = sub_pair<BF16>(c[2], lo);
              r[4 * i + 2] = sub_pair<BF16>(c[1], hi); r[4 * i + 3] = sub_pair<BF16>(c[3], hi);
              if (!EXACT) {
                const uint32_t sc = rec.sc[half][i / 2][j], s_lo = __byte_perm(sc, 0, 0x1010), s_hi = __byte_perm(sc, 0, 0x3232);
                r[4 * i] = mul_pair<BF16>(r[4 * i], s_lo); r[4 * i + 1] = mul_pair<BF16>(r[4 * i + 1], s_lo);
                r[4 * i + 2] = mul_pair<BF16>(r[4 * i + 2], s_hi); r[4 * i + 3] = mul_pair<BF16>(r[4 * i + 3], s_hi);
              }
            }
            tmem_st_16x256b_x4(dst + ((uint32_t)(j * 16) << 16) + s * 64 + (half0 + half) * 32, r);
          }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(w_full(s));
        if (++s == kW4Ops) { s = 0; ph ^= 1; }
      };
      // the next record is read while one is expanded
      Rec r0, r1;
      int b = b0, dead = 0;
      auto step = [&](const Rec &now, Rec &then) {
        dead = given_up();
        give_back();
        if (b + 1 < b1) take(then);
        wait(w_empty(s), ph);
        tc_fence_after();
        expand(now);
        ++b;
      };
      take(r0);
      while (true) {
        step(r0, r1);
        if (b >= b1 || dead) break;
        step(r1, r0);
        if (b >= b1 || dead) break;
      }
    }
  }
  if (warp >= kFirstAdd) {
    // ------------------------------ sums ------------------------------
    if constexpr (EXACT) regs_up<160>();
    const int row = (warp & 3) * 32 + lane, col0 = (warp - kFirstAdd) / 4 * Cfg::kCols, cols = min(Cfg::kCols, p.bn - col0);
    const int gr = row & 7, quad = row >> 6;
    const uint32_t lane_tmem = tmem + ((uint32_t)((warp & 3) * 32) << 16) + col0;
    int rs = 0, d = 0;
    uint32_t rph = 0, dph = 0;
    for (int u = cl; u < units; u += n_cl) {
      const int quad0 = u % p.row_tiles * 2, n = (quad0 * 4) * 16 + row;
      const int m = quad0 + quad < g.quads ? g.tiles_of(quad0 + quad) : 0;
      // the row's scales in a record: groups 128 bytes apart
      if constexpr (EXACT) {
        const uint32_t sc_at = quad * rec4 + m * 2 * kW4TileBytes + gr * 16 + ((row >> 4) & 3) * 4 + ((row >> 3) & 1) * 2;
        float acc[Cfg::kCols];
#pragma unroll
        for (int i = 0; i < Cfg::kCols; ++i) acc[i] = 0.f;
        // a record's scales, read one record ahead, so that its slot is free as soon as its codes are expanded
        uint32_t sc[4], sc_next[4] = {0, 0, 0, 0};
        auto fetch = [&]() {
          wait(raw_full(rs), rph);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i < per) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(sc_next[i]) : "r"(rec0 + rs * p.raw_bytes + sc_at + i * 128));
          __syncwarp();
          if (lane == 0) mbar_arrive(raw_empty(rs));
          if (++rs == kRaw) { rs = 0; rph ^= 1; }
        };
        fetch();
        for (int b = b0, dead = 0; b < b1 && !dead; ++b) {
          dead = given_up();
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[i] = sc_next[i];
          if (b + 1 < b1) fetch();
#pragma unroll 1
          for (int i = 0; i < per; ++i) {
            const float scale = to_float<BF16>((uint16_t)sc[0]);
            sc[0] = sc[1]; sc[1] = sc[2]; sc[2] = sc[3];
            wait(d_full(d), dph);
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < Cfg::kCols; c += 16) {
              if (c >= cols) break;
              uint32_t v[16];
              tmem_ld16(lane_tmem + d * kW4Acc + c, v);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) acc[c + j] = fmaf(__uint_as_float(v[j]), scale, acc[c + j]);
            }
            if (b + 1 == b1 && i + 1 == per) break;      // (the unit's last accumulator is kept)
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(d_empty(d));
            d ^= 1;
            if (d == 0) dph ^= 1;
          }
        }
        // The sums go back to the accumulator they were last read from, to leave it by a loop of few instructions (written out for every
        // register, the stores were 40 KB of code, which cost more to fetch than to run: 50 us a unit).
#pragma unroll
        for (int c = 0; c < Cfg::kCols; c += 16)
          if (c < cols) tmem_st16f(lane_tmem + d * kW4Acc + c, acc + c);
        tmem_st_wait();
        __syncwarp();
      } else {
        wait(d_full(d), dph);
        tc_fence_after();
      }
      const int tok0 = u / p.row_tiles * p.bn + col0, n_tok = min(cols, a.T - tok0);
      const uint32_t out_tmem = lane_tmem + d * kW4Acc;
      if (cluster == 1) {
        const float bias = a.bias && n < g.n ? to_float<BF16>(a.bias[n]) : 0.f;
        const bool store = n < g.n && !*s_abort;
        using Out = std::conditional_t<EXACT, float, uint16_t>;
        Out *out = static_cast<Out *>(a.y) + (long long)tok0 * a.y_stride + n;
#pragma unroll 1
        for (int c = 0; c < n_tok; c += 16) {
          uint32_t v[16];
          tmem_ld16(out_tmem + c, v);
          tmem_ld_wait();
          if (!EXACT && c == 0) odd = fmaf(__uint_as_float(v[0]), 0.f, odd);
#pragma unroll
          for (int j = 0; j < 16; ++j, out += a.y_stride)
            if (store && c + j < n_tok) {
              const float sum = __uint_as_float(v[j]) + bias;
              if constexpr (EXACT) *out = sum; else *out = from_float<BF16>(sum);
            }
        }
      } else {
        // (one unit a cluster) token c of the tile goes to block c / share, where its sums stand [block][token][row]
        const int share = (p.bn + cluster - 1) / cluster;
        __syncwarp();
        cluster_sync_all();                              // every block is done with its stages
        int owner = col0 / share, left = share - col0 % share;
#pragma unroll 1
        for (int c = 0; c < cols; c += 8) {
          uint32_t v[8];
          tmem_ld8(out_tmem + c, v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t to = stage0 + ((rank * share + share - left) * 128 + row) * 4;
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_u32(to, owner)), "f"(__uint_as_float(v[j])) : "memory");
            if (--left == 0) { left = share; ++owner; }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(d_empty(d));
      d ^= 1;
      if (d == 0) dph ^= 1;
    }
  } else if (cluster > 1) {
    __syncwarp();
    cluster_sync_all();
  }
  __syncwarp();
  abort_drain(s_abort);
  tc_fence_before();
  if (cluster > 1) {
    cluster_sync_all();
    const int share = (p.bn + cluster - 1) / cluster, tok0 = cl / p.row_tiles * p.bn + rank * share;
    const int n_tok = min(min(share, p.bn - rank * share), a.T - tok0), row0 = cl % p.row_tiles * 128;
    const float *part = reinterpret_cast<const float *>(smem);
    if (!*s_abort)
      for (int i = tid; i < n_tok * 128; i += Cfg::kThreads) {
        const int t = i >> 7, n = row0 + (i & 127);
        float v = 0.f;
        for (int r = 0; r < cluster; ++r) v += part[(r * share) * 128 + i];
        if (!EXACT) odd = fmaf(v, 0.f, odd);
        if (n < g.n) w4_store<BF16>(a, tok0 + t, n, v);
      }
  }
  const bool again = __syncthreads_or(!EXACT && odd != odd) && !*s_abort;
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
  if (!EXACT && again) w4_again<BF16>(args, Cfg::kThreads);
}

}  // namespace ftmoe
