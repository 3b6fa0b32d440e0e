// Products with 4-bit weights and group scales: y[t][n] = sum_k x[t][k] s[n][k/G] (q[n][k] - z[n][k/G]) + bias[n].
//
// Image of a matrix (w4_pack_kernel): for each quad (64 rows: four tiles of 16, the last quad with as many as there are rows for) and each
// block of 128 k, one contiguous record:
//   codes : [half of 64 k][tile] 512 bytes; lane (g, q) = 4g + q of a warp owns 16 of them = 4 words, word j holds rows g and g+8 of the tile at
//           k = 16j + 4q .. +3 of the half: the A fragments of one mma.sync m16n8k16, whose K order is free (x in the same order: 8 bytes of a
//           token a lane), and what a lane writes to tensor memory for 16 rows x 16 k
//   scales: [group of k][g][4 tiles] pairs (row g, row g+8) in the activations' type: 16 bytes a lane for four tiles
//   zeros : the same places, a byte each (only with zero points)
// Rows are padded to 16, k to 128, with scales of 0.  A quad's records follow one another along k: a warp's share of a row of quads is one
// stretch of memory.
// A word's nibble pairs stand where the top mantissa bits of two 16-bit numbers of exponent 4 are (bits 3 .. 6 for bf16, 6 .. 9 for fp16),
// in place or after one shift or rotation: (w & mask) | magic is the pair 16 + q, from which 16 + z is subtracted exactly.
//
// w4_stream_kernel, up to 16 tokens (32 for float results): weights on M, tokens on N = 8, 16 or 32.  Bound: HBM for large matrices (N K / 2
// bytes), launch and latency for small ones.  Measured: 37 us for 5 tokens through 2048 x 150001 (4.5 TB/s; 18.5 instructions per 256 weights)
// and 55 for 16, 4.7 us for one token through 2048 x 5120, 9.9 us through 7168 x 7168.
#pragma once
#include <type_traits>

#include "async.cuh"
#include "cluster.cuh"
#include "common.cuh"
#include "dense_norm.cuh"

namespace ftmoe {

constexpr int kW4TileBytes = 512, kW4Block = 128;
constexpr uint32_t kWithholdW4Stream = 1u, kWithholdW4Tile = 2u;   // ft_dense_debug_inject

struct W4Geom {
  int32_t n, k, nb, tiles, quads, group, zeros;   // nb: blocks of 128 k
  int32_t extra;                                  // bytes of a record behind its codes
  __host__ __device__ __forceinline__ int tiles_of(int quad) const { const int m = tiles - 4 * quad; return m < 4 ? m : 4; }
  // bytes of a record of m tiles
  __host__ __device__ __forceinline__ int record(int m) const { return m * 2 * kW4TileBytes + extra; }
  // the first record of a quad
  __host__ __device__ __forceinline__ long long quad_at(int quad) const { return (long long)quad * nb * record(4); }
  __host__ __device__ __forceinline__ long long bytes() const { return quad_at(quads - 1) + (long long)nb * record(tiles_of(quads - 1)); }
};
inline W4Geom w4_geom(long long n, long long k, int group, bool zeros) {
  W4Geom g;
  g.n = (int)n; g.k = (int)k; g.group = group; g.zeros = zeros ? 1 : 0;
  g.nb = (int)((k + kW4Block - 1) / kW4Block);
  g.tiles = (int)((n + 15) / 16);
  g.quads = (g.tiles + 3) / 4;
  g.extra = kW4Block / group * (zeros ? 192 : 128);
  return g;
}

// Position of nibble pair i (0 .. 3) of a word: (low half's bit, high half's bit); a nibble may run over bit 31 to bit 0.
template <bool BF16> __host__ __device__ constexpr int w4_bit(int i) { return BF16 ? (i < 3 ? 3 + 4 * i : 15) : (i == 0 ? 6 : i == 1 ? 10 : i == 2 ? 2 : 14); }

__device__ __forceinline__ uint32_t rotl32(uint32_t v, int n) { return __funnelshift_l(v, v, n); }

// The two constants of the expansion, kept in registers (an instruction takes only one as a literal).
template <bool BF16>
struct W4Const {
  uint32_t mask, magic;
  __device__ __forceinline__ W4Const() {
    asm volatile("mov.b32 %0, %1;" : "=r"(mask) : "n"(BF16 ? 0x00780078 : 0x03c003c0));
    asm volatile("mov.b32 %0, %1;" : "=r"(magic) : "n"(BF16 ? 0x41804180 : 0x4c004c00));
  }
  __device__ __forceinline__ uint32_t pick(uint32_t w) const {       // (w & mask) | magic
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "r"(mask), "r"(magic));
    return d;
  }
};
// Codes 16 + q of a word as four pairs: rows g, g+8 at the first two k, then at the next two.
template <bool BF16>
__device__ __forceinline__ void w4_expand(const W4Const<BF16> &c, uint32_t w, uint32_t (&p)[4]) {
  p[0] = c.pick(w);
  p[1] = c.pick(w >> 4);
  p[2] = c.pick(BF16 ? w >> 8 : w << 4);
  p[3] = c.pick(__funnelshift_r(w, w, BF16 ? 12 : 8));
}
template <bool BF16>
__device__ __forceinline__ uint32_t sub_pair(uint32_t a, uint32_t b) {
  uint32_t d;
  if (BF16) asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <bool BF16>
__device__ __forceinline__ uint32_t mul_pair(uint32_t a, uint32_t b) {
  uint32_t d;
  if (BF16) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// 16 + z of both rows of a pair of zero-point bytes, each as a pair.
template <bool BF16>
__device__ __forceinline__ void w4_zero_pairs(uint32_t z, uint32_t &lo, uint32_t &hi) {
  const uint32_t magic = BF16 ? 0x4180u : 0x4c00u;
  const int sh = BF16 ? 3 : 6;
  lo = ((z & 0xffu) << sh | magic) * 0x10001u;
  hi = (((z >> 8) & 0xffu) << sh | magic) * 0x10001u;
}
// d = a b + c
template <bool BF16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float *c) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// ---- layout of an image: a warp per record ----
template <bool BF16>
__global__ void __launch_bounds__(256) w4_pack_kernel(const W4Geom g, const uint8_t *codes, long long codes_stride, const uint16_t *scales,
                                                      const uint8_t *zeros, uint8_t *image) {
  grid_let_next();
  grid_wait();
  const int lane = threadIdx.x & 31, gr = lane >> 2, q = lane & 3, k_groups = g.k / g.group, per = kW4Block / g.group;
  const long long records = (long long)g.quads * g.nb, warps = (long long)gridDim.x * (blockDim.x / 32);
  for (long long i = (long long)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32; i < records; i += warps) {
    const int quad = (int)(i / g.nb), block = (int)(i - (long long)quad * g.nb), m = g.tiles_of(quad);
    uint8_t *rec = image + g.quad_at(quad) + (long long)block * g.record(m);
    for (int part = 0; part < 2 * m; ++part) {           // 64 k of a tile
      const int tile = quad * 4 + part % m;
      uint32_t w[4] = {0, 0, 0, 0};
      for (int half = 0; half < 2; ++half) {
        const long long row = (long long)tile * 16 + gr + 8 * half;
        for (int j = 0; j < 4; ++j) {
          const int k = block * kW4Block + part / m * 64 + 16 * j + 4 * q;
          if (row >= g.n || k >= g.k) continue;            // (k is a multiple of 32)
          const uint8_t *src = codes + row * codes_stride + k / 2;
#pragma unroll
          for (int b = 0; b < 2; ++b) {                     // k + 2b, k + 2b + 1: pair 2b + half
            const uint32_t c = src[b];
            const int bit = w4_bit<BF16>(2 * b + half);
            w[j] |= rotl32(c & 15u, bit) | rotl32(c >> 4, bit + 16);
          }
        }
      }
      *reinterpret_cast<uint4 *>(rec + part * kW4TileBytes + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    uint8_t *sc = rec + 2 * m * kW4TileBytes;
    for (int s = 0; s < per; ++s) {                         // lane (g, q): row pair g of tile q
      const int kg = block * per + s;
      uint32_t v = 0, z = 0;
      for (int half = 0; half < 2; ++half) {
        const long long row = (long long)(quad * 4 + q) * 16 + gr + 8 * half;
        if (row >= g.n || kg >= k_groups) continue;
        v |= (uint32_t)scales[row * k_groups + kg] << (16 * half);
        if (zeros) z |= min((uint32_t)zeros[row * k_groups + kg], 15u) << (8 * half);
      }
      reinterpret_cast<uint32_t *>(sc)[s * 32 + lane] = v;
      if (zeros) reinterpret_cast<uint16_t *>(sc + per * 128)[s * 32 + lane] = (uint16_t)z;
    }
  }
}

struct W4Args {
  W4Geom g;
  int32_t T, out32;
  const uint16_t *x, *bias;
  const uint8_t *image;
  void *y;
  long long x_stride, y_stride;
  uint32_t *status;
};

template <bool BF16>
__device__ __forceinline__ void w4_put(const W4Args &a, long long t, int n, float v) {
  if (a.out32) static_cast<float *>(a.y)[t * a.y_stride + n] = v;
  else static_cast<uint16_t *>(a.y)[t * a.y_stride + n] = from_float<BF16>(v);
}
template <bool BF16>
__device__ __forceinline__ void w4_store(const W4Args &a, long long t, int n, float v) {
  w4_put<BF16>(a, t, n, a.bias ? v + to_float<BF16>(a.bias[n]) : v);
}


constexpr int kW4MaxCluster = 8, kW4MaxSlots = 6;
// Warps of a block: 16, or 8 with twice the registers where the sums of 32 tokens have to be held.
template <int NT> constexpr int kW4Warps = NT > 2 ? 8 : 16;
// A lane's place in the partial sums of a warp: values of an accumulator apart, so that neighbouring rows are in different banks.
__device__ __forceinline__ constexpr int w4_slot(int part, int e, int lane) { return part * 133 + e * 33 + lane; }
constexpr int kW4PartBytes = 8 * 133 * 4;                        // of 8 accumulators

struct W4Stream {        // how the quads are shared out
  int32_t cluster, wk;   // blocks of a cluster and warps of each that share a quad's k
  int32_t slots, slot_bytes;
};
// Shares the quads out.  A warp of a group of `workers` does ceil(nb / workers) records of each of its group's quads, then the group adds its
// sums, which takes about as long as a record (two, over a cluster); the split with the least of both is taken, and of equals the one with the
// fewer warps to a quad.  `clusters`: how many clusters of a size the GPU holds at once.
inline void w4_stream_share(const W4Geom &g, const int *clusters, int warps, W4Stream &s) {
  double best = 1e30;
  auto consider = [&](int cluster, int wk) {
    const int groups = clusters[cluster] * (warps / wk), workers = cluster * wk;
    if (groups == 0 || (workers > 1 && workers >= 2 * g.nb)) return;
    const double cost = (double)((g.quads + groups - 1) / groups) * ((g.nb + workers - 1) / workers + (workers == 1 ? 0.5 : cluster == 1 ? 1. : 2.));
    if (cost < best) { best = cost; s.cluster = cluster; s.wk = wk; }
  };
  for (int wk = 1; wk <= warps; wk *= 2) consider(1, wk);
  for (int cluster = 2; cluster <= kW4MaxCluster; ++cluster) consider(cluster, warps);
}
template <int NT> constexpr int kW4Join = 64 * 8 * NT + 32 * kW4MaxCluster;     // floats of a buffer of sums of a cluster's blocks
// The slots' size and number, as many as fit; returns the bytes of dynamic shared memory.
template <int NT>
inline int w4_stream_memory(const W4Geom &g, W4Stream &s) {
  const int rec = g.record(4), rest = kW4Warps<NT> * kW4MaxSlots * 8 + 8 + kW4Warps<NT> * 4 + (s.cluster > 1 ? 2 * kW4Join<NT> * 4 : 0);
  s.slot_bytes = ((rec > kW4PartBytes ? rec : kW4PartBytes) + 127) / 128 * 128;
  s.slots = (227 * 1024 - rest) / (kW4Warps<NT> * s.slot_bytes);
  const int most = kW4MaxSlots * 8 / kW4Warps<NT>;
  if (s.slots > most) s.slots = most;
  return kW4Warps<NT> * s.slots * s.slot_bytes + rest;
}

// A block of 16 warps an SM.  `wk` warps of each block of a cluster share the k of a quad of 64 rows: each takes its records along k in turn,
// which bulk copies bring into slots of its own, up to three ahead, so that no warp waits for another but for the sums at a quad's end:
// those are left in the slot just read, and added in a fixed order.
template <bool BF16, int G, bool ZERO, int NT>
__global__ void __launch_bounds__(kW4Warps<NT> * 32, 1) w4_stream_kernel(const W4Args a, const W4Stream p) {
  constexpr int kGroups = kW4Block / G, kSub = G < 64 ? 64 / G : 1;      // scale groups of a record; of 64 k
  constexpr int kTiles = NT > 2 ? 2 : 4, kRounds = 4 / kTiles;           // tiles whose sums are added at a time
  constexpr int kOut = kTiles * 16 * 8 * NT;                             // results of a round
  extern __shared__ __align__(128) unsigned char smem[];
  grid_let_next();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, q = lane & 3, gr = lane >> 2;
  const W4Geom &g = a.g;
  const int cluster = p.cluster, rank = blockIdx.x % cluster, wk = p.wk;
  const int per_block = kW4Warps<NT> / wk, group = blockIdx.x / cluster * per_block + warp / wk, n_groups = (int)gridDim.x / cluster * per_block;
  const int first_warp = warp / wk * wk, me = rank * wk + warp % wk, workers = wk * cluster;
  const int n_b = (g.nb - me + workers - 1) / workers;                   // records of this warp in a quad (none where k is short)
  const int tok0 = blockIdx.y * 8 * NT;
  unsigned char *s_slot = smem + warp * p.slots * p.slot_bytes;
  uint64_t *s_bar = reinterpret_cast<uint64_t *>(smem + kW4Warps<NT> * p.slots * p.slot_bytes);
  volatile int *s_abort = reinterpret_cast<volatile int *>(s_bar + kW4Warps<NT> * kW4MaxSlots);
  int *s_held = reinterpret_cast<int *>(s_bar + kW4Warps<NT> * kW4MaxSlots + 1);      // where each warp's sums are
  float *s_join = reinterpret_cast<float *>(s_held + kW4Warps<NT>);                   // the sums of a cluster's blocks that this one adds
  const uint32_t bars = smem_u32(s_bar + warp * kW4MaxSlots);
  if (tid == 0) *s_abort = 0;
  if (lane == 0) {
    for (int s = 0; s < p.slots; ++s) mbar_init(bars + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (cluster > 1) cluster_sync_all(); else __syncthreads();
  const W4Const<BF16> con;
  // the record to bring next
  int in_quad = group, in_left = n_b, in_slot = 0, in_bytes = 0;
  const uint8_t *in_at = nullptr;
  auto enter = [&]() {
    if (in_quad >= g.quads) return;
    in_bytes = g.record(g.tiles_of(in_quad));
    in_at = a.image + g.quad_at(in_quad) + (long long)me * in_bytes;
    in_left = n_b;
  };
  const uint32_t slots_at = smem_u32(s_slot);
  bool withhold = blockIdx.x == 0 && blockIdx.y == 0 && warp == 0 && (g_debug_withhold & kWithholdW4Stream);
  auto bring = [&]() {
    if (in_quad >= g.quads) return;
    if (lane == 0 && !*s_abort) {
      mbar_expect_tx(bars + 8 * in_slot, in_bytes);
      if (!withhold) bulk_g2s(slots_at + in_slot * p.slot_bytes, in_at, in_bytes, bars + 8 * in_slot);     // (withheld: test hook)
      withhold = false;
    }
    if (++in_slot == p.slots) in_slot = 0;
    in_at += workers * in_bytes;
    if (--in_left == 0) { in_quad += n_groups; enter(); }
  };
  // the lane's tokens; those past the last one read it again: their results are not stored
  const uint16_t *x_at[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) x_at[t] = a.x + (long long)min(tok0 + 8 * t + gr, a.T - 1) * a.x_stride + q * 4;
  grid_wait();
  if (n_b > 0) {
    enter();
    for (int s = 0; s < p.slots; ++s) bring();
  }
  auto wait = [&](int slot, uint32_t phase) {
    if (mbar_try_wait(bars + 8 * slot, phase)) return;
    mbar_wait(bars + 8 * slot, phase, s_abort, a.status);
  };
  auto group_sync = [&]() {
    if (wk == kW4Warps<NT>) __syncthreads();
    else if (wk > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / wk), "r"(wk * 32) : "memory");
    else __syncwarp();
  };

  const int share = (kOut / 32 + cluster - 1) / cluster * 32;           // results that a block of a cluster finishes
  int slot = 0, turn = 0;
  uint32_t phase = 0;
  for (int quad = group; quad < g.quads; quad += n_groups) {
    const int m = g.tiles_of(quad);
    float acc[4][NT][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][t][e] = 0.f;
    int held = -1;
    for (int i = 0; i < n_b; ++i) {
      const int b = me + i * workers;
      constexpr int kHalves = NT > 2 ? 1 : 2;
      uint32_t x[kHalves][NT][8];
      auto load_x = [&](int half, uint32_t (&xr)[NT][8]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint16_t *src = x_at[t] + b * kW4Block + half * 64;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint2 v = make_uint2(0u, 0u);
            if (G == kW4Block || b * kW4Block + half * 64 + 16 * j < g.k) v = *reinterpret_cast<const uint2 *>(src + 16 * j);
            xr[t][2 * j] = v.x; xr[t][2 * j + 1] = v.y;
          }
        }
      };
      load_x(0, x[0]);
      if constexpr (kHalves == 2) load_x(1, x[1]);
      wait(slot, phase);
      const uint32_t rec = slots_at + slot * p.slot_bytes;
      // full quads without a test between the tiles, so that their chains overlap
      auto multiply = [&](const int m, auto full) {
        const uint32_t sc_at = rec + m * 2 * kW4TileBytes;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (kHalves == 1 && half == 1) load_x(1, x[0]);
          const uint32_t (&xr)[NT][8] = x[kHalves == 2 ? half : 0];
          uint4 sc[kSub];
          uint2 z[kSub];
#pragma unroll
          for (int s = 0; s < kSub; ++s) {
            const int at = half * kGroups / 2 + s;
            sc[s] = lds_v4(sc_at + at * 128 + gr * 16);
            if (ZERO) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(z[s].x), "=r"(z[s].y) : "r"(sc_at + kGroups * 128 + at * 64 + gr * 8));
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (!decltype(full)::value && r >= m) break;
            const uint4 w = lds_v4(rec + (half * m + r) * kW4TileBytes + lane * 16);
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int s = 0; s < kSub; ++s) {
              uint32_t lo = BF16 ? 0x41c041c0u : 0x4e004e00u, hi = lo;      // 16 + 8
              if (ZERO) w4_zero_pairs<BF16>((r < 2 ? z[s].x : z[s].y) >> (16 * (r & 1)), lo, hi);
              float sum[NT][4];
#pragma unroll
              for (int j = s * (4 / kSub); j < (s + 1) * (4 / kSub); ++j) {
                uint32_t c[4];
                w4_expand<BF16>(con, words[j], c);
                c[0] = sub_pair<BF16>(c[0], lo); c[1] = sub_pair<BF16>(c[1], hi);
                c[2] = sub_pair<BF16>(c[2], lo); c[3] = sub_pair<BF16>(c[3], hi);
                const float none[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_16816<BF16>(sum[t], c, xr[t][2 * j], xr[t][2 * j + 1], j == s * (4 / kSub) ? none : sum[t]);
              }
              float s0, s1;
              to_float2<BF16>(r == 0 ? sc[s].x : r == 1 ? sc[s].y : r == 2 ? sc[s].z : sc[s].w, s0, s1);
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                acc[r][t][0] = fmaf(s0, sum[t][0], acc[r][t][0]);
                acc[r][t][1] = fmaf(s0, sum[t][1], acc[r][t][1]);
                acc[r][t][2] = fmaf(s1, sum[t][2], acc[r][t][2]);
                acc[r][t][3] = fmaf(s1, sum[t][3], acc[r][t][3]);
              }
            }
          }
        }
      };
      if (NT == 1 && m == 4) multiply(4, std::true_type());
      else multiply(m, std::false_type());
      __syncwarp();
      if (i + 1 < n_b) bring(); else held = slot;     // (the last one of a quad holds the sums first)
      if (++slot == p.slots) { slot = 0; phase ^= 1u; }
    }
    if (workers == 1) {              // the warp has the whole sums
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int n = (quad * 4 + r) * 16 + gr + (e & 2) * 4;
          if (n >= g.n) continue;
          const float bias = a.bias ? to_float<BF16>(a.bias[n]) : 0.f;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int tok = tok0 + 8 * t + 2 * q + (e & 1);
            if (tok < a.T) w4_put<BF16>(a, tok, n, acc[r][t][e] + bias);
          }
        }
      bring();
      continue;
    }
    // the warps' sums of the quad, then the blocks' of a cluster
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
      const int row0 = (quad * 4 + round * kTiles) * 16;
      if (held >= 0) {
        float *part = reinterpret_cast<float *>(s_slot + held * p.slot_bytes);
#pragma unroll
        for (int r = 0; r < kTiles; ++r)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[w4_slot(r * NT + t, e, lane)] = acc[round * kTiles + r][t][e];
      }
      if (lane == 0) s_held[warp] = (warp * p.slots + held) * p.slot_bytes;
      group_sync();
      const int n_hold = max(0, min(wk, g.nb - rank * wk));             // warps of the group that had records
      for (int o = (warp - first_warp) * 32 + lane; o < kOut; o += wk * 32) {
        // result o: row n and token t; where an accumulator of the warps has it
        const int n = o % (kTiles * 16), t = o / (kTiles * 16);
        const int at = w4_slot((n >> 4) * NT + (t >> 3), (t & 1) + ((n & 8) >> 2), (n & 7) * 4 + ((t & 7) >> 1));
        float v = 0.f;
        for (int w = 0; w < n_hold; ++w) v += reinterpret_cast<const float *>(smem + s_held[first_warp + w])[at];
        if (cluster == 1) {
          if (tok0 + t < a.T && row0 + n < g.n) w4_store<BF16>(a, tok0 + t, row0 + n, v);
        } else {
          const int owner = (o >> 5) % cluster, to = turn * kW4Join<NT> + rank * share + (o >> 5) / cluster * 32 + (o & 31);
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_u32(smem_u32(s_join + to), owner)), "f"(v) : "memory");
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // (the slot's next contents come by a bulk copy)
      if (cluster > 1) {
        cluster_sync_all();
        for (int i = tid; i < share; i += kW4Warps<NT> * 32) {
          const int o = ((i >> 5) * cluster + rank) * 32 + (i & 31);
          if (o >= kOut) break;
          const int n = o % (kTiles * 16), t = o / (kTiles * 16);
          float v = 0.f;
          for (int w = 0; w < cluster; ++w) v += s_join[turn * kW4Join<NT> + w * share + i];
          if (tok0 + t < a.T && row0 + n < g.n) w4_store<BF16>(a, tok0 + t, row0 + n, v);
        }
        turn ^= 1;
      } else {
        group_sync();
      }
    }
    if (held >= 0) bring();
  }
  abort_drain(s_abort);
}

}  // namespace ftmoe
