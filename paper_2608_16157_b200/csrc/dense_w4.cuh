// Products with 4-bit weights and group scales: y[t][n] = sum_k x[t][k] s[n][k/G] (q[n][k] - z[n][k/G]) + bias[n].
//
// Image of a matrix (w4_pack_kernel), three sections:
//   codes : tiles of 16 rows x 64 k = 512 bytes in the order [group of 128 rows][block of 64 k][tile of the group]; lane (g, q) = 4g + q of a
//           warp owns 16 bytes = 4 words, word j holds rows p and p+8 of the tile, p = g/2 + 4 (g%2), at k = 32 (j/2) + 8q + 4 (j%2) .. +3:
//           the A fragments of one mma.sync m16n8k16, whose rows and K order are free (x in the same order: 16 bytes of a token a lane).
//           Neighbouring g four rows apart: 16-byte stores of a warp to 128-byte-swizzled rows meet no bank twice.
//   scales: [tile][group of k][g] pairs (row p, row p+8) in the activations' type.
//   zeros : the same places, a byte each (only with zero points).
// Rows are padded to 16, k to 64, with scales of 0.
// A word's nibble pairs stand where the top mantissa bits of two 16-bit numbers of exponent 4 are (bits 3 .. 6 for bf16, 6 .. 9 for fp16),
// in place or after one shift or rotation: (w & mask) | magic is the pair 16 + q, from which 16 + z is subtracted exactly.
//
// w4_stream_kernel, up to 16 tokens: weights on M, tokens on N = 8 or 16.  Bound: HBM for large matrices (N K / 2 bytes), launch and
// latency for small ones.
#pragma once
#include "async.cuh"
#include "cluster.cuh"
#include "common.cuh"
#include "dense_norm.cuh"

namespace ftmoe {

constexpr int kW4TileBytes = 512;

struct W4Geom {
  int32_t n, k, kb, tiles, groups, group;       // kb: blocks of 64 k; groups: groups of k in the padded k
  long long scales_at, zeros_at;                // byte offsets in the image
};
inline W4Geom w4_geom(long long n, long long k, int group) {
  W4Geom g;
  g.n = (int)n; g.k = (int)k; g.group = group;
  g.kb = (int)((k + 63) / 64);
  g.tiles = (int)((n + 15) / 16);
  g.groups = g.kb * 64 / group;
  g.scales_at = (long long)g.tiles * g.kb * kW4TileBytes;
  g.zeros_at = g.scales_at + (long long)g.tiles * g.groups * 32;
  return g;
}
// Byte offset of a tile's first block and bytes from block to block.
__host__ __device__ __forceinline__ long long w4_tile_at(const W4Geom &g, int tile, int &step) {
  const int rg = tile >> 3;
  step = min(8, g.tiles - rg * 8) * kW4TileBytes;
  return ((long long)rg * 8 * g.kb) * kW4TileBytes + (tile & 7) * kW4TileBytes;
}

// Position of nibble pair i (0 .. 3) of a word: (low half's bit, high half's bit); a nibble may run over bit 31 to bit 0.
template <bool BF16> __host__ __device__ constexpr int w4_bit(int i) { return BF16 ? (i < 3 ? 3 + 4 * i : 15) : (i == 0 ? 6 : i == 1 ? 10 : i == 2 ? 2 : 14); }

// Row of a tile that lane group g holds (and that plus 8).
__host__ __device__ __forceinline__ constexpr int w4_row(int g) { return (g >> 1) + 4 * (g & 1); }

__device__ __forceinline__ uint32_t rotl32(uint32_t v, int n) { return __funnelshift_l(v, v, n); }

// Codes 16 + q of a word as four pairs: rows g, g+8 at the first two k, then at the next two.
template <bool BF16>
__device__ __forceinline__ void w4_expand(uint32_t w, uint32_t (&p)[4]) {
  const uint32_t mask = BF16 ? 0x00780078u : 0x03c003c0u, magic = BF16 ? 0x41804180u : 0x4c004c00u;
  p[0] = (w & mask) | magic;
  p[1] = ((w >> 4) & mask) | magic;
  p[2] = ((BF16 ? w >> 8 : w << 4) & mask) | magic;
  p[3] = (__funnelshift_r(w, w, BF16 ? 12 : 8) & mask) | magic;
}
template <bool BF16>
__device__ __forceinline__ uint32_t sub_pair(uint32_t a, uint32_t b) {
  uint32_t d;
  if (BF16) asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
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
template <bool BF16>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF16) mma_bf16(c, a[0], a[1], a[2], a[3], b0, b1);
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ---- layout of an image: one thread per lane's 16 bytes, then one per pair of scales ----
template <bool BF16>
__global__ void __launch_bounds__(256) w4_pack_kernel(const W4Geom g, const uint8_t *codes, long long codes_stride, const uint16_t *scales,
                                                      const uint8_t *zeros, uint8_t *image) {
  grid_let_next();
  grid_wait();
  const long long n_code = (long long)g.tiles * g.kb * 32, n_scale = (long long)g.tiles * g.groups * 8;
  const int k_groups = g.k / g.group;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n_code + n_scale; i += (long long)gridDim.x * blockDim.x) {
    if (i < n_code) {
      const int lane = (int)(i & 31), kb = (int)((i >> 5) % g.kb), tile = (int)((i >> 5) / g.kb), row_in = w4_row(lane >> 2), q = lane & 3;
      int step;
      long long at = w4_tile_at(g, tile, step);
      at += (long long)kb * step + lane * 16;
      uint32_t w[4] = {0, 0, 0, 0};
      for (int half = 0; half < 2; ++half) {
        const long long row = (long long)tile * 16 + row_in + 8 * half;
        for (int h = 0; h < 2; ++h) {
          const int k = kb * 64 + 32 * h + 8 * q;
          if (row >= g.n || k >= g.k) continue;
          const uint8_t *src = codes + row * codes_stride + k / 2;
#pragma unroll
          for (int b = 0; b < 4; ++b) {                   // k + 2b, k + 2b + 1: word 2h + b/2, pair 2 (b % 2) + half
            const uint32_t c = src[b];
            const int bit = w4_bit<BF16>(2 * (b & 1) + half);
            w[2 * h + b / 2] |= rotl32(c & 15u, bit) | rotl32(c >> 4, bit + 16);
          }
        }
      }
      *reinterpret_cast<uint4 *>(image + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      const long long s = i - n_code;
      const int gr = (int)(s & 7), kg = (int)((s >> 3) % g.groups);
      const long long tile = (s >> 3) / g.groups;
      uint32_t sc = 0, z = 0;
      for (int half = 0; half < 2; ++half) {
        const long long row = tile * 16 + w4_row(gr) + 8 * half;
        if (row >= g.n || kg >= k_groups) continue;
        sc |= (uint32_t)scales[row * k_groups + kg] << (16 * half);
        if (zeros) z |= min((uint32_t)zeros[row * k_groups + kg], 15u) << (8 * half);
      }
      *reinterpret_cast<uint32_t *>(image + g.scales_at + s * 4) = sc;
      if (zeros) *reinterpret_cast<uint16_t *>(image + g.zeros_at + s * 2) = (uint16_t)z;
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
};

template <bool BF16>
__device__ __forceinline__ void w4_store(const W4Args &a, long long t, int n, float v) {
  if (a.bias) v += to_float<BF16>(a.bias[n]);
  if (a.out32) static_cast<float *>(a.y)[t * a.y_stride + n] = v;
  else static_cast<uint16_t *>(a.y)[t * a.y_stride + n] = from_float<BF16>(v);
}


// Accumulates four words of codes (rows of one tile, 64 k) times x; `lo`, `hi`: 16 + z of the lane's rows per scale group.
template <bool BF16, int NT>
__device__ __forceinline__ void w4_word(uint32_t w, uint32_t lo, uint32_t hi, const uint32_t (*x)[8], int j, float (*sum)[4]) {
  uint32_t p[4];
  w4_expand<BF16>(w, p);
  p[0] = sub_pair<BF16>(p[0], lo); p[1] = sub_pair<BF16>(p[1], hi);
  p[2] = sub_pair<BF16>(p[2], lo); p[3] = sub_pair<BF16>(p[3], hi);
#pragma unroll
  for (int t = 0; t < NT; ++t) mma_16816<BF16>(sum[t], p, x[t][2 * j], x[t][2 * j + 1]);
}

constexpr int kW4Warps = 8, kW4MaxCluster = 8;
// A lane's place in the partial sums of a warp: values of an accumulator apart, so that neighbouring rows are in different banks.
__device__ __forceinline__ constexpr int w4_slot(int part, int e, int lane) { return part * 133 + e * 33 + lane; }

template <bool BF16, int G, bool ZERO, int NT, int R>
__global__ void __launch_bounds__(kW4Warps * 32, 2) w4_stream_kernel(const W4Args a, const int cluster) {
  constexpr int kSub = G < 64 ? 64 / G : 1;                       // scale groups in a block of 64 k
  constexpr int kOut = R * 16 * 8 * NT, kPart = R * NT * 133;     // results of a chunk of R tiles; floats of a warp's partial sums
  __shared__ float s_part[2][kW4Warps][kPart];
  __shared__ float s_join[2][kOut];                               // of a cluster's blocks, each the results that this block finishes
  grid_let_next();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, q = lane & 3, gr = lane >> 2;
  const int rank = blockIdx.x % cluster, n_cl = gridDim.x / cluster, cl = blockIdx.x / cluster;
  if (cluster > 1) cluster_arrive();
  const W4Geom &g = a.g;
  const int t_begin = (int)((long long)g.tiles * cl / n_cl), t_end = (int)((long long)g.tiles * (cl + 1) / n_cl);
  const int chunks = (t_end - t_begin + R - 1) / R, workers = kW4Warps * cluster, me = rank * kW4Warps + warp;
  const int n_k = (g.kb - me + workers - 1) / workers;            // blocks of 64 k of this warp (may be none)
  const int tok0 = blockIdx.y * 8 * NT;
  const uint32_t *scales = reinterpret_cast<const uint32_t *>(a.image + g.scales_at) + gr;
  const uint16_t *zeros = reinterpret_cast<const uint16_t *>(a.image + g.zeros_at) + gr;
  grid_wait();

  struct Buf {
    uint4 w[R];
    uint32_t sc[R][kSub], z[R][kSub], x[NT][8];
  };
  auto load = [&](Buf &b, int c, int i) {
    const int kb = me + i * workers, first = t_begin + c * R;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (first + r >= t_end) break;
      int step;
      const long long at = w4_tile_at(g, first + r, step);
      b.w[r] = ld_stream_16(a.image + at + (long long)kb * step + lane * 16);
#pragma unroll
      for (int s = 0; s < kSub; ++s) {
        const long long sg = ((long long)(first + r) * g.groups + (G >= 64 ? kb / (G / 64) : kb * kSub + s)) * 8;
        b.sc[r][s] = __ldg(scales + sg);
        b.z[r][s] = ZERO ? (uint32_t)__ldg(zeros + sg) : 0u;
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const bool has = tok0 + 8 * t + gr < a.T;
      const uint16_t *x = a.x + (long long)(tok0 + 8 * t + gr) * a.x_stride + kb * 64 + q * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (has && kb * 64 + 32 * h < g.k) v = *reinterpret_cast<const uint4 *>(x + 32 * h);
        b.x[t][4 * h] = v.x; b.x[t][4 * h + 1] = v.y; b.x[t][4 * h + 2] = v.z; b.x[t][4 * h + 3] = v.w;
      }
    }
  };
  float acc[R][NT][4];
  auto clear = [&]() {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][t][e] = 0.f;
  };
  auto compute = [&](const Buf &b, int c) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (t_begin + c * R + r >= t_end) break;
      const uint32_t words[4] = {b.w[r].x, b.w[r].y, b.w[r].z, b.w[r].w};
#pragma unroll
      for (int s = 0; s < kSub; ++s) {
        uint32_t lo = BF16 ? 0x41c041c0u : 0x4e004e00u, hi = lo;      // 16 + 8
        if (ZERO) w4_zero_pairs<BF16>(b.z[r][s], lo, hi);
        float sum[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t][0] = sum[t][1] = sum[t][2] = sum[t][3] = 0.f;
#pragma unroll
        for (int j = s * (4 / kSub); j < (s + 1) * (4 / kSub); ++j) w4_word<BF16, NT>(words[j], lo, hi, b.x, j, sum);
        float s0, s1;
        to_float2<BF16>(b.sc[r][s], s0, s1);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[r][t][0] = fmaf(s0, sum[t][0], acc[r][t][0]);
          acc[r][t][1] = fmaf(s0, sum[t][1], acc[r][t][1]);
          acc[r][t][2] = fmaf(s1, sum[t][2], acc[r][t][2]);
          acc[r][t][3] = fmaf(s1, sum[t][3], acc[r][t][3]);
        }
      }
    }
  };
  // the warps' sums of a chunk, then the blocks' of a cluster
  auto finish = [&](int c) {
    const int buf = c & 1, first = (t_begin + c * R) * 16;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_part[buf][warp][w4_slot(r * NT + t, e, lane)] = acc[r][t][e];
    __syncthreads();
    if (cluster > 1 && c == 0) cluster_wait();
    for (int o = tid; o < kOut; o += kW4Warps * 32) {
      const int n = o % (R * 16), t = o / (R * 16), r = n >> 4, row = n & 7;
      // rows of a tile to lanes: row = (g >> 1) + 4 (g & 1), its half in the accumulator's upper pair
      const int ln = (((row & 3) * 2 + (row >> 2)) << 2) + ((t & 7) >> 1), e = (t & 1) + ((n & 8) >> 2);
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kW4Warps; ++w) v += s_part[buf][w][w4_slot(r * NT + (t >> 3), e, ln)];
      if (cluster == 1) {
        if (tok0 + t < a.T && first + n < min(g.n, t_end * 16)) w4_store<BF16>(a, tok0 + t, first + n, v);
      } else {
        const int owner = (o >> 5) % cluster, at = rank * (kOut / cluster) + (o >> 5) / cluster * 32 + (o & 31);
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_u32(smem_u32(&s_join[buf][at]), owner)), "f"(v) : "memory");
      }
    }
    if (cluster > 1) {
      cluster_sync_all();
      const int share = kOut / cluster;
      for (int i = tid; i < share; i += kW4Warps * 32) {
        const int o = ((i >> 5) * cluster + rank) * 32 + (i & 31), n = o % (R * 16), t = o / (R * 16);
        float v = 0.f;
        for (int w = 0; w < cluster; ++w) v += s_join[buf][w * share + i];
        if (tok0 + t < a.T && first + n < min(g.n, t_end * 16)) w4_store<BF16>(a, tok0 + t, first + n, v);
      }
    }
  };

  clear();
  if (n_k <= 0) {
    for (int c = 0; c < chunks; ++c) finish(c);
    return;
  }
  // one step ahead: the loads of the next block of k, or of the next chunk's first, are on their way
  Buf b0, b1;
  int c = 0, i = 0;
  auto step = [&](const Buf &now, Buf &next) {
    const bool last = i + 1 == n_k;
    const int nc = last ? c + 1 : c, ni = last ? 0 : i + 1;
    if (nc < chunks) load(next, nc, ni);
    compute(now, c);
    if (last) {
      finish(c);
      clear();
    }
    c = nc;
    i = ni;
  };
  if (chunks > 0) load(b0, 0, 0);
  while (c < chunks) {
    step(b0, b1);
    if (c >= chunks) break;
    step(b1, b0);
  }
}

}  // namespace ftmoe
