// Attention of requests with few query rows (n tokens x Hq/Hkv heads <= 16: single tokens, short drafts) over the paged
// cache.  Every key and value is needed once per 16 rows and used for 4*16*D flops per 4*D bytes: bound by HBM.
//
// The key blocks (64 keys) of all requests and key/value heads form one flat list that is cut into equal shares, one
// CTA per SM (the work partition of attn_plan.cuh), so the cache streams at an even rate whatever the lengths are.  A
// producer warp brings a block's pages with TMA tile loads (128-byte swizzle) into a ring of 160 KB; the consumer
// warps take 16 keys each of a block: S = Q K^T and O += P V with mma.sync m16n8k16 (the rows on M), the running maximum
// m and sum l of every row per warp:
//   m' = max(m, max_j s_j),  l' = l 2^(m-m') + sum_j 2^(s_j-m'),  O' = O 2^(m-m') + sum_j 2^(s_j-m') v_j,  s in units of log2
// P is rounded to the values' type for the second product (relative 2^-9 of each weight on average, below the rounding of
// the result); l sums the unrounded weights; everything else stays in 32 bits.
// At the end of a (request, head) the warps' (m, l, O) are joined in shared memory.  A request that was cut leaves its
// parts in global memory; the CTA that arrives last (a counter per request and head) joins them in the order of the
// CTAs, so results do not depend on who is last.
// Measured (32 query and 4 kv heads of 128): 302 us for 128 requests with 2.03 GB of cache (6.74 TB/s, the rate of a copy), 17.4 us for 8
// requests of 4000 tokens, 8.2 us for one of 1000, where launch, tables, first block and join follow one another.  More rows a
// request (several tiles in a warp, or a group of warps each) lose against the tiled kernel on long contexts: 283 and 300 against
// 247 us for 16 drafts of 5 rows x 8 heads of 64 over 32768 tokens.
// Values that no row attends to (behind the last token, before a window) are zeroed in shared memory before use: their
// weights are 0, but what stands there may be NaN.
#pragma once
#include "attn_plan.cuh"
#include "attn_rope.cuh"
#include "tcgen.cuh"

namespace ftmoe {

struct AttnFwdArgs {
  AttnWork w;
  int32_t n_q, n_kv, group, page_shift, n_pages, window;
  const uint16_t *q, *cache;
  long long q_stride, out_stride, table_stride;
  const int32_t *table;
  uint16_t *out;
  float *lse;
  float scale_log2;       // scale * log2(e)
  float *part;            // partial results of cut requests
  uint32_t *arrive;       // arrival counters, zero between launches
  uint32_t *status;
};

constexpr uint32_t kWithholdAttnStream = 1u, kWithholdAttnTile = 2u;
template <int D> struct StreamCfg {
  // four warps share a block's keys; with D = 64, where a block is half the bytes but nearly the same chain of latencies, two such
  // groups take the blocks in turn (one group: 850 clocks a block where HBM gives one in 700)
  static constexpr int kGroups = D == 128 ? 1 : 2;
  static constexpr int kWarps = 4 * kGroups, kConsumers = kWarps * 32, kThreads = kConsumers + 32;
  static constexpr int kHalf = kDecKeys * D * 2;            // bytes of the keys (or values) of a block
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = D == 128 ? 5 : 10;
  static constexpr int kRow = D + 8;                        // floats per row of the join buffer (bank-conflict free)
  static constexpr int kJoin = kWarps * kDecRows * kRow * 4;
  static constexpr int kSmem = 1024 + kStages * kStage + kJoin + kWarps * kDecRows * 8 + 2 * kStages * 8 + 64;
  static constexpr int kPart = kDecRows * (D + 2);          // floats of one partial result: m[16], l[16], O[16][D]
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ void mma_16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF16)
    mma_bf16(c, a[0], a[1], a[2], a[3], b0, b1);
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *tm, int x, int y, int z, int v, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(tm), "r"(x), "r"(y), "r"(z), "r"(v), "r"(w), "r"(bar)
      : "memory");
}
// Of a row with reference m (log2 units) and sum l: the factor of its results and log(sum_j exp(s_j)).  Only an empty sum is a
// row that attends to nothing; a sum that is not a number (an infinite or NaN score) stays one.
__device__ __forceinline__ float row_inv(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f; }

// Bounded wait without anything between the polls (limit: g_wait_polls, read once): a wait is on the critical path of every
// block several times.  Returns false, after latching, if the phase never completes.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, uint32_t limit, volatile int *abort_flag, uint32_t *status) {
  for (uint32_t i = 0; i <= limit; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (__builtin_expect((i & 255u) == 255u, 0) && *abort_flag) return false;
  }
  *abort_flag = 1;
  atomicOr(status, kStatTimeout);
  return false;
}
__device__ __forceinline__ void named_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }

template <int D, bool BF16>
__global__ void __launch_bounds__(StreamCfg<D>::kThreads, 1)
attn_stream_kernel(const __grid_constant__ CUtensorMap tm, const AttnFwdArgs a) {
  using Cfg = StreamCfg<D>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float *s_join = reinterpret_cast<float *>(smem + Cfg::kStages * Cfg::kStage);
  float *s_ml = s_join + Cfg::kJoin / 4;                                  // [warp][16][m, l]
  uint64_t *s_bar = reinterpret_cast<uint64_t *>(s_ml + Cfg::kWarps * kDecRows * 2);
  volatile int *s_abort = reinterpret_cast<volatile int *>(s_bar + 2 * Cfg::kStages);
  volatile int *s_last = s_abort + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t ring = smem_u32(smem), bars = smem_u32(s_bar);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (Cfg::kStages + s); };

  grid_let_next();
  if (tid == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 4); }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  grid_wait();
  const AttnPlanHdr hdr = *a.w.hdr;
  const AttnStart start = a.w.dec_start[blockIdx.x];     // (stale beyond the shares in use: not looked at)
  const long long u_first = (long long)blockIdx.x * hdr.dec_quota;
  if (u_first >= hdr.dec_units) return;
  const int u_end = (int)min(u_first + hdr.dec_quota, (long long)hdr.dec_units);

  const int page_tokens = 1 << a.page_shift;
  const int box_shift = min(a.page_shift, 6), box_rows = 1 << box_shift, boxes = kDecKeys >> box_shift;   // boxes of a block
  WorkWalk w;
  w.start(start);
  int s = 0;            // stage of the next block and its phase
  uint32_t ph = 0;
  const uint32_t limit = g_wait_polls;

  if (warp == Cfg::kWarps) {
    // ------------------------------ producer ------------------------------
    const bool hook = g_debug_withhold & kWithholdAttnStream;
    // one 5-D box per page (or 64 tokens of one): 64 elements, tokens, 64-element chunks of D, keys and values
    for (; w.load(hdr.n_dec, a.n_kv, kDecCost, u_end); w.next(a.n_kv, u_end)) {
      const AttnEntry &e = w.e;
      const int blk = w.blk, take = w.take, head = w.head;
      const int hi = max(0, e.pos0 + e.n_tok), lo = a.window > 0 ? max(0, e.pos0 - a.window + 1) : 0;
      const int32_t *row = a.table + (long long)e.req * a.table_stride;
      bool withhold = hook && w.k == 0 && head == 0 && blk == 0;
      // the lanes hold the pages of the boxes of 32 / boxes blocks at a time, the next ones on their way
      const int per = 32 >> (6 - box_shift);
      auto pages_of = [&](int b) -> int {
        const int key = (e.b0 + b) * kDecKeys + lane * box_rows;
        return key < hi && key + box_rows > lo ? row[key >> a.page_shift] : 0;
      };
      int pages = 0, next = pages_of(blk), i0 = 0;
      for (int b = blk; b < blk + take; ++b, i0 += boxes) {
        if (((b - blk) & (per - 1)) == 0) {
          pages = next;
          i0 = 0;
          if (b + per < blk + take) next = pages_of(b + per);
          if ((uint32_t)pages >= (uint32_t)a.n_pages) {                // never followed: a box beyond the pool, which is zeros
            atomicOr(a.status, kStatBadIndex);
            pages = a.n_pages;
          }
        }
        const int key0 = (e.b0 + b) * kDecKeys;
        const int first = max(0, lo - key0) >> box_shift, last = min(boxes, (max(0, hi - key0) + box_rows - 1) >> box_shift);
        wait_phase(empty_bar(s), ph ^ 1u, limit, s_abort, a.status);
        if (*s_abort) break;
        if (elect_one()) mbar_expect_tx(full_bar(s), (uint32_t)(max(0, last - first) * box_rows * D * 4));
        __syncwarp();
        const bool skip = withhold;                                    // test hook: the block's copies never come
        withhold = false;
        for (int i = first; i < last && !skip; ++i) {
          const int z = __shfl_sync(0xffffffffu, pages, i0 + i) * 2 * a.n_kv + head;
          if (elect_one())
            tma_load_5d(ring + s * Cfg::kStage + i * box_rows * D * 4, &tm, 0, (key0 + i * box_rows) & (page_tokens - 1), 0, 0, z, full_bar(s));
          __syncwarp();
        }
        if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
      }
      if (*s_abort) break;
      w.fetch(a.w.dec, hdr.n_dec, a.n_kv, u_end);
    }
    // copies of a CTA that gave up must land before its shared memory goes away
    abort_drain(s_abort);
    return;
  }

  // ------------------------------ consumers ------------------------------
  const int g = lane >> 2, t4 = lane & 3;
  // this warp's 16 keys of a block: in box key0 / box_rows, whose parts are [keys, values][chunk of D][token][64 elements]
  const int key0 = (warp & 3) * 16, chunk = box_rows * 128;
  const uint32_t my_keys = (key0 >> box_shift) * (box_rows * D * 4) + (key0 & (box_rows - 1)) * 128, my_values = my_keys + box_rows * D * 2;
  for (; w.load(hdr.n_dec, a.n_kv, kDecCost, u_end); w.next(a.n_kv, u_end)) {
    w.fetch(a.w.dec, hdr.n_dec, a.n_kv, u_end);
    const AttnEntry &e = w.e;
    const int blk = w.blk, take = w.take, head = w.head;
    const int hi = max(0, e.pos0 + e.n_tok), lo = a.window > 0 ? max(0, e.pos0 - a.window + 1) : 0;
    const int rows = e.n_tok * a.group;
    // query fragments: row r = token r / group, head of the group r % group
    uint32_t q[D / 16][4];
    int pos[2];
    {
      const uint16_t *qp[2];
      bool ok[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = g + 8 * i, tok = r / a.group;
        ok[i] = r < rows;
        pos[i] = ok[i] ? e.pos0 + tok : -1;
        qp[i] = a.q + (long long)(e.tok0 + (ok[i] ? tok : 0)) * a.q_stride + (head * a.group + (ok[i] ? r - tok * a.group : 0)) * D;
      }
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          q[kk][i] = ok[i & 1] ? *reinterpret_cast<const uint32_t *>(qp[i & 1] + kk * 16 + (i >> 1) * 8 + t4 * 2) : 0u;
    }
    float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;

    for (int b = blk; b < blk + take; ++b) {
      const int st = s;
      const uint32_t st_ph = ph;
      if (++s == Cfg::kStages) { s = 0; ph ^= 1u; }
      if (Cfg::kGroups > 1 && (st & 1) != (warp >> 2)) continue;     // (an even number of stages then)
      const bool ok = wait_phase(full_bar(st), st_ph, limit, s_abort, a.status);
      const uint32_t kt = ring + st * Cfg::kStage + my_keys, vt = ring + st * Cfg::kStage + my_values;
      const int base = (e.b0 + b) * kDecKeys + key0;                    // position of this warp's first key
      if (ok && base < hi && base + 16 > lo) {
        const bool edge = base + 16 > hi || base < lo;
        if (edge) {
#pragma unroll 1
          for (int i = lane; i < 16 * (D / 8); i += 32) {
            const int r = i / (D / 8), c = i % (D / 8), key = base + r;
            if (key >= hi || key < lo)
              asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vt + (c >> 3) * chunk + r * 128 +
                                                                        (((c & 7) ^ (r & 7)) << 4)),
                           "r"(0u)
                           : "memory");
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the ring's next copy into these rows
          __syncwarp();
        }
        // S: two 8-key tiles, each as two chains over D
        float sc[2][2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) sc[i][j][x] = 0.f;
        {
          // matrices of an ldmatrix: (keys 0-7, d 0-7), (keys 0-7, d 8-15), (keys 8-15, d 0-7), (keys 8-15, d 8-15)
          const int r = (lane & 7) + ((lane >> 4) << 3), cj = (lane >> 3) & 1;
          const uint32_t ra = kt + r * 128;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            uint32_t bm[4];
            ldmatrix_x4(bm, ra + (kk >> 2) * chunk + ((((kk & 3) * 2 + cj) ^ (r & 7)) << 4));
            mma_16<BF16>(sc[0][kk & 1], q[kk], bm[0], bm[1]);
            mma_16<BF16>(sc[1][kk & 1], q[kk], bm[2], bm[3]);
          }
        }
        float sv[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) sv[i][x] = (sc[i][0][x] + sc[i][1][x]) * a.scale_log2;
        if (base + 15 > e.pos0 || (a.window > 0 && base <= e.pos0 + e.n_tok - 1 - a.window)) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int key = base + i * 8 + t4 * 2 + (x & 1), p = pos[x >> 1];
              if (key > p || (a.window > 0 && key <= p - a.window)) sv[i][x] = -INFINITY;
            }
        }
        uint32_t pa[4];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          float mx = fmaxf(fmaxf(sv[0][2 * h2], sv[0][2 * h2 + 1]), fmaxf(sv[1][2 * h2], sv[1][2 * h2 + 1]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          const float mn = fmaxf(m[h2], mx), base_m = mn == -INFINITY ? 0.f : mn;
          const float f = ex2(m[h2] - base_m);
          if (__any_sync(0xffffffffu, mn != m[h2])) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) { o[i][2 * h2] *= f; o[i][2 * h2 + 1] *= f; }
            l[h2] *= f;
          }
          m[h2] = mn;
          const float p0 = ex2(sv[0][2 * h2] - base_m), p1 = ex2(sv[0][2 * h2 + 1] - base_m);
          const float p2 = ex2(sv[1][2 * h2] - base_m), p3 = ex2(sv[1][2 * h2 + 1] - base_m);
          l[h2] += (p0 + p1) + (p2 + p3);
          pa[h2] = pack_pair<BF16>(p0, p1);
          pa[2 + h2] = pack_pair<BF16>(p2, p3);
        }
        {
          // matrices: (keys 0-7, d 0-7), (keys 8-15, d 0-7), (keys 0-7, d 8-15), (keys 8-15, d 8-15), transposed
          const int r = lane & 15, cj = lane >> 4;
          const uint32_t ra = vt + r * 128;
#pragma unroll
          for (int nn = 0; nn < D / 16; ++nn) {
            uint32_t bm[4];
            ldmatrix_x4_trans(bm, ra + (nn >> 2) * chunk + ((((nn & 3) * 2 + cj) ^ (r & 7)) << 4));
            mma_16<BF16>(o[2 * nn], pa, bm[0], bm[1]);
            mma_16<BF16>(o[2 * nn + 1], pa, bm[2], bm[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(st));
    }

    // join the warps: (m, l) and O of every row
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
      l[h2] += __shfl_xor_sync(0xffffffffu, l[h2], 1);
      l[h2] += __shfl_xor_sync(0xffffffffu, l[h2], 2);
      if (t4 == 0) {
        s_ml[(warp * kDecRows + g + 8 * h2) * 2] = m[h2];
        s_ml[(warp * kDecRows + g + 8 * h2) * 2 + 1] = l[h2];
      }
      float *dst = s_join + (warp * kDecRows + g + 8 * h2) * Cfg::kRow + t4 * 2;
      if (g + 8 * h2 < rows)
#pragma unroll
        for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2 *>(dst + i * 8) = make_float2(o[i][2 * h2], o[i][2 * h2 + 1]);
    }
    named_sync(1, Cfg::kConsumers);
    const int c_first = w.u / hdr.dec_quota, c_last = (w.u + e.nb - 1) / hdr.dec_quota;
    const bool whole = c_first == c_last;
    constexpr int kCols = D / 4;                       // a thread owns 4 columns of every (kConsumers / kCols)-th row
    const int col = (tid % kCols) * 4, row0 = tid / kCols;
    auto write_row = [&](int r, float mm, float ll, float4 v) {
      const float inv = row_inv(ll);
      const int tok = r / a.group, hq = head * a.group + r - tok * a.group;
      const long long t = e.tok0 + tok;
      *reinterpret_cast<uint2 *>(a.out + t * a.out_stride + hq * D + col) =
          make_uint2(pack_pair<BF16>(v.x * inv, v.y * inv), pack_pair<BF16>(v.z * inv, v.w * inv));
      if (a.lse && col == 0) a.lse[t * a.n_q + hq] = row_lse(mm, ll);
    };
    float *part = a.part + (size_t)(blockIdx.x * 2 + (blockIdx.x == c_first ? 1 : 0)) * Cfg::kPart;
    for (int r = row0; r < rows; r += Cfg::kConsumers / kCols) {
      float mm = -INFINITY, ll = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < Cfg::kWarps; ++i) mm = fmaxf(mm, s_ml[(i * kDecRows + r) * 2]);
      const float bm = mm == -INFINITY ? 0.f : mm;
#pragma unroll
      for (int i = 0; i < Cfg::kWarps; ++i) {
        const float f = ex2(s_ml[(i * kDecRows + r) * 2] - bm);
        const float4 x = *reinterpret_cast<const float4 *>(s_join + (i * kDecRows + r) * Cfg::kRow + col);
        ll = fmaf(f, s_ml[(i * kDecRows + r) * 2 + 1], ll);
        v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
      }
      if (whole) {
        write_row(r, mm, ll, v);
      } else {
        if (col == 0) { part[r] = mm; part[kDecRows + r] = ll; }
        *reinterpret_cast<float4 *>(part + 2 * kDecRows + r * D + col) = v;
      }
    }
    if (!whole) {
      named_sync(1, Cfg::kConsumers);
      if (tid == 0) {
        __threadfence();                   // (for the whole group: the barrier orders its stores before)
        uint32_t *cnt = a.arrive + (size_t)w.k * a.n_kv + head;
        const uint32_t n = (uint32_t)(c_last - c_first + 1);
        const bool last = atomicAdd(cnt, 1u) == n - 1;
        if (last) *cnt = 0u;
        *s_last = last;
        __threadfence();
      }
      named_sync(1, Cfg::kConsumers);
      if (*s_last) {
        // all of a thread's rows and four parts at a time: what costs here is one load waiting for another
        constexpr int kStep = Cfg::kConsumers / kCols, kMine = kDecRows / kStep;
        float mm[kMine], ll[kMine];
        float4 v[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) { mm[i] = -INFINITY; ll[i] = 0.f; v[i] = make_float4(0.f, 0.f, 0.f, 0.f); }
        for (int c0 = c_first; c0 <= c_last; c0 += 4) {
          float mc[4][kMine], lc[4][kMine];
          float4 x[4][kMine];
#pragma unroll
          for (int z = 0; z < 4; ++z)
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
              const int c = c0 + z, r = row0 + i * kStep;
              mc[z][i] = -INFINITY; lc[z][i] = 0.f; x[z][i] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (c <= c_last && r < rows) {
                const float *pc = a.part + (size_t)(c * 2 + (c == c_first ? 1 : 0)) * Cfg::kPart;
                mc[z][i] = __ldcg(pc + r);
                lc[z][i] = __ldcg(pc + kDecRows + r);
                x[z][i] = __ldcg(reinterpret_cast<const float4 *>(pc + 2 * kDecRows + r * D + col));
              }
            }
#pragma unroll
          for (int z = 0; z < 4; ++z)
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
              const float mn = fmaxf(mm[i], mc[z][i]), bm = mn == -INFINITY ? 0.f : mn;
              const float f0 = ex2(mm[i] - bm), f1 = ex2(mc[z][i] - bm);
              ll[i] = ll[i] * f0 + lc[z][i] * f1;
              v[i].x = v[i].x * f0 + x[z][i].x * f1; v[i].y = v[i].y * f0 + x[z][i].y * f1;
              v[i].z = v[i].z * f0 + x[z][i].z * f1; v[i].w = v[i].w * f0 + x[z][i].w * f1;
              mm[i] = mn;
            }
        }
#pragma unroll
        for (int i = 0; i < kMine; ++i)
          if (row0 + i * kStep < rows) write_row(row0 + i * kStep, mm[i], ll[i], v[i]);
      }
    }
    named_sync(1, Cfg::kConsumers);      // the join buffer is free again
  }
  abort_drain(s_abort);
}

}  // namespace ftmoe
