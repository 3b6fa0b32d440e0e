// RMS norm of every query and key head, rotation by position and the write of keys and values into the paged cache, in
// one pass.  Bound: HBM (each of the T x (Hq + 2 Hkv) x D elements is read once and written once) for many tokens,
// latency for few.
//   y = x * rsqrt(mean(x^2) + eps) * w;  (a, b) -> (a cos - b sin, b cos + a sin)
// D/(2V) lanes share a head; a lane owns 2V elements such that both members of a rotated pair are its own (no exchange but
// the sum of squares): V pairs (i, i + rot/2), or 2V neighbouring elements when pairs are interleaved.  V = 8 (16-byte
// accesses) where alignment and rot allow it, else 4.
// Two forms.  Few tokens: a lane group keeps the cosines and sines of its token in registers and walks over
// `heads_per_group` heads.  Many tokens: resident blocks, to whose shared memory a producer warp brings whole tokens and their
// table rows with bulk copies, several tokens ahead (the position is only known after a load, the table row after another:
// held in registers meanwhile, the data of too few tokens is on its way: 84 us for 16384 tokens of 32 + 2 x 4 heads of 128).
// Measured with these heads: 65.4 us for 16384 tokens (5.27 TB/s; a copy takes 52.5), 7.2 us for 1021, 2.4 us for 8.
#pragma once
#include "async.cuh"
#include "common.cuh"

namespace ftmoe {

struct RopeArgs {
  int32_t T, n_q, n_kv, page_shift, n_pages, rot_half, interleaved, max_pos, heads_per_group;
  const uint16_t *q, *k, *v, *w_q, *w_k;
  long long q_stride, k_stride, v_stride, out_stride;
  float eps;
  const float *cos_sin;
  const int32_t *position, *slot;
  uint16_t *q_out, *cache;
  uint32_t *status;
};

// Two floats in a register pair: one instruction for both.
__device__ __forceinline__ uint64_t f2(float lo, float hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ void f2_split(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <bool BF16>
__device__ __forceinline__ void unpack2(uint32_t v, float &a, float &b) {
  if (BF16) {
    a = __uint_as_float(v << 16);
    b = __uint_as_float(v & 0xffff0000u);
  } else {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v));
    a = f.x;
    b = f.y;
  }
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// V 16-bit elements as V/2 words; not through the read-only path, since the result may go where the input is.
template <int V>
__device__ __forceinline__ void load_elems(const uint16_t *p, uint32_t (&r)[V / 2]) {
  if constexpr (V == 8)
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
  else
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
}
template <int V>
__device__ __forceinline__ void store_elems(uint16_t *p, const uint32_t (&r)[V / 2]) {
  if constexpr (V == 8)
    *reinterpret_cast<uint4 *>(p) = make_uint4(r[0], r[1], r[2], r[3]);
  else
    *reinterpret_cast<uint2 *>(p) = make_uint2(r[0], r[1]);
}

template <int D, bool BF16, int V>
__global__ void __launch_bounds__(256) attn_rope_kernel(const RopeArgs a) {
  constexpr int L = D / (2 * V), kUnroll = V == 8 ? 4 : 8;   // lanes per head; heads in flight per lane
  grid_let_next();
  grid_wait();
  const int lane_in = threadIdx.x % L;
  const int heads = a.n_q + 2 * a.n_kv, parts = (heads + a.heads_per_group - 1) / a.heads_per_group;
  const long long group = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / L;
  const int t = (int)(group / parts), part = (int)(group - (long long)t * parts);
  if (t >= a.T) return;
  const uint32_t mask = ((1u << L) - 1u) << ((threadIdx.x & 31) / L * L);

  // the lane's elements: off0 .. off0+V-1 and off1 .. off1+V-1; its pairs from `pair` on (none: not rotated)
  int off0, off1, pair;
  if (a.interleaved) {
    off0 = lane_in * 2 * V;
    off1 = off0 + V;
    pair = off0 < 2 * a.rot_half ? lane_in * V : -1;
  } else {
    const int i = lane_in * V;
    pair = i < a.rot_half ? i : -1;
    off0 = pair >= 0 ? i : i + a.rot_half;            // what is not rotated: the halves of [rot, D)
    off1 = pair >= 0 ? i + a.rot_half : i + D / 2;
  }
  const int h_begin = part * a.heads_per_group, h_end = min(heads, h_begin + a.heads_per_group);
  uint32_t r0[kUnroll][V / 2], r1[kUnroll][V / 2];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u;
      if (h >= h_end) break;
      const uint16_t *src = h < a.n_q ? a.q + t * a.q_stride + h * D
                            : h < a.n_q + a.n_kv ? a.k + t * a.k_stride + (h - a.n_q) * D
                                                 : a.v + t * a.v_stride + (h - a.n_q - a.n_kv) * D;
      load_elems<V>(src + off0, r0[u]);
      load_elems<V>(src + off1, r1[u]);
    }
  };
  load(h_begin);

  int pos = a.position[t];
  const int sl = a.slot[t];
  if (pos >= a.max_pos && a.rot_half > 0) {
    if (lane_in == 0) atomicOr(a.status, kStatBadIndex);
    pos = -1;
  }
  const bool store_kv = sl >= 0 && sl < (a.n_pages << a.page_shift) && pos >= 0;
  if (sl >= (a.n_pages << a.page_shift) && lane_in == 0) atomicOr(a.status, kStatBadIndex);
  const long long page = sl >> a.page_shift, row = sl & ((1 << a.page_shift) - 1);
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) { c[i] = 1.f; s[i] = 0.f; }
  if (pair >= 0 && pos >= 0) {
    const float4 *cp = reinterpret_cast<const float4 *>(a.cos_sin + (long long)pos * 2 * a.rot_half + pair);
    const float4 *sp = reinterpret_cast<const float4 *>(a.cos_sin + (long long)pos * 2 * a.rot_half + a.rot_half + pair);
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      const float4 cc = cp[i], ss = sp[i];
      c[4 * i] = cc.x; c[4 * i + 1] = cc.y; c[4 * i + 2] = cc.z; c[4 * i + 3] = cc.w;
      s[4 * i] = ss.x; s[4 * i + 1] = ss.y; s[4 * i + 2] = ss.z; s[4 * i + 3] = ss.w;
    }
  }
  uint32_t wq0[V / 2], wq1[V / 2], wk0[V / 2], wk1[V / 2];     // (packed: read where they are used)
  if (a.w_q) { load_elems<V>(a.w_q + off0, wq0); load_elems<V>(a.w_q + off1, wq1); }
  if (a.w_k) { load_elems<V>(a.w_k + off0, wk0); load_elems<V>(a.w_k + off1, wk1); }

  for (int h0 = h_begin; h0 < h_end; h0 += kUnroll) {
    if (h0 > h_begin) load(h0);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u;
      if (h >= h_end) break;
      const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
      if (!is_v) {
        float x[2 * V], y[2 * V];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          unpack2<BF16>(r0[u][i], x[2 * i], x[2 * i + 1]);
          unpack2<BF16>(r1[u][i], x[V + 2 * i], x[V + 2 * i + 1]);
        }
        if (is_q ? a.w_q != nullptr : a.w_k != nullptr) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
          for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
          const float inv = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            float w0, w1, w2, w3;
            unpack2<BF16>(is_q ? wq0[i] : wk0[i], w0, w1);
            unpack2<BF16>(is_q ? wq1[i] : wk1[i], w2, w3);
            x[2 * i] *= inv * w0; x[2 * i + 1] *= inv * w1;
            x[V + 2 * i] *= inv * w2; x[V + 2 * i + 1] *= inv * w3;
          }
        }
        if (pair < 0) {                       // not rotated: an infinity must not reach its neighbour as infinity * 0
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) y[i] = x[i];
        } else if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            y[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
            y[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            y[i] = x[i] * c[i] - x[V + i] * s[i];
            y[V + i] = x[V + i] * c[i] + x[i] * s[i];
          }
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          r0[u][i] = pack_pair<BF16>(y[2 * i], y[2 * i + 1]);
          r1[u][i] = pack_pair<BF16>(y[V + 2 * i], y[V + 2 * i + 1]);
        }
      }
      uint16_t *dst = nullptr;
      if (is_q) {
        dst = a.q_out + t * a.out_stride + h * D;
        if (pos < 0) {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) r0[u][i] = r1[u][i] = 0u;
        }
      } else if (store_kv) {
        // keys 0 .. n_kv-1, values n_kv .. 2 n_kv-1: the cache's order
        dst = a.cache + (((page * 2 * a.n_kv + h - a.n_q) << a.page_shift) + row) * D;
      }
      if (dst) {
        store_elems<V>(dst + off0, r0[u]);
        store_elems<V>(dst + off1, r1[u]);
      }
    }
  }
}

constexpr uint32_t kWithholdRope = 4u;   // ft_attn_debug_inject
// The form for many tokens.  Dynamic shared memory: stages of [q row | k row | v row | table row], then the barriers.
constexpr int kRopeStages = 5, kRopeBlocks = 2;    // tokens ahead in a block, blocks an SM
__host__ __device__ inline int rope_stage_bytes(int heads, int D, int rot) { return (heads * D * 2 + rot * 4 + 127) / 128 * 128; }

template <int D, bool BF16>
__global__ void __launch_bounds__(544) attn_rope_stream_kernel(const RopeArgs a) {
  constexpr int V = 8, L = D / (2 * V);
  extern __shared__ __align__(128) unsigned char smem[];
  const int heads = a.n_q + 2 * a.n_kv, stage = rope_stage_bytes(heads, D, 2 * a.rot_half);
  uint64_t *s_bar = reinterpret_cast<uint64_t *>(smem + kRopeStages * stage);
  volatile int *s_abort = reinterpret_cast<volatile int *>(s_bar + 2 * kRopeStages);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, consumers = blockDim.x - 32;
  const uint32_t base = smem_u32(smem), bars = smem_u32(s_bar);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kRopeStages + s); };
  grid_let_next();
  if (tid == 0) {
    for (int s = 0; s < kRopeStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), consumers / 32); }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  grid_wait();
  const int q_bytes = a.n_q * D * 2, kv_bytes = a.n_kv * D * 2, step = gridDim.x;
  int s = 0;
  uint32_t ph = 0;
  auto advance = [&]() { if (++s == kRopeStages) { s = 0; ph ^= 1u; } };

  if (warp == consumers / 32) {
    // ------------------------------ producer: positions 32 tokens at a time ------------------------------
    bool withhold = blockIdx.x == 0 && (g_debug_withhold & kWithholdRope);
    for (int t0 = blockIdx.x; t0 < a.T && !*s_abort; t0 += 32 * step) {
      const int pos = t0 + lane * step < a.T ? a.position[t0 + lane * step] : -1;
      for (int i = 0; i < 32 && t0 + i * step < a.T; ++i) {
        const long long t = t0 + i * step;
        const int p = __shfl_sync(0xffffffffu, pos, i);
        const bool table = a.rot_half > 0 && p >= 0 && p < a.max_pos;
        mbar_wait(empty_bar(s), ph ^ 1u, s_abort, a.status);
        if (*s_abort) break;
        if (lane == 0) {
          const uint32_t dst = base + s * stage;
          mbar_expect_tx(full_bar(s), q_bytes + 2 * kv_bytes + (table ? 8 * a.rot_half : 0));
          if (!withhold) bulk_g2s(dst, a.q + t * a.q_stride, q_bytes, full_bar(s));     // (withheld: test hook)
          bulk_g2s(dst + q_bytes, a.k + t * a.k_stride, kv_bytes, full_bar(s));
          bulk_g2s(dst + q_bytes + kv_bytes, a.v + t * a.v_stride, kv_bytes, full_bar(s));
          if (table) bulk_g2s(dst + q_bytes + 2 * kv_bytes, a.cos_sin + (long long)p * 2 * a.rot_half, 8 * a.rot_half, full_bar(s));
        }
        __syncwarp();
        withhold = false;
        advance();
      }
    }
    abort_drain(s_abort);
    return;
  }

  // ------------------------------ consumers: one head's lane group each, some more than one head ------------------------------
  const int lane_in = tid % L, groups = consumers / L;
  const uint32_t mask = ((1u << L) - 1u) << (lane / L * L);
  int off0, off1, pair;
  if (a.interleaved) {
    off0 = lane_in * 2 * V;
    off1 = off0 + V;
    pair = off0 < 2 * a.rot_half ? lane_in * V : -1;
  } else {
    const int i = lane_in * V;
    pair = i < a.rot_half ? i : -1;
    off0 = pair >= 0 ? i : i + a.rot_half;
    off1 = pair >= 0 ? i + a.rot_half : i + D / 2;
  }
  uint32_t w0[V / 2], w1[V / 2];               // norm weights of the head at hand
  const uint16_t *w_now = nullptr;
  int pos_next = blockIdx.x < a.T ? a.position[blockIdx.x] : 0, slot_next = blockIdx.x < a.T ? a.slot[blockIdx.x] : 0;
  for (long long t = blockIdx.x; t < a.T; t += step) {
    int pos = pos_next;
    const int sl = slot_next;
    if (t + step < a.T) { pos_next = a.position[t + step]; slot_next = a.slot[t + step]; }
    if (pos >= a.max_pos && a.rot_half > 0) {
      if (tid == 0) atomicOr(a.status, kStatBadIndex);
      pos = -1;
    }
    const bool store_kv = sl >= 0 && sl < (a.n_pages << a.page_shift) && pos >= 0;
    if (sl >= (a.n_pages << a.page_shift) && tid == 0) atomicOr(a.status, kStatBadIndex);
    const long long page = sl >> a.page_shift, row = sl & ((1 << a.page_shift) - 1);
    const bool ok = mbar_wait(full_bar(s), ph, s_abort, a.status);
    const unsigned char *st = smem + s * stage;
    if (ok)
      for (int h = tid / L; h < heads; h += groups) {
        const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
        uint16_t *dst = nullptr;
        if (is_q) dst = a.q_out + t * a.out_stride + h * D;
        else if (store_kv) dst = a.cache + (((page * 2 * a.n_kv + h - a.n_q) << a.page_shift) + row) * D;
        if (!dst) continue;                    // (the same for the lanes of the group)
        const uint16_t *src = reinterpret_cast<const uint16_t *>(st) + h * D;
        uint4 v0 = *reinterpret_cast<const uint4 *>(src + off0), v1 = *reinterpret_cast<const uint4 *>(src + off1);
        if (!is_v) {
          uint32_t r0[4] = {v0.x, v0.y, v0.z, v0.w}, r1[4] = {v1.x, v1.y, v1.z, v1.w};
          uint64_t x0[4], x1[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float p, q;
            unpack2<BF16>(r0[i], p, q);
            x0[i] = f2(p, q);
            unpack2<BF16>(r1[i], p, q);
            x1[i] = f2(p, q);
          }
          const uint16_t *w = is_q ? a.w_q : a.w_k;
          if (w) {
            if (w != w_now) { load_elems<V>(w + off0, w0); load_elems<V>(w + off1, w1); w_now = w; }
            uint64_t acc0 = 0, acc1 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) { acc0 = fma2(x0[i], x0[i], acc0); acc1 = fma2(x1[i], x1[i], acc1); }
            float p, q;
            f2_split(add2(acc0, acc1), p, q);
            float sum = p + q;
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
            const float inv = rsqrtf(sum * (1.f / D) + a.eps);
            const uint64_t inv2 = f2(inv, inv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              unpack2<BF16>(w0[i], p, q);
              x0[i] = mul2(x0[i], mul2(inv2, f2(p, q)));
              unpack2<BF16>(w1[i], p, q);
              x1[i] = mul2(x1[i], mul2(inv2, f2(p, q)));
            }
          }
          if (pair >= 0 && pos >= 0) {
            const float *cp = reinterpret_cast<const float *>(st + q_bytes + 2 * kv_bytes) + pair, *sp = cp + a.rot_half;
            if (a.interleaved) {
              // a register pair is (a, b) of one pair: (a, b) cos + (b, a) (-sin, sin)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float p, q;
                f2_split(x0[i], p, q);
                x0[i] = f2(p * cp[i] - q * sp[i], q * cp[i] + p * sp[i]);
                f2_split(x1[i], p, q);
                x1[i] = f2(p * cp[4 + i] - q * sp[4 + i], q * cp[4 + i] + p * sp[4 + i]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const ulonglong2 c = *reinterpret_cast<const ulonglong2 *>(cp + 4 * i), z = *reinterpret_cast<const ulonglong2 *>(sp + 4 * i);
                const uint64_t sign = 0x8000000080000000ull;
                const uint64_t a0 = fma2(x0[2 * i], c.x, mul2(x1[2 * i], z.x) ^ sign), b0 = fma2(x0[2 * i], z.x, mul2(x1[2 * i], c.x));
                const uint64_t a1 = fma2(x0[2 * i + 1], c.y, mul2(x1[2 * i + 1], z.y) ^ sign), b1 = fma2(x0[2 * i + 1], z.y, mul2(x1[2 * i + 1], c.y));
                x0[2 * i] = a0; x1[2 * i] = b0; x0[2 * i + 1] = a1; x1[2 * i + 1] = b1;
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float p, q;
            f2_split(x0[i], p, q);
            r0[i] = pack_pair<BF16>(p, q);
            f2_split(x1[i], p, q);
            r1[i] = pack_pair<BF16>(p, q);
          }
          v0 = pos < 0 ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(r0[0], r0[1], r0[2], r0[3]);
          v1 = pos < 0 ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(r1[0], r1[1], r1[2], r1[3]);
        }
        *reinterpret_cast<uint4 *>(dst + off0) = v0;
        *reinterpret_cast<uint4 *>(dst + off1) = v1;
      }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty_bar(s));
    advance();
  }
  abort_drain(s_abort);
}

}  // namespace ftmoe
