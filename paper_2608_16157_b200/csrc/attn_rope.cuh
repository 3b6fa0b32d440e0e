// RMS norm of every query and key head, rotation by position and the write of keys and values into the paged cache, in
// one pass.  Bound: HBM (each of the T x (Hq + 2 Hkv) x D elements is read once and written once) for many tokens,
// latency for few.
//   y = x * rsqrt(mean(x^2) + eps) * w;  (a, b) -> (a cos - b sin, b cos + a sin)
// D/(2V) lanes share a head; a lane owns 2V elements such that both members of a rotated pair are its own (no exchange but
// the sum of squares): V pairs (i, i + rot/2), or 2V neighbouring elements when pairs are interleaved.  V = 8 (16-byte
// accesses) where alignment and rot allow it, else 4.  A lane group keeps the cosines and sines of its token in registers and
// walks over `heads_per_group` heads, kUnroll of them in flight.
#pragma once
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
        if (a.interleaved) {
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

}  // namespace ftmoe
