// RMS norm of every query and key head, rotation by position and the write of keys and values into the paged cache, in
// one pass.  Bound: HBM (each of the T x (Hq + 2 Hkv) x D elements is read once and written once) for many tokens,
// latency for few.
//   y = x * rsqrt(mean(x^2) + eps) * w;  (a, b) -> (a cos - b sin, b cos + a sin)
// D/8 lanes share a head; a lane owns 8 elements such that both members of a rotated pair are its own (no exchange but
// the sum of squares): 4 pairs (i, i + rot/2) as two 8-byte accesses D/16 lanes wide, or 8 neighbouring elements when
// pairs are interleaved.  A lane group keeps the cosines and sines of its token in registers and walks over
// `heads_per_group` heads, so that the table costs 1/heads_per_group of a read per head.
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
__device__ __forceinline__ void unpack4(uint2 v, float (&f)[4]) {
  if (BF16) {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
    const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&v.x));
    const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&v.y));
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
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

template <int D, bool BF16>
__global__ void __launch_bounds__(256) attn_rope_kernel(const RopeArgs a) {
  constexpr int L = D / 8, kUnroll = 4;                // lanes per head; heads in flight per lane
  const int lane_in = threadIdx.x % L;
  const int heads = a.n_q + 2 * a.n_kv, parts = (heads + a.heads_per_group - 1) / a.heads_per_group;
  const long long group = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / L;
  const int t = (int)(group / parts), part = (int)(group - (long long)t * parts);
  if (t >= a.T) return;
  const uint32_t mask = ((L == 32 ? 0u : (1u << L)) - 1u) << ((threadIdx.x & 31) / L * L);

  // the lane's elements: off0 .. off0+3 and off1 .. off1+3
  int off0, off1;
  float c[4], s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
  int pos = a.position[t];
  if (pos >= a.max_pos && a.rot_half > 0) {
    if (lane_in == 0) atomicOr(a.status, kStatBadIndex);
    pos = -1;
  }
  if (a.interleaved) {
    off0 = lane_in * 8;
    off1 = off0 + 4;
    if (off0 < 2 * a.rot_half && pos >= 0) {           // pairs 4*lane .. 4*lane+3
      const float4 cc = *reinterpret_cast<const float4 *>(a.cos_sin + (long long)pos * 2 * a.rot_half + lane_in * 4);
      const float4 ss = *reinterpret_cast<const float4 *>(a.cos_sin + (long long)pos * 2 * a.rot_half + a.rot_half + lane_in * 4);
      c[0] = cc.x; c[1] = cc.y; c[2] = cc.z; c[3] = cc.w;
      s[0] = ss.x; s[1] = ss.y; s[2] = ss.z; s[3] = ss.w;
    }
  } else {
    const int i = lane_in * 4;
    if (i < a.rot_half) {
      off0 = i;
      off1 = i + a.rot_half;
      if (pos >= 0) {
        const float4 cc = *reinterpret_cast<const float4 *>(a.cos_sin + (long long)pos * 2 * a.rot_half + i);
        const float4 ss = *reinterpret_cast<const float4 *>(a.cos_sin + (long long)pos * 2 * a.rot_half + a.rot_half + i);
        c[0] = cc.x; c[1] = cc.y; c[2] = cc.z; c[3] = cc.w;
        s[0] = ss.x; s[1] = ss.y; s[2] = ss.z; s[3] = ss.w;
      }
    } else {                                           // what is not rotated: the halves of [rot, D)
      off0 = i + a.rot_half;
      off1 = i + D / 2;
    }
  }
  const int sl = a.slot[t];
  const bool store_kv = sl >= 0 && sl < (a.n_pages << a.page_shift) && pos >= 0;
  if (sl >= 0 && !(sl < (a.n_pages << a.page_shift)) && lane_in == 0) atomicOr(a.status, kStatBadIndex);
  const long long page = sl >> a.page_shift, row = sl & ((1 << a.page_shift) - 1);

  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { wq[i] = 1.f; wk[i] = 1.f; }
  auto load_w = [&](const uint16_t *w, float (&f)[8]) {
    float x0[4], x1[4];
    unpack4<BF16>(*reinterpret_cast<const uint2 *>(w + off0), x0);
    unpack4<BF16>(*reinterpret_cast<const uint2 *>(w + off1), x1);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = x0[i]; f[4 + i] = x1[i]; }
  };
  if (a.w_q) load_w(a.w_q, wq);
  if (a.w_k) load_w(a.w_k, wk);

  const int h_end = min(heads, (part + 1) * a.heads_per_group);
  for (int h0 = part * a.heads_per_group; h0 < h_end; h0 += kUnroll) {
    uint2 r0[kUnroll], r1[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u;
      if (h >= h_end) break;
      const uint16_t *src = h < a.n_q ? a.q + t * a.q_stride + h * D
                            : h < a.n_q + a.n_kv ? a.k + t * a.k_stride + (h - a.n_q) * D
                                                 : a.v + t * a.v_stride + (h - a.n_q - a.n_kv) * D;
      r0[u] = *reinterpret_cast<const uint2 *>(src + off0);
      r1[u] = *reinterpret_cast<const uint2 *>(src + off1);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u;
      if (h >= h_end) break;
      uint2 o0 = r0[u], o1 = r1[u];
      const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
      if (!is_v) {
        float x[8], x0[4], x1[4];
        unpack4<BF16>(o0, x0);
        unpack4<BF16>(o1, x1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = x0[i]; x[4 + i] = x1[i]; }
        if (is_q ? a.w_q != nullptr : a.w_k != nullptr) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
          for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
          const float inv = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * (is_q ? wq[i] : wk[i]);
        }
        float y[8];
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
            y[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[i] = x[i] * c[i] - x[4 + i] * s[i];
            y[4 + i] = x[4 + i] * c[i] + x[i] * s[i];
          }
        }
        o0 = make_uint2(pack_pair<BF16>(y[0], y[1]), pack_pair<BF16>(y[2], y[3]));
        o1 = make_uint2(pack_pair<BF16>(y[4], y[5]), pack_pair<BF16>(y[6], y[7]));
      }
      if (is_q) {
        if (pos < 0) { o0 = make_uint2(0u, 0u); o1 = o0; }
        uint16_t *dst = a.q_out + t * a.out_stride + h * D;
        *reinterpret_cast<uint2 *>(dst + off0) = o0;
        *reinterpret_cast<uint2 *>(dst + off1) = o1;
      } else if (store_kv) {
        const int hk = h - a.n_q;            // keys 0 .. n_kv-1, values n_kv .. 2 n_kv-1: the cache's order
        uint16_t *dst = a.cache + (((page * 2 * a.n_kv + hk) << a.page_shift) + row) * D;
        *reinterpret_cast<uint2 *>(dst + off0) = o0;
        *reinterpret_cast<uint2 *>(dst + off1) = o1;
      }
    }
  }
}

}  // namespace ftmoe
