// A block's output joins the residual stream and the next block's input is normed, in one pass:
//   u = y, or y * rsqrt(mean(y^2) + eps) * (o + w_post);  r' = a r + b gate u;  h = r' * rsqrt(mean(r'^2) + eps) * (o + w_pre)
// Bound: HBM (y, r and a gate per element read once, r' and h written once) for many tokens, launch latency for few.
// `lanes` threads (32 .. 1024, a power of two) share a row; a thread holds E of its elements in float from the loads to the stores, so that
// a row is read once, whatever is written over it.  All loads of y, r and the gate go out before the first sum.  E = 16, or 8 for few rows, where
// latency counts.  Where d is a multiple of 8 a thread has 8 neighbouring elements at a time, in one access for each array whose rows all
// start on 16 bytes; else single elements, neighbouring threads on neighbouring elements (twice the time: the load and store units are
// then the bound).  Measured: 60 us for 16384 tokens of 2048 with a float stream (6.7 TB/s), 62 us in bf16 with norms on both sides and a
// gate per channel (4.3 TB/s), 2.1 us for 8 tokens.
#pragma once
#include "async.cuh"
#include "common.cuh"

namespace ftmoe {

constexpr int kNormMaxDim = 16384;

enum : uint32_t { kWideY = 1, kWideRes = 2, kWideGate = 4, kWidePost = 8, kWidePre = 16, kWideResOut = 32, kWideOut = 64, kWideAll = 127 };

struct NormArgs {
  int32_t T, d, lanes, post, gate_step;
  uint32_t wide;                     // kWide*: arrays that allow 16-byte accesses
  const uint16_t *y, *gate, *w_post, *w_pre;
  const void *res;
  void *res_out;
  uint16_t *out;
  long long y_stride, res_stride, gate_stride, res_out_stride, out_stride;
  float w_offset, eps, res_scale, y_scale;
  uint32_t mean_low;                 // bits of the float below which a mean of squares counts as lost
};

template <bool BF16>
__device__ __forceinline__ float to_float(uint16_t v) {
  return BF16 ? bf16_bits_to_float(v) : __half2float(__ushort_as_half(v));
}
template <bool BF16>
__device__ __forceinline__ uint16_t from_float(float v) {
  return BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
template <bool BF16>
__device__ __forceinline__ void to_float2(uint32_t v, float &a, float &b) {
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
__device__ __forceinline__ uint32_t from_float2(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// VEC elements of a 16-bit or a float array.
template <bool BF16, int VEC>
__device__ __forceinline__ void load_16(const uint16_t *p, float *x, bool wide) {
  if constexpr (VEC == 8) {
    if (!wide) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_float<BF16>(p[i]);
      return;
    }
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    to_float2<BF16>(v.x, x[0], x[1]); to_float2<BF16>(v.y, x[2], x[3]);
    to_float2<BF16>(v.z, x[4], x[5]); to_float2<BF16>(v.w, x[6], x[7]);
  } else {
    x[0] = to_float<BF16>(*p);
  }
}
template <int VEC>
__device__ __forceinline__ void load_32(const float *p, float *x, bool wide) {
  if constexpr (VEC == 8) {
    if (!wide) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[i];
      return;
    }
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    x[0] = *p;
  }
}
template <bool BF16, int VEC>
__device__ __forceinline__ void store_16(uint16_t *p, const float *x, bool wide) {
  if (VEC == 8 && wide) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(from_float2<BF16>(x[0], x[VEC > 1]), from_float2<BF16>(x[VEC / 4], x[VEC * 3 / 8]),
                                               from_float2<BF16>(x[VEC / 2], x[VEC * 5 / 8]), from_float2<BF16>(x[VEC * 3 / 4], x[VEC * 7 / 8]));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = from_float<BF16>(x[i]);
  }
}
template <int VEC>
__device__ __forceinline__ void store_32(float *p, const float *x, bool wide) {
  if constexpr (VEC == 8) {
    if (wide) {
      *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) p[i] = x[i];
}

// Sum over the threads of a row; `s` holds a float per warp.  Where a row has more than a warp, it has a block of its own.
__device__ __forceinline__ float row_sum(float v, int lanes, float *s) {
  v = warp_sum(v);
  if (lanes == 32) return v;
  const int n = lanes >> 5;
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
  for (int i = 0; i < n; ++i) t += s[i];
  return t;
}

__device__ __forceinline__ float row_max(float v, int lanes, float *s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (lanes == 32) return v;
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
  for (int i = 0; i < lanes >> 5; ++i) t = fmaxf(t, s[i]);
  return t;
}
// 1 / sqrt(mean(x^2) + eps) of a row from the sum of its squares.  Where the squares have left the floats' range (a sum that is infinite, or below 2^-100
// with an eps that does not cover what is lost), x becomes x f and what is returned belongs to that, f a power of two: then the larger of the
// largest element and the root of eps is near one.
template <int E>
__device__ __forceinline__ float row_inv_rms(const NormArgs &a, float (&x)[E], float sum, float (*s)[32]) {
  float mean = sum / (float)a.d, eps = a.eps;
  // (the same for all of a row's threads; one comparison of the bits, beyond which infinity and NaN stand too)
  if (__builtin_expect(__float_as_uint(mean) - a.mean_low >= 0x7f800000u - a.mean_low, 0)) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) top = fmaxf(top, fabsf(x[i]));
    top = row_max(top, a.lanes, s[0]);
    if (top > 0.f && top < INFINITY) {
      int e = -ilogbf(top);
      if (eps > 0.f) e = min(e, -ilogbf(eps) / 2);
      const float f = ldexpf(1.f, max(min(e, 126), -127));
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] *= f;
        sum = fmaf(x[i], x[i], sum);
      }
      mean = row_sum(sum, a.lanes, s[1]) / (float)a.d;
      eps = eps * f * f;
    }
  }
  return rsqrtf(mean + eps);
}

// VEC elements at a time; ALL: every array allows 16-byte accesses.
template <bool BF16, bool RES32, bool POST, bool GATE, int VEC, bool ALL, int E>
__global__ void __launch_bounds__(1024) add_norm_kernel(const NormArgs a) {
  constexpr int N = E / VEC;
  __shared__ float s_sum[6][32];
  grid_let_next();
  const int lane = threadIdx.x & (a.lanes - 1);
  const long long t = (long long)blockIdx.x * (blockDim.x / a.lanes) + threadIdx.x / a.lanes;
  const uint16_t *y = a.y + t * a.y_stride, *gate = a.gate + t * a.gate_stride;
  grid_wait();
  if (t >= a.T) return;                     // (only where a row is a warp's)
  float r[E], u[E];
  uint32_t g[GATE ? (E + 1) / 2 : 1];
#pragma unroll
  for (int i = 0; i < E; ++i) r[i] = u[i] = 0.f;
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = (j * a.lanes + lane) * VEC;
      if (i < a.d) f(i, j * VEC);
    }
  };
  if (a.y) each([&](int i, int j) { load_16<BF16, VEC>(y + i, u + j, ALL || (a.wide & kWideY)); });
  if (a.res) {
    const char *res = static_cast<const char *>(a.res) + t * a.res_stride * (RES32 ? 4 : 2);
    each([&](int i, int j) {
      if (RES32) load_32<VEC>(reinterpret_cast<const float *>(res) + i, r + j, ALL || (a.wide & kWideRes));
      else load_16<BF16, VEC>(reinterpret_cast<const uint16_t *>(res) + i, r + j, ALL || (a.wide & kWideRes));
    });
  }
  if (GATE) each([&](int i, int j) {
    if constexpr (VEC == 8) {
      uint4 v;
      if (ALL || (a.wide & kWideGate)) v = *reinterpret_cast<const uint4 *>(gate + i);
      else
        v = make_uint4(gate[i] | (uint32_t)gate[i + 1] << 16, gate[i + 2] | (uint32_t)gate[i + 3] << 16, gate[i + 4] | (uint32_t)gate[i + 5] << 16,
                       gate[i + 6] | (uint32_t)gate[i + 7] << 16);
      g[j / 2] = v.x; g[j / 2 + 1] = v.y; g[j / 2 + 2] = v.z; g[j / 2 + 3] = v.w;
    } else {
      if (j % 2 == 0) g[j / 2] = gate[i]; else g[j / 2] |= (uint32_t)gate[i] << 16;
    }
  });
  // what is left out counts nothing; a gate of one value a token is part of the scale
  const float r_scale = a.res ? a.res_scale : 0.f;
  const float y_scale = !a.y ? 0.f : !GATE && a.gate ? a.y_scale * to_float<BF16>(*gate) : a.y_scale;
  float inv = 1.f;
  if (POST) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) sum = fmaf(u[i], u[i], sum);
    inv = row_inv_rms<E>(a, u, row_sum(sum, a.lanes, s_sum[0]), s_sum + 2);
  }
  float sum = 0.f;
  char *res_out = static_cast<char *>(a.res_out) + t * a.res_out_stride * (RES32 ? 4 : 2);
  each([&](int i, int j) {
    float f[VEC];                           // the factors of u
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] = 1.f;
    if (POST) {
      if (a.w_post) {
        load_16<BF16, VEC>(a.w_post + i, f, ALL || (a.wide & kWidePost));
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] = inv * (a.w_offset + f[k]);
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] = inv;
      }
    }
#pragma unroll
    for (int k = 0; k < VEC; k += 2) {
      if (GATE) {
        float g0, g1;
        to_float2<BF16>(VEC == 1 && j % 2 ? g[j / 2] >> 16 : g[(j + k) / 2], g0, g1);
        f[k] *= g0;
        if (VEC > 1) f[k + 1 < VEC ? k + 1 : k] *= g1;
      }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float v = POST || GATE ? u[j + k] * f[k] : u[j + k];
      r[j + k] = fmaf(y_scale, v, r_scale * r[j + k]);
      sum = fmaf(r[j + k], r[j + k], sum);
    }
    if (a.res_out) {
      if (RES32) store_32<VEC>(reinterpret_cast<float *>(res_out) + i, r + j, ALL || (a.wide & kWideResOut));
      else store_16<BF16, VEC>(reinterpret_cast<uint16_t *>(res_out) + i, r + j, ALL || (a.wide & kWideResOut));
    }
  });
  if (!a.out) return;
  inv = row_inv_rms<E>(a, r, row_sum(sum, a.lanes, s_sum[1]), s_sum + 4);
  uint16_t *out = a.out + t * a.out_stride;
  each([&](int i, int j) {
    float h[VEC];
    if (a.w_pre) {
      load_16<BF16, VEC>(a.w_pre + i, h, ALL || (a.wide & kWidePre));
#pragma unroll
      for (int k = 0; k < VEC; ++k) h[k] = r[j + k] * (inv * (a.w_offset + h[k]));
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) h[k] = r[j + k] * inv;
    }
    store_16<BF16, VEC>(out + i, h, ALL || (a.wide & kWideOut));
  });
}

}  // namespace ftmoe
