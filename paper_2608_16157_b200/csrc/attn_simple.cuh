// Attention of the packed query rows over the paged cache, the plain form: one warp per (row, query head), one key at a
// time, running maximum and sum.  Right for every case; every key is read once per query head and row.
#pragma once
#include "attn_stream.cuh"

namespace ftmoe {

template <int D, bool BF16>
__global__ void __launch_bounds__(256) attn_simple_kernel(const AttnFwdArgs a) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const AttnPlanHdr hdr = *a.w.hdr;
  const int n = hdr.n_tile;
  const AttnEntry *list = a.w.tile;
  auto tof = [](uint16_t b) { return BF16 ? __uint_as_float((uint32_t)b << 16) : __half2float(__ushort_as_half(b)); };
  for (int ei = blockIdx.x; ei < n; ei += gridDim.x) {
    const AttnEntry e = list[ei];
    for (int w = threadIdx.x / 32; w < e.n_tok * a.n_q; w += blockDim.x / 32) {
      const int i = w / a.n_q, h = w % a.n_q, hk = h / (a.n_q / a.n_kv), pos = e.pos0 + i;
      const uint16_t *q = a.q + (long long)(e.tok0 + i) * a.q_stride + h * D;
      float qv[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
      for (int x = 0; x < E; ++x) { qv[x] = tof(q[x * 32 + lane]) * (a.scale_log2 * 0.693147180559945f); o[x] = 0.f; }
      const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
      for (int j = lo; j <= pos; ++j) {
        const int page = a.table[e.req * a.table_stride + (j >> a.page_shift)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) { if (lane == 0) atomicOr(a.status, kStatBadIndex); continue; }
        const long long row = (((long long)page * 2 * a.n_kv + hk) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        const uint16_t *k = a.cache + row * D, *v = k + ((long long)a.n_kv << a.page_shift) * D;
        float s = 0.f;
#pragma unroll
        for (int x = 0; x < E; ++x) s = fmaf(qv[x], tof(k[x * 32 + lane]), s);
        s = warp_sum(s);
        const float mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - mn), p = expf(s - mn);
        l = l * f + p;
#pragma unroll
        for (int x = 0; x < E; ++x) o[x] = o[x] * f + p * tof(v[x * 32 + lane]);
        m = mn;
      }
      uint16_t *dst = a.out + (long long)(e.tok0 + i) * a.out_stride + h * D;
#pragma unroll
      for (int x = 0; x < E; ++x) dst[x * 32 + lane] = (uint16_t)pack_pair<BF16>(l > 0.f ? o[x] / l : 0.f, 0.f);
      if (a.lse && lane == 0) a.lse[(long long)(e.tok0 + i) * a.n_q + h] = l > 0.f ? m + logf(l) : -INFINITY;
    }
  }
}

}  // namespace ftmoe
