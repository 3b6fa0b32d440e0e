// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits, in one pass over them.
// Bound: HBM (T x vocab logits read once); for few rows launch and the chain load -> exponentials -> join.
//   l = c x;  S = sum 2^((x - m) c log2 e),  U = sum of the same times its exponent;  lse and entropy follow from S, U and m
// A cluster of blocks shares a row while there are fewer rows than SMs.  Every thread walks over its 16-byte pieces of the row with a
// running maximum m, S and U of its own (rescaled only where a piece brings a new maximum), which are joined at the end in a fixed
// order.  The maxima also find the alternatives: the k-th largest of the threads' maxima is a lower bound of the k-th largest logit, so
// only threads whose maximum reaches it (k of them, and ties) read their pieces again, from L2, and keep what reaches it.  The main
// loop thus does nothing for them.  Candidates are ranked by counting, as keys (logit, then lowest id).
#pragma once
#include "async.cuh"
#include "cluster.cuh"
#include "common.cuh"

namespace ftmoe {

constexpr int kLogpThreads = 512, kLogpWarps = kLogpThreads / 32, kLogpTop = 32, kLogpCluster = 8;

struct LogpArgs {
  const void *logits;
  long long stride;
  int32_t T, vocab, n_tokens, top_k;
  float scale;                       // c
  const int32_t *tokens;
  long long tokens_stride;
  float *logprob, *entropy, *top_logprobs;
  int32_t *top_ids;
  uint32_t *status;
};

enum { kLogpBf16 = 0, kLogpFp16 = 1, kLogpFp32 = 2 };
template <int TY>
struct LogpType {
  static constexpr int kBytes = TY == kLogpFp32 ? 4 : 2, kVec = 16 / kBytes;     // elements of a 16-byte piece
  static __device__ __forceinline__ float at(const void *p, long long i) {
    if (TY == kLogpFp32) return static_cast<const float *>(p)[i];
    const uint16_t v = static_cast<const uint16_t *>(p)[i];
    return TY == kLogpBf16 ? bf16_bits_to_float(v) : __half2float(__ushort_as_half(v));
  }
  static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[kVec]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TY == kLogpFp32) {
        x[i] = __uint_as_float(w[i]);
      } else if constexpr (TY == kLogpBf16) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
    }
  }
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Order-preserving map to unsigned (-0 folded into +0); -infinity and NaN are no alternatives: 0.
__device__ __forceinline__ uint32_t logp_order(float x) {
  if (!(x > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float logp_value(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }

// Running maximum, sum and weighted sum of exponents; m starts at the lowest finite value, so that x - m is never infinity - infinity
// for a -infinity.
struct LogpAcc {
  float m = -3.402823466e38f, s = 0.f, u = 0.f;
  __device__ __forceinline__ void raise(float to, float c2) {     // to > m
    const float d = (m - to) * c2;
    if (d < -200.f) {
      if (!(s != s)) s = 0.f;
      u = 0.f;
    } else {
      const float f = exp2_approx(d);
      u = f * fmaf(d, s, u);
      s *= f;
    }
    m = to;
  }
  __device__ __forceinline__ void add(float x, float c2) {
    const float t = (x - m) * c2, e = exp2_approx(t);
    s += e;
    u = fmaf(e, fmaxf(t, -1000.f), u);       // (0 times -infinity)
  }
  __device__ __forceinline__ void join(LogpAcc o, float c2) {
    if (o.m > m) raise(o.m, c2);
    else if (m > o.m) o.raise(m, c2);
    s += o.s;
    u += o.u;
  }
};

struct LogpSmem {
  float m[kLogpWarps], s[kLogpWarps], u[kLogpWarps];
  uint32_t best[kLogpWarps][32];                       // the threads' maxima, sorted descending, per warp
  uint64_t key[kLogpCluster * kLogpTop];               // block 0 of the cluster: candidates of all blocks
  uint64_t own[kLogpWarps * kLogpTop];
  float part[kLogpCluster][3];
  uint32_t n_own, n_all, tau;
};

// Sorts a value per lane, descending.
__device__ __forceinline__ uint32_t warp_sort(uint32_t v, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2) {
      const uint32_t o = __shfl_xor_sync(0xffffffffu, v, j);
      const bool keep_max = ((lane & k) == 0) == ((lane & j) == 0);
      v = keep_max ? max(v, o) : min(v, o);
    }
  return v;
}
// Of two descending lists the 32 largest, descending.
__device__ __forceinline__ uint32_t warp_merge(uint32_t a, uint32_t b_reversed, int lane) {
  uint32_t v = max(a, b_reversed);
#pragma unroll
  for (int j = 16; j > 0; j /= 2) {
    const uint32_t o = __shfl_xor_sync(0xffffffffu, v, j);
    v = (lane & j) == 0 ? max(v, o) : min(v, o);
  }
  return v;
}

__device__ __forceinline__ void st_cluster_u64(uint32_t addr, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory"); }
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ uint32_t add_cluster_u32(uint32_t addr, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(addr), "r"(v) : "memory");
  return old;
}

template <int TY>
__global__ void __launch_bounds__(kLogpThreads, 2) logprobs_kernel(const LogpArgs a, const int cluster) {
  using Y = LogpType<TY>;
  constexpr int E = Y::kVec;
  __shared__ LogpSmem sm;
  grid_let_next();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x % cluster;
  const long long row = blockIdx.x / cluster;
  if (tid == 0) sm.n_own = sm.n_all = 0;
  if (cluster > 1) cluster_arrive();
  grid_wait();
  const uint8_t *base = static_cast<const uint8_t *>(a.logits) + row * a.stride * Y::kBytes;
  const float c2 = a.scale * 1.44269504088896f;

  // the row: `head` elements up to a 16-byte boundary, n_vec pieces, the rest
  const int head = min(a.vocab, (int)(((16 - ((uintptr_t)base & 15)) & 15) / Y::kBytes));
  const int n_vec = (a.vocab - head) / E, edge = a.vocab - n_vec * E;       // elements outside pieces: head and rest
  const uint4 *vec = reinterpret_cast<const uint4 *>(base + head * Y::kBytes);
  const int v0 = (int)((long long)n_vec * rank / cluster), v1 = (int)((long long)n_vec * (rank + 1) / cluster);
  // token asked for: loaded ahead of the pass
  int tok = -1;
  float x_tok = 0.f;
  if (rank == 0 && a.tokens && tid < a.n_tokens) {
    tok = a.tokens[row * a.tokens_stride + tid];
    if (tok >= 0 && tok < a.vocab) x_tok = Y::at(base, tok);
  }
  LogpAcc acc;
  auto edge_index = [&](int i) { return i < head ? i : n_vec * E + i; };
  const bool has_edge = rank == 0 && tid < edge;
  const float x_edge = has_edge ? Y::at(base, edge_index(tid)) : -INFINITY;
  if (has_edge) {
    if (x_edge > acc.m) acc.raise(x_edge, c2);
    acc.add(x_edge, c2);
  }
  auto take = [&](const uint4 &v) {
    float x[E];
    Y::unpack(v, x);
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < E; ++i) mx = fmaxf(mx, x[i]);
    if (mx > acc.m) acc.raise(mx, c2);
#pragma unroll
    for (int i = 0; i < E; ++i) acc.add(x[i], c2);
  };
  constexpr int kAhead = 4;
  int v = v0 + tid;
  for (; v + (kAhead - 1) * kLogpThreads < v1; v += kAhead * kLogpThreads) {
    uint4 q[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) q[i] = vec[v + i * kLogpThreads];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) take(q[i]);
  }
  for (; v < v1; v += kLogpThreads) take(vec[v]);

  // alternatives: the k-th largest of the threads' maxima
  const bool seen = acc.s > 0.f || acc.s != acc.s;
  const uint32_t mine = seen ? logp_order(acc.m) : 0u;
  if (a.top_k > 0) {
    uint32_t b = warp_sort(mine, lane);
    sm.best[warp][lane] = b;
#pragma unroll
    for (int n = 1; n < kLogpWarps; n *= 2) {
      __syncthreads();
      if ((warp & (2 * n - 1)) == 0) {
        b = warp_merge(b, sm.best[warp + n][31 - lane], lane);
        sm.best[warp][lane] = b;
      }
    }
    if (warp == 0 && lane == a.top_k - 1) sm.tau = max(b, 1u);
    __syncthreads();
    const uint32_t tau = sm.tau;
    const bool again = mine >= tau;
    if (__any_sync(0xffffffffu, again)) {
      uint64_t list = 0;                      // lane i: the warp's i-th best key
      uint64_t least = 0;                     // the k-th best one
      auto keep = [&](float x, int id, bool ok) {
        const uint32_t o = logp_order(x);
        const uint64_t key = ((uint64_t)o << 32) | (0xffffffffu - (uint32_t)id);
        uint32_t todo = __ballot_sync(0xffffffffu, ok && o >= tau && key > least);
        while (todo) {
          const int from = __ffs(todo) - 1;
          todo &= todo - 1;
          const uint64_t k = __shfl_sync(0xffffffffu, key, from);
          if (k <= least) continue;
          const int pos = __popc(__ballot_sync(0xffffffffu, list > k));
          const uint64_t up = __shfl_up_sync(0xffffffffu, list, 1);
          list = lane < pos ? list : lane == pos ? k : up;
          least = __shfl_sync(0xffffffffu, list, a.top_k - 1);
        }
      };
      keep(x_edge, has_edge ? edge_index(tid) : 0, has_edge && again);
      for (int w = v0 + warp * 32; w < v1; w += kLogpThreads) {
        const int p = w + lane;
        const bool ok = again && p < v1;
        float x[E];
        if (ok) Y::unpack(vec[p], x);
        else
#pragma unroll
          for (int i = 0; i < E; ++i) x[i] = -INFINITY;
        float mx = x[0];
#pragma unroll
        for (int i = 1; i < E; ++i) mx = fmaxf(mx, x[i]);
        if (!__any_sync(0xffffffffu, ok && logp_order(mx) >= tau)) continue;
#pragma unroll
        for (int i = 0; i < E; ++i) keep(x[i], head + p * E + i, ok);
      }
      const bool have = lane < a.top_k && list != 0;
      const uint32_t m = __ballot_sync(0xffffffffu, have);
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&sm.n_own, (uint32_t)__popc(m));
      at = __shfl_sync(0xffffffffu, at, 0);
      if (have) sm.own[at + lane] = list;
    }
  }

  // join of the block's sums
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    LogpAcc other;
    other.m = __shfl_down_sync(0xffffffffu, acc.m, o);
    other.s = __shfl_down_sync(0xffffffffu, acc.s, o);
    other.u = __shfl_down_sync(0xffffffffu, acc.u, o);
    acc.join(other, c2);
  }
  if (lane == 0) { sm.m[warp] = acc.m; sm.s[warp] = acc.s; sm.u[warp] = acc.u; }
  __syncthreads();
  // to block 0 of the cluster: the block's sums, and of its candidates the k best
  if (cluster > 1) cluster_wait();
  auto lead = [&](const void *p) { return cluster > 1 ? mapa_u32(smem_u32(p), 0) : smem_u32(p); };
  if (tid == 0) {
    LogpAcc all;
    all.m = sm.m[0]; all.s = sm.s[0]; all.u = sm.u[0];
    for (int w = 1; w < kLogpWarps; ++w) {
      LogpAcc o;
      o.m = sm.m[w]; o.s = sm.s[w]; o.u = sm.u[w];
      all.join(o, c2);
    }
    st_cluster_f32(lead(&sm.part[rank][0]), all.m);
    st_cluster_f32(lead(&sm.part[rank][1]), all.s);
    st_cluster_f32(lead(&sm.part[rank][2]), all.u);
  }
  const int n_own = a.top_k > 0 ? (int)sm.n_own : 0;
  for (int i = tid; i < n_own; i += kLogpThreads) {
    const uint64_t k = sm.own[i];
    int above = 0;
    for (int j = 0; j < n_own; ++j) above += sm.own[j] > k;
    if (above < a.top_k) st_cluster_u64(lead(&sm.key[add_cluster_u32(lead(&sm.n_all), 1u)]), k);
  }
  if (cluster > 1) cluster_sync_all(); else __syncthreads();
  if (rank != 0) return;

  LogpAcc all;
  all.m = sm.part[0][0]; all.s = sm.part[0][1]; all.u = sm.part[0][2];
  for (int r = 1; r < cluster; ++r) {
    LogpAcc o;
    o.m = sm.part[r][0]; o.s = sm.part[r][1]; o.u = sm.part[r][2];
    all.join(o, c2);
  }
  constexpr float kLn2 = 0.693147180559945f;
  const bool bad = !(all.s < INFINITY), none = all.s == 0.f;
  const float log2_s = log2f(all.s);
  auto logprob = [&](float x) { return bad ? NAN : none ? -INFINITY : (x - all.m) * a.scale - log2_s * kLn2; };
  if (tid == 0 && a.entropy) a.entropy[row] = bad ? NAN : none ? 0.f : fmaxf((log2_s - all.u / all.s) * kLn2, 0.f);
  if (a.tokens)
    for (int i = tid; i < a.n_tokens; i += kLogpThreads) {
      if (i >= kLogpThreads) {
        tok = a.tokens[row * a.tokens_stride + i];
        if (tok >= 0 && tok < a.vocab) x_tok = Y::at(base, tok);
      }
      float r = logprob(x_tok);
      if (tok < 0) r = 0.f;
      if (tok >= a.vocab) { r = NAN; atomicOr(a.status, kStatBadIndex); }
      a.logprob[row * a.n_tokens + i] = r;
    }
  if (a.top_k > 0) {
    const int n = (int)sm.n_all;
    for (int i = tid; i < n; i += kLogpThreads) {
      const uint64_t k = sm.key[i];
      int above = 0;
      for (int j = 0; j < n; ++j) above += sm.key[j] > k;
      if (above < a.top_k) {
        a.top_ids[row * a.top_k + above] = bad ? -1 : (int32_t)(0xffffffffu - (uint32_t)k);
        a.top_logprobs[row * a.top_k + above] = logprob(logp_value((uint32_t)(k >> 32)));
      }
    }
    if (tid >= n && tid < a.top_k) {
      a.top_ids[row * a.top_k + tid] = -1;
      a.top_logprobs[row * a.top_k + tid] = bad ? NAN : -INFINITY;
    }
  }
}

}  // namespace ftmoe
