// Log probabilities of given tokens, entropy and the most likely alternatives of rows of logits, in one pass over them.
// Bound: HBM (T x vocab logits read once); for few rows launch and the chain load -> exponentials -> join.
//   t = x c - r in units of log 2 (c with log2 e in it);  S = sum 2^t,  U = sum 2^t t;  lse and entropy follow from S, U and r
// A cluster of blocks shares a row while there are fewer rows than places for blocks.  Every thread walks over its 16-byte pieces of the row,
// four at a time, with a reference r = its running maximum times c, S and U of its own, which are rescaled only where four pieces bring a new
// maximum, and joined at the end in a fixed order.  The maxima also find the alternatives: where q warps have j threads each whose maximum
// reaches a value, and q j >= k, that value is a lower bound of the k-th largest logit (with q and j near the root of k hardly more than k
// reach it); so only threads whose maximum reaches it look into their pieces again, and of these only into those fours whose maximum, kept
// in 16 bits, reaches it.  The four with a thread's maximum waits in shared memory (read again from
// global memory it took 2.4 us a row, the rows under way being more than L2 holds).  The main loop thus does next to nothing for them.
// Candidates are ranked by counting, as keys (logit, then lowest id).
// Measured: 127 us for 2048 rows of 150000 in bf16 (4.8 TB/s, 0.75 of a copy's rate), 77 us for 1024 rows of 100000 floats (5.3 TB/s), 7.4 us for one
// row of 150000.
#pragma once
#include "async.cuh"
#include "cluster.cuh"
#include "common.cuh"
#include "float2.cuh"

namespace ftmoe {

constexpr int kLogpTop = 32, kLogpCluster = 8, kLogpMarks = 32;

struct LogpArgs {
  const void *logits;
  long long stride;
  int32_t T, vocab, n_tokens, top_k;
  float scale, c2, twice_c2, plain_below;      // c; c log2 e; see logp_scale
  const int32_t *tokens;
  long long tokens_stride;
  float *logprob, *entropy, *top_logprobs;
  int32_t *top_ids;
  uint32_t *status;
};

constexpr float kLogpMaxScale = 8.507059173023462e37f;   // 2^126: twice c log2 e is finite

// The scale, and below which magnitude of the maximum m exponents may be taken from the rounded product m c2: no product overflows, and |m c2| < 2^25, so
// that what the product lost in rounding, which is the maximum's own exponent, stays within 1.  (It is 64 for -1e9, where the weighted sum loses as many times
// its own rounding when that is taken out again, and some hundreds for -1e10: sums of 0 or infinity.)
inline void logp_scale(LogpArgs &a, float scale) {
  a.scale = scale;
  a.c2 = scale * 1.44269504088896f;
  a.twice_c2 = 2.f * a.c2;
  a.plain_below = a.c2 >= 1e8f ? 0.f : a.c2 < 33554432.f / 1e29f ? 1e29f : 33554432.f / a.c2;
}

enum { kLogpBf16 = 0, kLogpFp16 = 1, kLogpFp32 = 2 };
template <int TY>
struct LogpType {
  static constexpr int kBytes = TY == kLogpFp32 ? 4 : 2, kVec = 16 / kBytes;     // elements of a 16-byte piece
  // What a -infinity is raised to, so that 0 times an exponent is 0.
  static __device__ __forceinline__ float floor_value() { return TY == kLogpFp16 ? -65504.f : -1.0141204801825835e30f; }   // (-2^99.68: bf16 0xf14d)
  static __device__ __forceinline__ uint32_t floor_bits() { return TY == kLogpFp16 ? 0xfbfffbffu : TY == kLogpBf16 ? 0xf14df14du : 0xf14d0000u; }
  static __device__ __forceinline__ float at(const void *p, long long i) {
    if (TY == kLogpFp32) return static_cast<const float *>(p)[i];
    const uint16_t v = static_cast<const uint16_t *>(p)[i];
    return TY == kLogpBf16 ? bf16_bits_to_float(v) : __half2float(__ushort_as_half(v));
  }
  // Largest of the words' elements; a NaN among other values does not count.
  static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
    uint32_t d;
    if (TY == kLogpFp32) asm("max.f32 %0, %1, %2;" : "=f"(reinterpret_cast<float &>(d)) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
    else if (TY == kLogpBf16) asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ float max_of(uint32_t w) {
    float x, y;
    split(w, x, y);
    return TY == kLogpFp32 ? x : fmaxf(x, y);
  }
  // The same with a NaN counting above all.
  static __device__ __forceinline__ uint32_t max_nan(uint32_t a, uint32_t b) {
    uint32_t d;
    if (TY == kLogpFp32) asm("max.NaN.f32 %0, %1, %2;" : "=f"(reinterpret_cast<float &>(d)) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
    else if (TY == kLogpBf16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ uint32_t min_nan(uint32_t a, uint32_t b) {
    uint32_t d;
    if (TY == kLogpFp32) asm("min.NaN.f32 %0, %1, %2;" : "=f"(reinterpret_cast<float &>(d)) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
    else if (TY == kLogpBf16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ uint32_t raise_word(uint32_t a) { return max_nan(a, floor_bits()); }
  static __device__ __forceinline__ void split(uint32_t w, float &x, float &y) {
    if constexpr (TY == kLogpFp32) {
      x = y = __uint_as_float(w);
    } else if constexpr (TY == kLogpBf16) {
      x = __uint_as_float(w << 16);
      y = __uint_as_float(w & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
      x = f.x;
      y = f.y;
    }
  }
  static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[kVec]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      split(w[i], lo, hi);
      x[i * kVec / 4] = lo;
      if (TY != kLogpFp32) x[i * kVec / 4 + kVec / 4 - 1] = hi;
    }
  }
};

// The larger of both; NaN where one is.
__device__ __forceinline__ float max_or_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
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

// Half of x - m: the difference itself may pass the largest float.
__device__ __forceinline__ float half_less(float x, float m) { return fmaf(x, 0.5f, -0.5f * m); }

// Of some logits: the largest, m, and the sums of 2^t and 2^t t with t = x c2 - (m c2 + del); del is what the product m c2 lost when it was
// rounded, so that sums with different references can be joined exactly.  m = -infinity: none yet (s then is 0, or NaN).
struct LogpAcc {
  float m = -INFINITY, del = 0.f, s = 0.f, u = 0.f;
  __device__ __forceinline__ void rescale(float to_m, float to_del, float twice_c2) {
    const float d = fmaf(half_less(m, to_m), twice_c2, del - to_del);
    if (!(d >= -200.f)) {                 // (-infinity and NaN too: what there is, a NaN stays)
      if (s == s) s = 0.f;
      u = 0.f;
    } else {
      const float f = exp2_approx(d);
      u = f * fmaf(d, s, u);
      s *= f;
    }
    m = to_m;
    del = to_del;
  }
};

template <int WARPS>
struct LogpSmem {
  uint32_t top[WARPS], nth[WARPS];                     // of the warps' maxima the largest, the j-th largest (logp_order)
  float sum[2][WARPS];
  uint4 four[4][WARPS * 32];                           // the thread's four with its maximum
  uint16_t mark[kLogpMarks][WARPS * 32];               // maxima of a thread's fours, as the upper half of logp_order
  uint64_t key[kLogpCluster * kLogpTop];               // block 0 of the cluster: candidates of all blocks
  uint64_t own[WARPS * kLogpTop];
  float part[kLogpCluster][2];                         // and of all blocks: sums, maxima
  uint32_t part_top[kLogpCluster];
  uint32_t n_own, n_all;
};

__device__ __forceinline__ void st_cluster_u64(uint32_t addr, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory"); }
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ uint32_t add_cluster_u32(uint32_t addr, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(addr), "r"(v) : "memory");
  return old;
}

template <int TY, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 512 ? 1 : 1024 / THREADS) logprobs_kernel(const LogpArgs a, const int cluster) {
  using Y = LogpType<TY>;
  constexpr int E = Y::kVec, kWarps = THREADS / 32, kAhead = 4;
  extern __shared__ __align__(16) unsigned char smem[];
  LogpSmem<kWarps> &sm = *reinterpret_cast<LogpSmem<kWarps> *>(smem);
  grid_let_next();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x % cluster;
  const long long row = blockIdx.x / cluster;
  if (tid == 0) sm.n_own = sm.n_all = 0;
  if (cluster > 1) cluster_arrive();
  grid_wait();
  const uint8_t *base = static_cast<const uint8_t *>(a.logits) + row * a.stride * Y::kBytes;
  const float c2 = a.c2;

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
  // `plain`: exponents in one instruction from the rounded product ref = m c2, -infinities at the floor; not where the floor would count, or beyond
  // plain_below.  Else the difference is taken first.
  LogpAcc acc;
  float ref = 0.f;
  bool plain = false;
  auto raise = [&](float to) {
    plain = fabsf(to) < a.plain_below && (Y::floor_value() - to) * c2 < -200.f;
    ref = plain ? to * c2 : 0.f;
    acc.rescale(to, plain ? -fmaf(to, c2, -ref) : 0.f, a.twice_c2);
  };
  auto add_one = [&](float x) {                  // any x, not above the maximum, which is not -infinity (x = -infinity counts nothing)
    const float t = max_or_nan(plain ? fmaf(x, c2, -ref) : half_less(x, acc.m) * a.twice_c2, -1000.f), e = exp2_approx(t);
    acc.s += e;
    acc.u = fmaf(e, t, acc.u);
  };
  // plain: two logits at a time, in packed arithmetic
  auto add_pair = [&](float x, float y, uint64_t c22, uint64_t ref2, uint64_t &s2, uint64_t &u2) {
    const uint64_t t = fma2(f2(x, y), c22, ref2);
    float t0, t1;
    f2_split(t, t0, t1);
    const uint64_t e = f2(exp2_approx(t0), exp2_approx(t1));
    s2 = add2(s2, e);
    u2 = fma2(e, t, u2);
  };
  auto edge_index = [&](int i) { return i < head ? i : n_vec * E + i; };
  const bool has_edge = rank == 0 && tid < edge;
  const float x_edge = has_edge ? Y::at(base, edge_index(tid)) : -INFINITY;
  if (has_edge) {
    if (x_edge > acc.m) raise(x_edge);
    if (x_edge != -INFINITY) add_one(x_edge);
  }
  // fours of pieces; several fours to a mark where a thread has many
  const int fours = (v1 - v0 + kAhead * THREADS - 1) / (kAhead * THREADS);
  int shift = 0;
  while ((fours - 1) >> shift >= kLogpMarks) ++shift;
  int best_four = -1;
  auto take = [&](const uint4 (&q)[kAhead], int four) {
    uint32_t mx = Y::max_word(Y::max_word(q[0].x, q[0].y), Y::max_word(q[0].z, q[0].w));
#pragma unroll
    for (int i = 1; i < kAhead; ++i) mx = Y::max_word(mx, Y::max_word(Y::max_word(q[i].x, q[i].y), Y::max_word(q[i].z, q[i].w)));
    const float top = Y::max_of(mx);
    if (a.top_k > 0) {
      const uint16_t now = (uint16_t)(logp_order(top) >> 16);
      if (shift == 0) sm.mark[four][tid] = now;
      else {
        uint16_t &mark = sm.mark[four >> shift][tid];
        mark = (four & ((1 << shift) - 1)) == 0 || now > mark ? now : mark;
      }
    }
    if (top > acc.m) {
      raise(top);
      best_four = four;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) sm.four[i][tid] = q[i];
    }
    if (plain) {
      const uint64_t c22 = f2(c2, c2), ref2 = f2(-ref, -ref);
      uint64_t s2 = f2(acc.s, 0.f), u2 = f2(acc.u, 0.f);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
        for (int j = 0; j < 4; j += TY == kLogpFp32 ? 2 : 1) {
          float x, y;
          Y::split(Y::raise_word(w[j]), x, y);
          if (TY == kLogpFp32) y = __uint_as_float(Y::raise_word(w[j + 1 < 4 ? j + 1 : j]));
          add_pair(x, y, c22, ref2, s2, u2);
        }
      }
      float lo, hi;
      f2_split(s2, lo, hi);
      acc.s = lo + hi;
      f2_split(u2, lo, hi);
      acc.u = lo + hi;
    } else if (acc.m == -INFINITY) {             // nothing but -infinities, or NaN among them
      uint32_t any = 0xff800000u;
      if (TY == kLogpBf16) any = 0xff80ff80u;
      if (TY == kLogpFp16) any = 0xfc00fc00u;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) any = Y::max_nan(Y::max_nan(any, Y::max_nan(q[i].x, q[i].y)), Y::max_nan(q[i].z, q[i].w));
      float x, y;
      Y::split(any, x, y);
      if (x != x || y != y) acc.s = NAN;
    } else {
      // (where a mask's value is all that a thread has seen, as a rule all elements are that)
      uint32_t least = Y::min_nan(Y::min_nan(q[0].x, q[0].y), Y::min_nan(q[0].z, q[0].w));
#pragma unroll
      for (int i = 1; i < kAhead; ++i) least = Y::min_nan(least, Y::min_nan(Y::min_nan(q[i].x, q[i].y), Y::min_nan(q[i].z, q[i].w)));
      float lo, hi;
      Y::split(least, lo, hi);
      if (lo == acc.m && hi == acc.m && lo < INFINITY) {
        acc.s += (float)(kAhead * E);
      } else {
#pragma unroll 1
        for (int i = 0; i < kAhead; ++i) {
          const uint4 p = i == 0 ? q[0] : i == 1 ? q[1] : i == 2 ? q[2] : q[3];
          float x[E];
          Y::unpack(p, x);
#pragma unroll
          for (int j = 0; j < E; ++j) add_one(x[j]);
        }
      }
    }
  };
  constexpr uint32_t kNone = TY == kLogpFp32 ? 0xff800000u : TY == kLogpBf16 ? 0xff80ff80u : 0xfc00fc00u;      // -infinities
  auto load = [&](uint4 (&q)[kAhead], int four) {
    if (v0 + (four + 1) * kAhead * THREADS <= v1) {
      const uint4 *p = vec + v0 + four * kAhead * THREADS + tid;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) q[i] = ld_stream_16(p + i * THREADS);
      return;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int v = v0 + (four * kAhead + i) * THREADS + tid;
      q[i] = make_uint4(kNone, kNone, kNone, kNone);
      if (v < v1) q[i] = ld_stream_16(vec + v);
    }
  };
  // (the next four are on their way while one is taken)
  uint4 qa[kAhead], qb[kAhead];
  if (fours > 0) load(qa, 0);
  for (int f = 0; f < fours; f += 2) {
    if (f + 1 < fours) load(qb, f + 1);
    take(qa, f);
    if (f + 1 < fours) {
      if (f + 2 < fours) load(qa, f + 2);
      take(qb, f + 1);
    }
  }

  // the block's largest logit, and the bound for the alternatives
  const uint32_t mine = logp_order(acc.m);
  int q = 1;
  while (q < kWarps && q * q < a.top_k) ++q;
  {
    uint32_t nth = 0, left = mine;
    const uint32_t top = __reduce_max_sync(0xffffffffu, mine);
    for (int j = 0; j < a.top_k; j += q) {               // ceil(k / q) times
      nth = __reduce_max_sync(0xffffffffu, left);
      if (lane == __ffs(__ballot_sync(0xffffffffu, left == nth)) - 1) left = 0;
    }
    if (lane == 0) { sm.top[warp] = top; sm.nth[warp] = nth; }
  }
  __syncthreads();
  const uint32_t block_top = __reduce_max_sync(0xffffffffu, lane < kWarps ? sm.top[lane] : 0u);
  if (a.top_k > 0) {
    const uint32_t nth = lane < kWarps ? sm.nth[lane] : 0u;
    int above = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const uint32_t o = __shfl_sync(0xffffffffu, nth, i);
      above += o > nth || (o == nth && i < lane);
    }
    const uint32_t tau = max(__shfl_sync(0xffffffffu, nth, __ffs(__ballot_sync(0xffffffffu, lane < kWarps && above == q - 1)) - 1), 1u);
    const bool again = mine >= tau;
    const int marks = fours > 0 ? ((fours - 1) >> shift) + 1 : 0;
    const uint16_t tau_mark = (uint16_t)(tau >> 16);
    // as a rule a few more than k reach it: each thread adds its own to the block's list
    if (again) {
      bool room = true;
      auto add = [&](float x, int id) {
        const uint32_t o = logp_order(x);
        if (o < tau || !room) return;
        const uint32_t at = atomicAdd(&sm.n_own, 1u);
        room = at < kWarps * kLogpTop;
        if (room) sm.own[at] = ((uint64_t)o << 32) | (0xffffffffu - (uint32_t)id);
      };
      if (has_edge) add(x_edge, edge_index(tid));
      auto look = [&](const uint4 (&q)[kAhead], int f) {
#pragma unroll 1
        for (int i = 0; i < kAhead; ++i) {
          const uint4 p = i == 0 ? q[0] : i == 1 ? q[1] : i == 2 ? q[2] : q[3];
          if (logp_order(Y::max_of(Y::max_word(Y::max_word(p.x, p.y), Y::max_word(p.z, p.w)))) < tau) continue;
          float x[E];
          Y::unpack(p, x);
          const int id = head + (v0 + (f * kAhead + i) * THREADS + tid) * E;
#pragma unroll
          for (int j = 0; j < E; ++j) add(x[j], id + j);
        }
      };
      if (best_four >= 0) {                    // (the maximum may stand outside the pieces)
        uint4 q[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) q[i] = sm.four[i][tid];
        look(q, best_four);
      }
      // (each thread to its own next mark first, so that a warp's loads go out together)
      for (int k = -1; room;) {
        while (++k < marks && (sm.mark[k][tid] < tau_mark || (shift == 0 && k == best_four))) {
        }
        if (k >= marks) break;
        for (int f = k << shift; f < min(fours, (k + 1) << shift); ++f) {
          if (f == best_four) continue;
          load(qb, f);
          look(qb, f);
        }
      }
    }
    __syncthreads();
    // more of them (many equal logits, say): the warps keep lists of their k best
    const bool many = sm.n_own > kWarps * kLogpTop;
    __syncthreads();
    if (many) {
      if (tid == 0) sm.n_own = 0;
      __syncthreads();
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
        for (int k = 0; k < marks; ++k) {
          const bool on = again && sm.mark[k][tid] >= tau_mark;
          if (!__any_sync(0xffffffffu, on)) continue;
          for (int f = k << shift; f < min(fours, (k + 1) << shift); ++f) {
            uint4 q[kAhead];
            load(q, f);
#pragma unroll 1
            for (int i = 0; i < kAhead; ++i) {
              const uint4 p = i == 0 ? q[0] : i == 1 ? q[1] : i == 2 ? q[2] : q[3];
              float x[E];
              Y::unpack(p, x);
              float mx = x[0];
#pragma unroll
              for (int j = 1; j < E; ++j) mx = fmaxf(mx, x[j]);
              if (!__any_sync(0xffffffffu, logp_order(mx) >= tau)) continue;
              const int id = head + (v0 + (f * kAhead + i) * THREADS + tid) * E;
#pragma unroll 1
              for (int j = 0; j < E; ++j) {
                float xj = x[0];
#pragma unroll
                for (int l = 1; l < E; ++l) xj = j == l ? x[l] : xj;
                keep(xj, id + j, on);
              }
            }
          }
        }
        const bool have = lane < a.top_k && list != 0;
        const uint32_t mask = __ballot_sync(0xffffffffu, have);
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&sm.n_own, (uint32_t)__popc(mask));
        at = __shfl_sync(0xffffffffu, at, 0);
        if (have) sm.own[at + lane] = list;
      }
    }
  }

  // the block's sums, all with its largest logit as reference
  auto sum_lanes = [&](float &x, float &y) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      x += __shfl_xor_sync(0xffffffffu, x, o);
      y += __shfl_xor_sync(0xffffffffu, y, o);
    }
  };
  auto value = [](uint32_t o) { return o ? logp_value(o) : -INFINITY; };
  acc.rescale(value(block_top), 0.f, a.twice_c2);
  sum_lanes(acc.s, acc.u);
  if (lane == 0) { sm.sum[0][warp] = acc.s; sm.sum[1][warp] = acc.u; }
  __syncthreads();
  // to block 0 of the cluster: the block's sums, and of its candidates the k best
  if (cluster > 1) cluster_wait();
  auto lead = [&](const void *p) { return cluster > 1 ? mapa_u32(smem_u32(p), 0) : smem_u32(p); };
  if (warp == 0) {
    float x = lane < kWarps ? sm.sum[0][lane] : 0.f, y = lane < kWarps ? sm.sum[1][lane] : 0.f;
    sum_lanes(x, y);
    if (lane == 0) {
      st_cluster_u32(lead(&sm.part_top[rank]), block_top);
      st_cluster_f32(lead(&sm.part[rank][0]), x);
      st_cluster_f32(lead(&sm.part[rank][1]), y);
    }
  }
  const int n_own = a.top_k > 0 ? (int)sm.n_own : 0;
  for (int i = tid; i < n_own; i += THREADS) {
    const uint64_t k = sm.own[i];
    int above = 0;
    for (int j = 0; j < n_own; ++j) above += sm.own[j] > k;
    if (above < a.top_k) st_cluster_u64(lead(&sm.key[add_cluster_u32(lead(&sm.n_all), 1u)]), k);
  }
  if (cluster > 1) cluster_sync_all(); else __syncthreads();
  if (rank != 0) return;

  // every warp joins the cluster's sums, in the same order
  LogpAcc all;
  {
    const bool mine_too = lane < cluster;
    const uint32_t o = mine_too ? sm.part_top[lane] : 0u, top = __reduce_max_sync(0xffffffffu, o);
    if (mine_too) { all.m = value(o); all.s = sm.part[lane][0]; all.u = sm.part[lane][1]; }
    all.rescale(value(top), 0.f, a.twice_c2);
    sum_lanes(all.s, all.u);
  }
  constexpr float kLn2 = 0.693147180559945f;
  const bool bad = !(all.s < INFINITY), none = all.s == 0.f;
  const float log2_s = log2f(all.s), rest = log2_s * kLn2;
  auto logprob = [&](float x) { return bad ? NAN : none ? -INFINITY : fmaf(half_less(x, all.m), 2.f * a.scale, -rest); };
  if (tid == 0 && a.entropy) a.entropy[row] = bad ? NAN : none ? 0.f : fmaxf((log2_s - all.u / all.s) * kLn2, 0.f);
  if (a.tokens)
    for (int i = tid; i < a.n_tokens; i += THREADS) {
      if (i >= THREADS) {
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
    for (int i = tid; i < n; i += THREADS) {
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
