// Log probabilities of given tokens, with the entropy and the likeliest alternatives, and
// the gradient with respect to the logits.
//
// For a row z_j = logits_j / temperature over the allowed j, with m the running maximum:
//   S = sum e^(z_j - m),  A = sum (z_j - m) e^(z_j - m)
//   lse = m + log S,  logp = z_t - lse,  entropy = log S - A / S
// in one pass: each thread keeps its own (m, S, A) and rescales the sums when m grows; the
// partial sums of threads and CTAs join by the same rule.  Sums are in units of log 2, since
// the hardware's exponential is 2^x.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxWarps = 16;
constexpr int kUnroll = 4;            // 16-byte loads in flight a thread
constexpr int kCap = 2048;            // candidates kept before they are cut to the best
constexpr int kMaxTop = 32;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct Stat {
  float m, S, A;      // m: largest logit as given (before the temperature)
};

// Logits at or below this count as not allowed, so a mask written with the lowest finite value
// of bf16 or fp32 works as one of minus infinity does.  They are raised to it on loading, which
// keeps every difference finite, and a row whose largest logit it is has no class.  (bf16: the
// largest value of the type that is not above -1e30.)
template <typename T> constexpr float kNone = -1e30f;
template <> constexpr float kNone<__nv_bfloat16> = -1.0002555517425873e30f;

// Order of floats (no NaN) as unsigned integers, and back: 2^31 plus or minus the magnitude's bits, so
// that zeros of both signs are the same.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u & 0x80000000u ? 0u - u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : 0u - o);
}

// The warp's sums, the same in every lane; c = log2(e) / temperature.
__device__ __forceinline__ Stat warp_join(Stat s, float c) {
  const float m = from_ordered(__reduce_max_sync(~0u, ordered(s.m)));
  const float d = max_nan((s.m - m) * c, -200.0f), e = exp2_fast(d);
  Stat r = {m, s.S * e, (s.A + s.S * d) * e};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r.S += __shfl_xor_sync(~0u, r.S, o);
    r.A += __shfl_xor_sync(~0u, r.A, o);
  }
  return r;
}

// Keys order by value, equal values by lower index.
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
  return (static_cast<uint64_t>(ordered(v)) << 32) | static_cast<uint32_t>(~index);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  return from_ordered(static_cast<uint32_t>(k >> 32));
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return ~static_cast<uint32_t>(k); }
// 0 orders below the key of every value, minus infinity's among them.

struct FwdArgs {
  const void* logits;
  const void* targets;
  const uint8_t* allowed;
  int64_t rows, classes, ld, allowed_ld;
  float inv_t;
  int top;
  bool wide_targets;
  float *logp, *entropy, *lse, *top_logp;
  int* top_index;
};

struct TopState {
  uint64_t keys[kCap];
  uint64_t best[kMaxTop];
  uint64_t bar;                    // keys below it are not among the best
  uint32_t warp_low[kMaxWarps];
  int count;
};

// Descending bitonic sort of keys[0, n), n a power of two, by the whole CTA.
template <int THREADS>
__device__ __noinline__ void sort_keys(uint64_t* keys, int n) {
  for (int k = 2; k <= n; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < n / 2; i += THREADS) {
        const int x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x | j;
        const uint64_t a = keys[x], b = keys[y];
        const bool down = (x & k) == 0;
        if (down ? a < b : a > b) {
          keys[x] = b;
          keys[y] = a;
        }
      }
    }
  __syncthreads();
}

// Keeps the best `top` candidates, in order; the bar rises to the last of them.  Few
// candidates (the common case) are ranked by counting the larger ones, by all threads at
// once: `per` neighbours share a candidate.
template <int THREADS>
__device__ __noinline__ void cut(TopState& s, int top) {
  __syncthreads();
  const int count = min(s.count, kCap), tid = threadIdx.x;
  if (count <= THREADS) {
    int per = 32;
    while (per > 1 && count * per > THREADS) per >>= 1;
    const int c = tid / per, part = tid % per;
    const uint64_t k = c < count ? s.keys[c] : ~0ull;
    int rank = 0;
#pragma unroll 4
    for (int i = part; i < count; i += per) rank += s.keys[i] > k;
    for (int o = per >> 1; o > 0; o >>= 1) rank += __shfl_xor_sync(~0u, rank, o);
    if (c < count && part == 0 && rank < top) s.best[rank] = k;
    __syncthreads();
    if (tid < min(count, top)) s.keys[tid] = s.best[tid];
  } else {
    int n = 2 * THREADS;
    while (n < count) n <<= 1;
    for (int i = count + tid; i < n; i += THREADS) s.keys[i] = 0;
    sort_keys<THREADS>(s.keys, n);
  }
  if (tid == 0) s.count = min(count, top);
  __syncthreads();
  if (tid == 0 && count >= top) s.bar = s.keys[top - 1];
  __syncthreads();
}

// The same place of shared memory in CTA `rank` of the cluster.
template <typename T>
__device__ __forceinline__ T from_cta(const T* p, int rank) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "word or double word");
  const uint32_t la = static_cast<uint32_t>(__cvta_generic_to_shared(p));
  uint32_t ra;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(la), "r"(rank));
  if constexpr (sizeof(T) == 4) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(ra) : "memory");
    return *reinterpret_cast<T*>(&v);
  } else {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(ra) : "memory");
    return *reinterpret_cast<T*>(&v);
  }
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename T> constexpr int kVec = 16 / sizeof(T);
template <typename T> constexpr bool kIsBf16 = false;
template <> constexpr bool kIsBf16<__nv_bfloat16> = true;

template <typename T>
__device__ __forceinline__ void unpack(uint4 w, float* v) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
  } else {
    widen2<T>(w.x, v[0], v[1]); widen2<T>(w.y, v[2], v[3]);
    widen2<T>(w.z, v[4], v[5]); widen2<T>(w.w, v[6], v[7]);
  }
}

// Raises a vector's entries to kNone where they are below it or not allowed; returns the
// largest (not a NaN).  16-bit entries stay packed, two to an instruction.
template <typename T>
__device__ __forceinline__ float clean(uint4& w, const uint8_t* ok) {
  constexpr int N = kVec<T>;
  uint32_t* x = &w.x;
  if (ok) {
    uint32_t m[2];
    if ((reinterpret_cast<uintptr_t>(ok) & (N - 1)) == 0) {
      m[0] = *reinterpret_cast<const uint32_t*>(ok);
      if constexpr (N == 8) m[1] = *reinterpret_cast<const uint32_t*>(ok + 4);
    } else {
#pragma unroll
      for (int h = 0; h < N / 4; ++h)
        m[h] = ok[4 * h] | (ok[4 * h + 1] << 8) | (ok[4 * h + 2] << 16) | (ok[4 * h + 3] << 24);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool out = ((m[i >> 2] >> (8 * (i & 3))) & 0xFFu) == 0;
      if constexpr (N == 4) {
        if (out) x[i] = 0xFF800000u;                       // minus infinity
      } else {
        constexpr uint32_t inf = sizeof(T) == 2 && kIsBf16<T> ? 0xFF80u : 0xFC00u;
        if (out) x[i >> 1] = i & 1 ? (x[i >> 1] & 0xFFFFu) | (inf << 16) : (x[i >> 1] & 0xFFFF0000u) | inf;
      }
    }
  }
  float top;
  if constexpr (kIsBf16<T>) {
    const __nv_bfloat162 low = __float2bfloat162_rn(kNone<T>);
    __nv_bfloat162 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&x[i]), low);
      x[i] = *reinterpret_cast<const uint32_t*>(&h[i]);
    }
    const __nv_bfloat162 t = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    top = fmaxf(__low2float(t), __high2float(t));
  } else if constexpr (sizeof(T) == 2) {
    __half2 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = *reinterpret_cast<const __half2*>(&x[i]);
    const __half2 t = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    top = fmaxf(__low2float(t), __high2float(t));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(max_nan(__uint_as_float(x[i]), kNone<T>));
    top = fmaxf(fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])),
                fmaxf(__uint_as_float(x[2]), __uint_as_float(x[3])));
  }
  return top;
}

// A thread's sums, over even and odd entries apart.
struct Sums {
  float m;
  Pair S, A;
};
// A new largest value: the sums are rescaled to it.
__device__ __forceinline__ void raise(Sums& s, float top, float c) {
  if (top > s.m) {
    const float d = max_nan((s.m - top) * c, -200.0f), e = exp2_fast(d);
    s.A = mul2(fma2(s.S, pair(d, d), s.A), pair(e, e));
    s.S = mul2(s.S, pair(e, e));
    s.m = top;
  }
}
__device__ __forceinline__ void add_pair(Sums& s, float a, float b, float c) {
  const Pair d = mul2(add2(pair(a, b), pair(-s.m, -s.m)), pair(c, c));
  float x, y;
  halves(d, x, y);
  const Pair e = pair(exp2_fast(x), exp2_fast(y));
  s.S = add2(s.S, e);
  s.A = fma2(e, d, s.A);
}
template <typename T>
__device__ __forceinline__ void add_vec(Sums& s, const uint4& w, float c) {
  float v[kVec<T>];
  unpack<T>(w, v);
  if constexpr (sizeof(T) == 2 && !kIsBf16<T>) {
    // minus infinity in fp16 has not been raised yet
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v[i] = max_nan(v[i], kNone<T>);
  }
#pragma unroll
  for (int i = 0; i < kVec<T>; i += 2) add_pair(s, v[i], v[i + 1], c);
}

__device__ __forceinline__ int64_t target_of(const void* targets, bool wide, int64_t row) {
  return wide ? static_cast<const int64_t*>(targets)[row] : static_cast<const int*>(targets)[row];
}

// The sum A of a row whose distances to the largest logit pass fp32's range (logits near its end, a
// temperature near 0): 0 * inf, which is NaN where S is not.  The row is then summed once more, by
// one CTA, with the distances cut off where 2^d is 0 (a cut in the loop above would cost every row).
template <typename T, int THREADS>
__device__ __noinline__ float sum_again(const T* z, const uint8_t* ok, int classes, float m, float c, float* part) {
  float A = 0.0f;
  for (int j = threadIdx.x; j < classes; j += THREADS) {
    const float v = Elem<T>::up(z[j]);
    if (!(v > kNone<T>) || (ok && !ok[j])) continue;
    const float d = fmaxf((v - m) * c, -200.0f);
    A = fmaf(exp2_fast(d), d, A);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) A += __shfl_xor_sync(~0u, A, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = A;
  __syncthreads();
  A = 0.0f;
  for (int w = 0; w < THREADS / 32; ++w) A += part[w];
  return A;
}

// One cluster a row; its CTAs take equal shares of the row's 16-byte vectors.
template <typename T, bool TOP, bool MASK, int THREADS>
__global__ void __launch_bounds__(THREADS, (TOP ? 1024 : 1536) / THREADS) k_logprobs(const __grid_constant__ FwdArgs a) {
  constexpr int V = kVec<T>, kWarps = THREADS / 32;
  __shared__ Stat warp_stat[kWarps];
  __shared__ Stat cta_stat, row_stat;
  __shared__ float again[kWarps];
  extern __shared__ __align__(16) unsigned char dyn[];
  TopState& ts = *reinterpret_cast<TopState*>(dyn);

  uint32_t rank, parts;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const int64_t row = blockIdx.x / parts;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const uint8_t* ok = MASK ? a.allowed + row * a.allowed_ld : nullptr;
  const int tid = threadIdx.x, lane = tid & 31;
  const float c = a.inv_t * kLog2e;
  const int classes = static_cast<int>(a.classes);

  // The vectors start at the row's first 16-byte boundary; the entries before and after
  // them are taken one by one, by the first and the last CTA.
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int head = min(classes, shift ? V - shift : 0);
  const int vecs = (classes - head) / V;
  const int v0 = static_cast<int>(static_cast<int64_t>(vecs) * rank / parts);
  const int v1 = static_cast<int>(static_cast<int64_t>(vecs) * (rank + 1) / parts);
  const int tail = head + vecs * V;
  const T* zv = z + head;
  const uint8_t* okv = MASK ? ok + head : nullptr;

  Sums sums = {kNone<T>, pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
  if (TOP) {
    if (tid == 0) {
      ts.count = 0;
      ts.bar = 0;
    }
    __syncthreads();
  }

  // What is left over of the row: at most 2 (V - 1) entries.
  int one = -1;
  float one_z = kNone<T>;
  if (rank == 0 && tid < head) one = tid;
  if (rank == parts - 1 && tid >= 32 && tail + tid - 32 < classes) one = tail + tid - 32;
  if (one >= 0 && (!MASK || ok[one])) {
    one_z = max_nan(Elem<T>::up(z[one]), kNone<T>);
    sums.m = one_z;
    sums.S = pair(1.0f, 0.0f);
  }

  for (int r = v0; r < v1; r += THREADS * kUnroll) {
    uint4 w[kUnroll];
    float top[kUnroll];
    const bool whole = r + THREADS * kUnroll <= v1;     // without checks
    if (whole) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) w[u] = __ldcs(reinterpret_cast<const uint4*>(zv) + r + u * THREADS + tid);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        top[u] = clean<T>(w[u], MASK ? okv + (r + u * THREADS + tid) * V : nullptr);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = r + u * THREADS + tid;
        top[u] = kNone<T>;
        if (i < v1) w[u] = __ldcs(reinterpret_cast<const uint4*>(zv) + i);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = r + u * THREADS + tid;
        if (i < v1) top[u] = clean<T>(w[u], MASK ? okv + i * V : nullptr);
      }
    }
    raise(sums, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), c);
    static_assert(kUnroll == 4, "");
    if (whole) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) add_vec<T>(sums, w[u], c);
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (r + u * THREADS + tid < v1) add_vec<T>(sums, w[u], c);
    }
  }

  if (TOP) {
    // A bound from below for the best: each of the warps whose threads all have entries has `share`
    // threads whose largest reaches the warp's bound, those warps together at least `top` entries.
    // (With idle warps among them there would be no bound: 1 row of 2048, 20 best, 23 us.)
    const int full = max(1, min(kWarps, (v1 - v0) / 32)), share = (a.top + full - 1) / full, warp = tid >> 5;
    const uint32_t most = ordered(sums.m);
    uint32_t left = most, low = 0;
    for (int i = 0; i < share; ++i) {
      low = __reduce_max_sync(~0u, left);
      // the threads that hold it are many only for equal values; one of them leaves
      if (lane == __ffs(__ballot_sync(~0u, left == low)) - 1) left = 0;
    }
    if (lane == 0) ts.warp_low[warp] = warp < full ? low : ~0u;
    __syncthreads();
    low = __reduce_min_sync(~0u, ts.warp_low[lane % kWarps]);
    // Entries over the bar become candidates.  They are among the vectors of the threads whose
    // largest entry is over it; the lanes of a warp read such threads' vectors again together,
    // `per` lanes a thread.  What finds no room waits until the candidates have been cut to
    // the best and the bar raised.
    uint32_t hot = __ballot_sync(~0u, sums.m > kNone<T> && most >= low);
    bool one_done = !(one_z > kNone<T>);
    int per = 1;
    while (per < 32 && v0 + per * THREADS < v1) per *= 2;
    const int skip = lane / per;
    int j0 = 0;                                       // first of the threads' vectors
    uint32_t done = 0;                                // entries of this lane's vector
    while (true) {
      uint64_t bar = static_cast<uint64_t>(low) << 32;
      if (ts.bar > bar) bar = ts.bar;
      const float bar_value = key_value(bar);
      auto offer = [&](float x, int index) {          // false: no room
        const uint64_t k = key_of(x, static_cast<uint32_t>(index));
        if (!(x > kNone<T>) || k < bar) return true;
        const int place = atomicAdd(&ts.count, 1);
        if (place < kCap) ts.keys[place] = k;
        return place < kCap;
      };
      if (!one_done) one_done = offer(one_z, one);
      bool waiting = !one_done;
      while (hot && !__any_sync(~0u, waiting)) {
        uint32_t rest = hot;
        for (int x = 0; x < skip; ++x) rest &= rest - 1;
        const int i = v0 + (j0 + lane % per) * THREADS + warp * 32 + __ffs(rest) - 1;
        if (rest && i < v1) {
          uint4 x = *(reinterpret_cast<const uint4*>(zv) + i);
          if (!(clean<T>(x, MASK ? okv + i * V : nullptr) < bar_value)) {
            float v[V];
            unpack<T>(x, v);
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (!(done >> e & 1u)) {
                if (offer(v[e], head + i * V + e)) done |= 1u << e;
                else waiting = true;
              }
          }
        }
        if (__any_sync(~0u, waiting)) break;
        done = 0;
        j0 += per;
        if (v0 + j0 * THREADS >= v1) {
          j0 = 0;
          for (int x = 0; x < 32 / per; ++x) hot &= hot - 1;
        }
      }
      if (!__syncthreads_or(waiting)) break;
      cut<THREADS>(ts, a.top);
    }
  }

  // Threads, warps and CTAs of the row join their sums.
  Stat s = {sums.m, 0.0f, 0.0f};
  {
    float x, y;
    halves(sums.S, x, y);
    s.S = x + y;
    halves(sums.A, x, y);
    s.A = x + y;
  }
  s = warp_join(s, c);
  if (lane == 0) warp_stat[tid >> 5] = s;
  if (TOP) cut<THREADS>(ts, a.top);
  __syncthreads();
  if (tid < 32) {
    s = warp_join(tid < kWarps ? warp_stat[tid] : Stat{kNone<T>, 0.0f, 0.0f}, c);
    if (tid == 0) cta_stat = s;
  }
  if (parts > 1) {
    cluster_barrier();
    if (rank == 0) {
      if (tid < 32) {
        // one lane a CTA (at most kMaxCluster), so that their loads are in flight together
        s = {kNone<T>, 0.0f, 0.0f};
        if (tid < static_cast<int>(parts))
          s = {from_cta(&cta_stat.m, tid), from_cta(&cta_stat.S, tid), from_cta(&cta_stat.A, tid)};
        s = warp_join(s, c);
        if (tid == 0) row_stat = s;
      }
      if (TOP) {
        // the other CTAs' best after this one's
        for (int i = tid; i < static_cast<int>(parts - 1) * kMaxTop; i += THREADS) {
          const int q = 1 + i / kMaxTop, k = i % kMaxTop;
          const uint64_t key = from_cta(&ts.keys[k], q);
          if (k < from_cta(&ts.count, q)) ts.keys[atomicAdd(&ts.count, 1)] = key;
        }
        cut<THREADS>(ts, a.top);
      }
    }
    cluster_barrier();
    if (rank != 0) return;
    s = row_stat;
  } else {
    __syncthreads();
    s = cta_stat;
  }
  if (s.A != s.A && s.S == s.S) s.A = sum_again<T, THREADS>(z, ok, classes, s.m, c, again);

  const float log_s = log2f(s.S);
  const bool none = !(s.m > kNone<T>) && s.S == s.S;       // NaN stays
  const float lse = none ? -INFINITY : fmaf(s.m, a.inv_t, log_s * kLn2);
  if (tid == 0) {
    const int64_t t = target_of(a.targets, a.wide_targets, row);
    float lp = 0.0f;
    if (t >= a.classes) {
      lp = NAN;
    } else if (t >= 0) {
      float zt = Elem<T>::up(z[t]);
      if (zt <= kNone<T> || (MASK && !ok[t])) zt = -INFINITY;
      lp = none ? -INFINITY : fmaf(zt - s.m, a.inv_t, -log_s * kLn2);
    }
    a.logp[row] = lp;
    a.entropy[row] = none ? 0.0f : (log_s - s.A / s.S) * kLn2;
    a.lse[row] = lse;
  }
  if (TOP && tid < a.top) {
    const bool has = tid < ts.count && !none && lse == lse;
    const uint64_t k = has ? ts.keys[tid] : 0;
    a.top_logp[row * a.top + tid] =
        has ? fmaf(key_value(k) - s.m, a.inv_t, -log_s * kLn2) : (lse != lse ? NAN : -INFINITY);
    a.top_index[row * a.top + tid] = has ? static_cast<int>(key_index(k)) : -1;
  }
}

// ---- rows of few classes: a warp a row, which stays in its lanes' registers
// The maximum is known before the sums, so nothing is rescaled; the likeliest are taken from the
// lanes' own one after the other.  Only the latency of a row counts here, and warps hide it for one
// another (8192 rows of 10, fp32: 3.3 us, 22 with a CTA a row; 8192 of 1000, bf16: 8.6 and 23; 100000 of 16: 20
// and 239).
constexpr int kRowWarps = 8;
constexpr int kRowUnroll = 8;          // loads in flight of the gradient
template <typename T, bool TOP, int R>
__global__ void __launch_bounds__(kRowWarps * 32) k_logprobs_row(const __grid_constant__ FwdArgs a) {
  const int lane = threadIdx.x & 31, classes = static_cast<int>(a.classes);
  const float c = a.inv_t * kLog2e;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRowWarps;
  for (int64_t row = blockIdx.x * static_cast<int64_t>(kRowWarps) + (threadIdx.x >> 5); row < a.rows; row += step) {
    const T* z = static_cast<const T*>(a.logits) + row * a.ld;
    const uint8_t* ok = a.allowed ? a.allowed + row * a.allowed_ld : nullptr;
    const int64_t t = target_of(a.targets, a.wide_targets, row);
    float v[R];
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int j = u * 32 + lane;
      v[u] = j < classes ? Elem<T>::up(z[j]) : kNone<T>;  // all loads before the first use
    }
    if (ok) {
#pragma unroll
      for (int u = 0; u < R; ++u) {
        const int j = u * 32 + lane;
        const uint8_t in = j < classes ? ok[j] : 1;
        v[u] = in ? v[u] : kNone<T>;
      }
    }
    float zt = -INFINITY;
    if (t >= 0 && t < classes && (!ok || ok[t])) {
      const float x = Elem<T>::up(z[t]);
      if (!(x <= kNone<T>)) zt = x;
    }
    float m = kNone<T>;                                   // not a NaN
#pragma unroll
    for (int u = 0; u < R; ++u) {
      v[u] = max_nan(v[u], kNone<T>);
      m = fmaxf(m, v[u]);
    }
    m = from_ordered(__reduce_max_sync(~0u, ordered(m)));
    float S = 0.0f, A = 0.0f;
    // Distances that pass fp32's range are cut off at once where that is cheaper than a look at the sum:
    // 262144 rows of 16 49.6 us and 51.5, 65536 of 1000, 5 best, 128 and 139, none 54.6 and 53.9.
    constexpr bool cut = TOP || R <= 2;
    {
      constexpr int N = R < 4 ? R : 4;                    // sums side by side
      float s4[N], a4[N];
#pragma unroll
      for (int u = 0; u < R; ++u) {
        const float x = (v[u] - m) * c, d = cut ? max_nan(x, -200.0f) : x, e = exp2_fast(d);
        s4[u % N] = u < N ? e : s4[u % N] + e;
        a4[u % N] = u < N ? e * d : fmaf(e, d, a4[u % N]);
      }
#pragma unroll
      for (int u = 0; u < N; ++u) {
        S += s4[u];
        A += a4[u];
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      S += __shfl_xor_sync(~0u, S, o);
      A += __shfl_xor_sync(~0u, A, o);
    }
    if (!cut && A != A && S == S) {                       // as sum_again
      A = 0.0f;
#pragma unroll
      for (int u = 0; u < R; ++u) {
        const float d = fmaxf((v[u] - m) * c, -200.0f);
        A = fmaf(exp2_fast(d), d, A);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) A += __shfl_xor_sync(~0u, A, o);
    }
    const float log_s = log2f(S);
    const bool none = !(m > kNone<T>) && S == S;          // NaN stays
    const float lse = none ? -INFINITY : fmaf(m, a.inv_t, log_s * kLn2);
    if (lane == 0) {
      a.logp[row] = t >= classes ? NAN : t < 0 ? 0.0f : none ? -INFINITY : fmaf(zt - m, a.inv_t, -log_s * kLn2);
      a.entropy[row] = none ? 0.0f : (log_s - A / S) * kLn2;
      a.lse[row] = lse;
    }
    if (TOP) {
      // 0 for what is no candidate
      uint32_t most = 0, mine = 0, mine_index = 0;
      int at = 0;
      auto look = [&] {                                   // the lane's largest, the first of equal ones
        most = 0;
#pragma unroll
        for (int u = 0; u < R; ++u) {
          const uint32_t o = __float_as_uint(v[u]);
          if (o > most) {
            most = o;
            at = u;
          }
        }
      };
#pragma unroll
      for (int u = 0; u < R; ++u) v[u] = __uint_as_float(v[u] > kNone<T> ? ordered(v[u]) : 0u);
      look();
      bool has = false;
      for (int k = 0; k < a.top; ++k) {
        const uint32_t best = __reduce_max_sync(~0u, most);
        if (best == 0) break;
        const uint32_t index = __reduce_min_sync(~0u, most == best ? static_cast<uint32_t>(at * 32 + lane) : ~0u);
        if (lane == k) {
          has = true;
          mine = best;
          mine_index = index;
        }
        if (static_cast<int>(index & 31) == lane) {
#pragma unroll
          for (int u = 0; u < R; ++u)
            if (u == at) v[u] = 0.0f;
          look();
        }
      }
      if (lane < a.top) {
        has = has && !none && lse == lse;
        a.top_logp[row * a.top + lane] =
            has ? fmaf(from_ordered(mine) - m, a.inv_t, -log_s * kLn2) : (lse != lse ? NAN : -INFINITY);
        a.top_index[row * a.top + lane] = has ? static_cast<int>(mine_index) : -1;
      }
    }
  }
}

struct BwdArgs {
  const void* logits;
  const void* targets;
  const uint8_t* allowed;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* out;
  int64_t rows, classes, ld, allowed_ld, out_ld;
  float inv_t;
  bool wide_targets;
};

// d_j = (g (1[j = t] - p_j) - h p_j (log p_j + H)) / temperature, with p_j = e^(z_j - lse)
// read back from the forward's lse and entropy H; g and h are the gradients of logp and of
// the entropy.  With d = log2 p_j this is -p (h' d + k) plus g at the target.
template <bool ENT>
__device__ __forceinline__ float grad_of(float z, float inv_t, float lse, float h, float k) {
  const float d = fmaf(z, inv_t, -lse) * kLog2e;
  if constexpr (!ENT) return -exp2_fast(d) * k;
  const float f = max_nan(d, -200.0f);                   // minus infinity times 0
  return -exp2_fast(f) * fmaf(h, f, k);
}

constexpr int kBwdThreads = 256;
constexpr int kBwdUnroll = 4;

// A CTA takes kBwdThreads * kBwdUnroll vectors of a row.
template <typename T, bool ENT, bool MASK>
__global__ void __launch_bounds__(kBwdThreads) k_logprobs_backward(const __grid_constant__ BwdArgs a,
                                                                  int pieces) {
  constexpr int V = kVec<T>;
  const int64_t row = blockIdx.x / pieces;
  const int piece = static_cast<int>(blockIdx.x % pieces);
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  T* out = static_cast<T*>(a.out) + row * a.out_ld;
  const uint8_t* ok = MASK ? a.allowed + row * a.allowed_ld : nullptr;
  const int tid = threadIdx.x;
  const int classes = static_cast<int>(a.classes);
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int head = min(classes, shift ? V - shift : 0);
  const int vecs = (classes - head) / V;
  const int tail = head + vecs * V;
  const int base = piece * kBwdThreads * kBwdUnroll + tid;
  uint4 w[kBwdUnroll];
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int i = base + u * kBwdThreads;
    if (i < vecs) w[u] = __ldcs(reinterpret_cast<const uint4*>(z + head) + i);
  }

  const int64_t t64 = target_of(a.targets, a.wide_targets, row);
  const int t = t64 < 0 || t64 >= a.classes ? -1 : static_cast<int>(t64);
  const float lse0 = a.lse[row];
  const bool none = lse0 == -INFINITY;           // nothing allowed: no gradient
  const float lse = none ? INFINITY : lse0;      // every p is then 0
  const float g = t64 < 0 || none ? 0.0f : t64 >= a.classes ? NAN : a.dlogp[row] * a.inv_t;
  const float h0 = ENT && !none ? a.dentropy[row] * a.inv_t : 0.0f;
  const float h = h0 * kLn2;                     // d is in units of log 2
  const float k = ENT && !none ? fmaf(h0, a.entropy[row], g) : g;
  const bool wide_out = ((reinterpret_cast<uintptr_t>(out + head)) & 15) == 0;
  const int t_vec = t >= head && t < tail ? (t - head) / V : -1;

#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int i = base + u * kBwdThreads;
    if (i >= vecs) continue;
    const int at = head + i * V;
    float v[V];
    unpack<T>(w[u], v);
    uint32_t off = 0;                            // entries that are not allowed
    if (MASK) {
#pragma unroll
      for (int x = 0; x < V; ++x) off |= ok[at + x] ? 0u : 1u << x;
    }
    const float zt = i == t_vec ? Elem<T>::up(z[t]) : -INFINITY;
#pragma unroll
    for (int x = 0; x < V; ++x) {
      v[x] = grad_of<ENT>(v[x], a.inv_t, lse, h, k);
      if (MASK && (off >> x & 1u)) v[x] = 0.0f;
    }
    if (i == t_vec && zt > kNone<T> && !(MASK && !ok[t])) {
#pragma unroll
      for (int x = 0; x < V; ++x)
        if (at + x == t) v[x] += g;
    }
    if (wide_out) {
      uint4 o;
      if constexpr (sizeof(T) == 4)
        o = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      else
        o = make_uint4(narrow2<T>(v[0], v[1]), narrow2<T>(v[2], v[3]), narrow2<T>(v[4], v[5]), narrow2<T>(v[6], v[7]));
      __stcs(reinterpret_cast<uint4*>(out + at), o);
    } else {
#pragma unroll
      for (int x = 0; x < V; ++x) out[at + x] = Elem<T>::down(v[x]);
    }
  }
  if (piece == 0) {
    int i = -1;
    if (tid < head) i = tid;
    if (tid >= 32 && tail + tid - 32 < classes) i = tail + tid - 32;
    if (i >= 0) {
      const float z1 = Elem<T>::up(z[i]);
      const bool in = !MASK || ok[i];
      const float x = in ? grad_of<ENT>(z1, a.inv_t, lse, h, k) : 0.0f;
      out[i] = Elem<T>::down(in && i == t && z1 > kNone<T> ? x + g : x);
    }
  }
}

// The same for rows of few classes, a warp a row (8192 rows of 10, fp32: 3.1 us, 13 with a CTA a row;
// 8192 of 1000, bf16: 10.2 and 15.4; 100000 of 16: 17 and 130).
template <typename T, bool ENT>
__global__ void __launch_bounds__(kRowWarps * 32) k_logprobs_row_backward(const __grid_constant__ BwdArgs a) {
  const int lane = threadIdx.x & 31, classes = static_cast<int>(a.classes);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRowWarps;
  for (int64_t row = blockIdx.x * static_cast<int64_t>(kRowWarps) + (threadIdx.x >> 5); row < a.rows; row += step) {
    const T* z = static_cast<const T*>(a.logits) + row * a.ld;
    T* out = static_cast<T*>(a.out) + row * a.out_ld;
    const uint8_t* ok = a.allowed ? a.allowed + row * a.allowed_ld : nullptr;
    const int64_t t64 = target_of(a.targets, a.wide_targets, row);
    const int t = t64 < 0 || t64 >= classes ? -1 : static_cast<int>(t64);
    const float lse0 = a.lse[row];
    const bool none = lse0 == -INFINITY;
    const float lse = none ? INFINITY : lse0;
    const float g = t64 < 0 || none ? 0.0f : t64 >= classes ? NAN : a.dlogp[row] * a.inv_t;
    const float h0 = ENT && !none ? a.dentropy[row] * a.inv_t : 0.0f;
    const float h = h0 * kLn2, k = ENT && !none ? fmaf(h0, a.entropy[row], g) : g;
    for (int j0 = lane; j0 < classes; j0 += 32 * kRowUnroll) {
      T x[kRowUnroll];
      uint32_t in = ~0u;                                  // entries that are allowed
#pragma unroll
      for (int u = 0; u < kRowUnroll; ++u)
        if (j0 + u * 32 < classes) x[u] = z[j0 + u * 32];
      if (ok) {
#pragma unroll
        for (int u = 0; u < kRowUnroll; ++u)
          if (j0 + u * 32 < classes && !ok[j0 + u * 32]) in &= ~(1u << u);
      }
#pragma unroll
      for (int u = 0; u < kRowUnroll; ++u) {
        const int j = j0 + u * 32;
        if (j >= classes) break;
        const float f = Elem<T>::up(x[u]);
        float d = grad_of<ENT>(f, a.inv_t, lse, h, k);
        if (j == t && f > kNone<T>) d += g;
        out[j] = Elem<T>::down(in >> u & 1u ? d : 0.0f);
      }
    }
  }
}

// CTAs a row: enough that all rows fill the GPU twice (152 SMs), as long as each keeps
// half a round of loads.
int cluster_size(int64_t rows, int64_t bytes) {
  int parts = 1;
  while (parts < kMaxCluster && rows * parts < 304 && bytes / (2 * parts) >= 512 * kUnroll * 8) parts *= 2;
  return parts;
}

template <typename T, bool TOP, bool MASK, int THREADS>
cudaError_t launch_forward(const FwdArgs& a, int parts, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows * parts));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = TOP ? sizeof(TopState) : 0;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_logprobs<T, TOP, MASK, THREADS>, a);
}

// Few CTAs take 512 threads each; where they fill the GPU, half the threads have half the
// cost of a row's end and overlap it with other CTAs' loads (8192 rows of 32768 bf16: 104 us with
// 512 threads, 85 us with 256).
template <typename T, bool TOP, bool MASK>
cudaError_t forward_rows(const FwdArgs& a, cudaStream_t s) {
  const int parts = cluster_size(a.rows, a.classes * static_cast<int64_t>(sizeof(T)));
  return parts * a.rows < 152 ? launch_forward<T, TOP, MASK, 512>(a, parts, s)
                                   : launch_forward<T, TOP, MASK, 256>(a, parts, s);
}

// Rows of at most this many classes take a warp; beyond kShortRow of them the likeliest and the
// gradient take a CTA unless the rows' warps fill the GPU: one warp's chain of steps is longer
// (300 rows of 2048, 20 best: 14.7 us by warps, 6.9 by CTAs; 8192 rows, 8 best: 53 and 79; the
// gradient of one row of 1000: 3.6 and 2.1, of 8192 rows 9.9 and 15.4).
constexpr int kRowClasses = 2048, kShortRow = 512;
bool fills(int64_t rows) { return rows >= 152 * kRowWarps; }
unsigned row_grid(int64_t rows) { return static_cast<unsigned>(std::min<int64_t>((rows + kRowWarps - 1) / kRowWarps, 152 * 8)); }

template <typename T, bool TOP>
cudaError_t forward_few(const FwdArgs& a, cudaStream_t s) {
  const auto kernel = a.classes <= 64    ? k_logprobs_row<T, TOP, 2>
                      : a.classes <= 512 ? k_logprobs_row<T, TOP, 16>
                      : a.classes <= 1024 ? k_logprobs_row<T, TOP, 32>
                                         : k_logprobs_row<T, TOP, kRowClasses / 32>;
  kernel<<<row_grid(a.rows), kRowWarps * 32, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t forward_type(const FwdArgs& a, cudaStream_t s) {
  if (a.classes <= kRowClasses && (!a.top || a.classes <= kShortRow || fills(a.rows)))
    return a.top ? forward_few<T, true>(a, s) : forward_few<T, false>(a, s);
  if (a.top) return a.allowed ? forward_rows<T, true, true>(a, s) : forward_rows<T, true, false>(a, s);
  return a.allowed ? forward_rows<T, false, true>(a, s) : forward_rows<T, false, false>(a, s);
}

template <typename T, bool ENT, bool MASK>
cudaError_t launch_backward(const BwdArgs& a, cudaStream_t s) {
  const int64_t per = static_cast<int64_t>(kBwdThreads) * kBwdUnroll * kVec<T>;
  const int64_t pieces = (a.classes + per - 1) / per;
  if (a.rows * pieces > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
  k_logprobs_backward<T, ENT, MASK>
      <<<static_cast<unsigned>(a.rows * pieces), kBwdThreads, 0, s>>>(a, static_cast<int>(pieces));
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward_type(const BwdArgs& a, cudaStream_t s) {
  if (a.classes <= kShortRow || (a.classes <= kRowClasses / 2 && fills(a.rows))) {
    const auto kernel = a.dentropy ? k_logprobs_row_backward<T, true> : k_logprobs_row_backward<T, false>;
    kernel<<<row_grid(a.rows), kRowWarps * 32, 0, s>>>(a);
    return cudaGetLastError();
  }
  if (a.dentropy)
    return a.allowed ? launch_backward<T, true, true>(a, s) : launch_backward<T, true, false>(a, s);
  return a.allowed ? launch_backward<T, false, true>(a, s) : launch_backward<T, false, false>(a, s);
}

// Below 2^-126 the temperature's inverse is infinite; above, a class that is raised to kNone would be
// so close to the others that it had a probability.
constexpr float kMaxTemperature = 1e27f;
bool shape_ok(int type, int64_t rows, int64_t classes, int64_t ld, const void* logits,
              const void* targets, int target_bytes, int64_t allowed_ld, float temperature) {
  return type_ok(type) && rows >= 0 && classes >= 1 && classes <= 0x7FFFFFFF && ld >= classes &&
         (target_bytes == 4 || target_bytes == 8) && (allowed_ld == 0 || allowed_ld >= classes) &&
         temperature >= FLT_MIN && temperature <= kMaxTemperature && (rows == 0 || (logits && targets)) &&
         reinterpret_cast<uintptr_t>(logits) % type_size(type) == 0;
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_token_logprobs(const void* logits_dev, int type, int64_t rows,
                                       int64_t classes, int64_t ld, const void* targets_dev,
                                       int target_bytes, const uint8_t* allowed_dev,
                                       int64_t allowed_ld, float temperature, int top,
                                       float* logp_dev, float* entropy_dev, float* lse_dev,
                                       float* top_logp_dev, int32_t* top_index_dev, void* stream) {
  if (!shape_ok(type, rows, classes, ld, logits_dev, targets_dev, target_bytes, allowed_ld, temperature))
    return HA_EINVAL;
  if (top < 0 || (top > 0 && rows > 0 && (!top_logp_dev || !top_index_dev))) return HA_EINVAL;
  if (top > kMaxTop || rows > 0x7FFFFFFF / kMaxCluster) return HA_EUNSUPPORTED;
  if (rows == 0) return HA_OK;
  if (!logp_dev || !entropy_dev || !lse_dev) return HA_EINVAL;
  FwdArgs a = {logits_dev, targets_dev, allowed_dev, rows, classes, ld, allowed_ld,
               1.0f / temperature, top, target_bytes == 8, logp_dev, entropy_dev, lse_dev,
               top_logp_dev, top_index_dev};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = type == HA_TYPE_FP32   ? forward_type<float>(a, s)
                        : type == HA_TYPE_BF16 ? forward_type<__nv_bfloat16>(a, s)
                                               : forward_type<__half>(a, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}

extern "C" int hier_avg_token_logprobs_backward(
    const void* logits_dev, int type, int64_t rows, int64_t classes, int64_t ld,
    const void* targets_dev, int target_bytes, const uint8_t* allowed_dev, int64_t allowed_ld,
    float temperature, const float* lse_dev, const float* entropy_dev, const float* dlogp_dev,
    const float* dentropy_dev, void* dlogits_dev, int64_t dlogits_ld, void* stream) {
  if (!shape_ok(type, rows, classes, ld, logits_dev, targets_dev, target_bytes, allowed_ld, temperature))
    return HA_EINVAL;
  if (dlogits_ld < classes || reinterpret_cast<uintptr_t>(dlogits_dev) % type_size(type)) return HA_EINVAL;
  if (rows == 0) return HA_OK;
  if (!lse_dev || !dlogp_dev || !dlogits_dev || (dentropy_dev && !entropy_dev)) return HA_EINVAL;
  BwdArgs a = {logits_dev, targets_dev, allowed_dev, lse_dev, entropy_dev, dlogp_dev, dentropy_dev,
               dlogits_dev, rows, classes, ld, allowed_ld, dlogits_ld, 1.0f / temperature,
               target_bytes == 8};
  const int64_t per = static_cast<int64_t>(kBwdThreads) * kBwdUnroll * 4;
  if (rows > 0x7FFFFFFF / ((classes + per - 1) / per)) return HA_EUNSUPPORTED;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = type == HA_TYPE_FP32   ? backward_type<float>(a, s)
                        : type == HA_TYPE_BF16 ? backward_type<__nv_bfloat16>(a, s)
                                               : backward_type<__half>(a, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}
