// Log probabilities of given tokens, with the entropy and the likeliest alternatives, and
// the gradient with respect to the logits.
//
// For a row z_j = logits_j / temperature over the allowed j, with m the running maximum:
//   S = sum e^(z_j - m),  A = sum (z_j - m) e^(z_j - m)
//   lse = m + log S,  logp = z_t - lse,  entropy = log S - A / S
// in one pass: each thread keeps its own (m, S, A) and rescales the sums when m grows; the
// partial sums of threads and CTAs join by the same rule.  Sums are in units of log 2, since
// the hardware's exponential is 2^x.
#include <cmath>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kThreads = 512;
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
// Where m starts.  A logit at or below it adds nothing, so a mask written with the lowest
// finite value of bf16 or fp32 works as one of minus infinity does, and m stays finite.
constexpr float kNone = -1e30f;

// The sums of `b` added to those of `a`; c = log2(e) / temperature.
__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float da = max_nan((a.m - r.m) * c, -200.0f), db = max_nan((b.m - r.m) * c, -200.0f);
  const float ea = exp2_fast(da), eb = exp2_fast(db);
  r.S = a.S * ea + b.S * eb;
  r.A = (a.A + a.S * da) * ea + (b.A + b.S * db) * eb;
  return r;
}

// Keys order by value, equal values by lower index.
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
  const uint32_t u = __float_as_uint(v);
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (static_cast<uint64_t>(o) << 32) | static_cast<uint32_t>(~index);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
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
  int count;
  uint64_t bar;       // keys below it are not among the best
};

// Descending bitonic sort of s.keys[0, n), n a power of two, by the whole CTA.
__device__ void sort_keys(uint64_t* keys, int n) {
  for (int k = 2; k <= n; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < n / 2; i += kThreads) {
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

// Sorts the candidates and keeps the best `top`; the bar rises to the last of them.
__device__ void cut(TopState& s, int top) {
  __syncthreads();
  const int count = min(s.count, kCap);
  int n = 64;
  while (n < count) n <<= 1;
  for (int i = count + threadIdx.x; i < n; i += kThreads) s.keys[i] = 0;
  sort_keys(s.keys, n);
  if (threadIdx.x == 0) {
    s.count = min(count, top);
    if (count >= top) s.bar = s.keys[top - 1];
  }
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

// Entries that are not allowed become minus infinity.
template <int N>
__device__ __forceinline__ void apply_mask(float* v, const uint8_t* a) {
  uint32_t w[2];
  if ((reinterpret_cast<uintptr_t>(a) & (N - 1)) == 0) {
    if constexpr (N == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(a);
      w[0] = x.x; w[1] = x.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(a);
    }
  } else {
#pragma unroll
    for (int h = 0; h < N / 4; ++h)
      w[h] = a[4 * h] | (a[4 * h + 1] << 8) | (a[4 * h + 2] << 16) | (a[4 * h + 3] << 24);
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (((w[i >> 2] >> (8 * (i & 3))) & 0xFFu) == 0) v[i] = -INFINITY;
}

template <int N>
__device__ __forceinline__ void add_stat(Stat& s, const float* v, float c) {
  float top = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
  if (top > s.m) {
    const float d = max_nan((s.m - top) * c, -200.0f), e = exp2_fast(d);
    s.A = (s.A + s.S * d) * e;
    s.S *= e;
    s.m = top;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // minus infinity gives 2^-200 = 0; NaN stays
    const float d = max_nan((v[i] - s.m) * c, -200.0f), e = exp2_fast(d);
    s.S += e;
    s.A = fmaf(e, d, s.A);
  }
}

__device__ __forceinline__ int64_t target_of(const void* targets, bool wide, int64_t row) {
  return wide ? static_cast<const int64_t*>(targets)[row] : static_cast<const int*>(targets)[row];
}

// One cluster a row; its CTAs take equal shares of the row's 16-byte vectors.
template <typename T, bool TOP, bool MASK>
__global__ void __launch_bounds__(kThreads, TOP ? 2 : 3) k_logprobs(const FwdArgs a) {
  constexpr int V = kVec<T>;
  __shared__ Stat warp_stat[kThreads / 32];
  __shared__ Stat cta_stat;
  extern __shared__ __align__(16) unsigned char dyn[];
  TopState& ts = *reinterpret_cast<TopState*>(dyn);

  uint32_t rank, parts;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  const int64_t row = blockIdx.x / parts;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const uint8_t* ok = MASK ? a.allowed + row * a.allowed_ld : nullptr;
  const int tid = threadIdx.x;
  const float c = a.inv_t * kLog2e;

  // The vectors start at the row's first 16-byte boundary; the entries before and after
  // them are taken one by one, by the first and the last CTA.
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int64_t head = min(a.classes, static_cast<int64_t>(shift ? V - shift : 0));
  const int64_t vecs = (a.classes - head) / V;
  const int64_t v0 = vecs * rank / parts, v1 = vecs * (rank + 1) / parts;
  const int64_t tail = head + vecs * V;

  Stat s = {kNone, 0.0f, 0.0f};
  if (TOP) {
    if (tid == 0) {
      ts.count = 0;
      ts.bar = 0;
    }
    __syncthreads();
  }

  const int64_t rounds = (v1 - v0 + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  for (int64_t r = 0; r <= rounds; ++r) {
    // round 0 .. rounds-1: vectors; the last: the single entries at the row's ends
    float v[kUnroll][V];
    int64_t at[kUnroll];
    if (r < rounds) {
      uint4 w[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t i = v0 + (r * kUnroll + u) * kThreads + tid;
        at[u] = i < v1 ? head + i * V : -1;
        if (i < v1) w[u] = __ldcs(reinterpret_cast<const uint4*>(z + at[u]));
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (at[u] < 0) {
#pragma unroll
          for (int i = 0; i < V; ++i) v[u][i] = -INFINITY;
          continue;
        }
        unpack<T>(w[u], v[u]);
        if (MASK) apply_mask<V>(v[u], ok + at[u]);
        add_stat<V>(s, v[u], c);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        at[u] = -1;
#pragma unroll
        for (int i = 0; i < V; ++i) v[u][i] = -INFINITY;
      }
      int64_t i = -1;
      if (rank == 0 && tid < head) i = tid;
      if (rank == parts - 1 && tid >= 32 && tail + tid - 32 < a.classes) i = tail + tid - 32;
      if (i >= 0 && (!MASK || ok[i])) {
        at[0] = i;
        v[0][0] = Elem<T>::up(z[i]);
        add_stat<1>(s, v[0], c);
      }
    }
    if (TOP) {
      float most = -INFINITY;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) most = fmaxf(most, v[u][i]);
      if (r == 0 && rounds > 0) {
        // The best `top` of the threads' largest entries bound the best of all from below.
        uint64_t k = 0;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
          for (int i = V - 1; i >= 0; --i)
            if (v[u][i] == most && most > kNone) {
              const uint64_t n = key_of(most, static_cast<uint32_t>(at[u] + i));
              k = n > k ? n : k;
            }
        if (k) ts.keys[atomicAdd(&ts.count, 1)] = k;
        cut(ts, a.top);
        if (tid == 0) ts.count = 0;
        __syncthreads();
      }
      // Entries over the bar become candidates.  What does not fit waits until the
      // candidates have been cut to the best and the bar raised.
      bool waiting = true;
      uint32_t done[kUnroll] = {};
      while (true) {
        const uint64_t bar = ts.bar;
        const float low = key_value(bar);
        if (waiting) {
          waiting = false;
          if (!(most < low) || bar == 0) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
#pragma unroll
              for (int i = 0; i < V; ++i) {
                if (!(v[u][i] > kNone) || (done[u] >> i & 1)) continue;
                const uint64_t k = key_of(v[u][i], static_cast<uint32_t>(at[u] + i));
                if (k >= bar) {
                  const int place = atomicAdd(&ts.count, 1);
                  if (place < kCap) {
                    ts.keys[place] = k;
                    done[u] |= 1u << i;
                  } else {
                    waiting = true;
                  }
                }
              }
          }
        }
        if (!__syncthreads_or(waiting)) break;
        cut(ts, a.top);
      }
    }
  }

  // Threads, warps and CTAs of the row join their sums.
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Stat b = {__shfl_xor_sync(~0u, s.m, o), __shfl_xor_sync(~0u, s.S, o), __shfl_xor_sync(~0u, s.A, o)};
    s = join(s, b, c);
  }
  if ((tid & 31) == 0) warp_stat[tid >> 5] = s;
  if (TOP) cut(ts, a.top);
  __syncthreads();
  if (tid < 32) {
    s = tid < kThreads / 32 ? warp_stat[tid] : Stat{kNone, 0.0f, 0.0f};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Stat b = {__shfl_xor_sync(~0u, s.m, o), __shfl_xor_sync(~0u, s.S, o), __shfl_xor_sync(~0u, s.A, o)};
      s = join(s, b, c);
    }
    if (tid == 0) cta_stat = s;
  }
  if (parts > 1) {
    cluster_barrier();
    if (rank == 0) {
      s = cta_stat;
      for (uint32_t q = 1; q < parts; ++q)
        s = join(s, {from_cta(&cta_stat.m, q), from_cta(&cta_stat.S, q), from_cta(&cta_stat.A, q)}, c);
      if (TOP) {
        // the other CTAs' best after this one's
        for (int i = tid; i < static_cast<int>(parts - 1) * kMaxTop; i += kThreads) {
          const int q = 1 + i / kMaxTop, k = i % kMaxTop;
          if (k < from_cta(&ts.count, q)) ts.keys[atomicAdd(&ts.count, 1)] = from_cta(&ts.keys[k], q);
        }
        cut(ts, a.top);
      }
    }
    cluster_barrier();
    if (rank != 0) return;
  } else {
    __syncthreads();
    s = cta_stat;
  }

  const float log_s = log2f(s.S);
  const bool none = s.S == 0.0f;
  const float lse = none ? -INFINITY : fmaf(s.m, a.inv_t, log_s * kLn2);
  if (tid == 0) {
    const int64_t t = target_of(a.targets, a.wide_targets, row);
    float lp = 0.0f;
    if (t >= a.classes) {
      lp = NAN;
    } else if (t >= 0) {
      float zt = Elem<T>::up(z[t]);
      if (zt <= kNone || (MASK && !ok[t])) zt = -INFINITY;
      lp = none ? -INFINITY : ((zt - s.m) * c - log_s) * kLn2;
    }
    a.logp[row] = lp;
    a.entropy[row] = none ? 0.0f : (log_s - s.A / s.S) * kLn2;
    a.lse[row] = lse;
  }
  if (TOP && tid < a.top) {
    const bool bad = !(fabsf(lse) < INFINITY);
    const bool has = tid < ts.count && !bad;
    const uint64_t k = has ? ts.keys[tid] : 0;
    a.top_logp[row * a.top + tid] =
        has ? ((key_value(k) - s.m) * c - log_s) * kLn2 : (lse != lse ? NAN : -INFINITY);
    a.top_index[row * a.top + tid] = has ? static_cast<int>(key_index(k)) : -1;
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
// the entropy.  p (log p + H) is taken as 0 where p is.
template <typename T, bool ENT>
__device__ __forceinline__ float grad_of(float z, float inv_t, float lse, float g, float h, float ent2) {
  const float d = max_nan(fmaf(z, inv_t, -lse) * kLog2e, -200.0f), p = exp2_fast(d);
  return ENT ? -p * fmaf(h, d + ent2, g) : -p * g;
}

constexpr int kBwdThreads = 256;
constexpr int kBwdUnroll = 4;

// grid.x: pieces of kBwdThreads * kBwdUnroll vectors of a row; grid.y: rows (strided).
template <typename T, bool ENT, bool MASK>
__global__ void __launch_bounds__(kBwdThreads) k_logprobs_backward(const BwdArgs a, int pieces) {
  constexpr int V = kVec<T>;
  const int64_t row = blockIdx.x / pieces;
  const int piece = static_cast<int>(blockIdx.x % pieces);
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  T* out = static_cast<T*>(a.out) + row * a.out_ld;
  const uint8_t* ok = MASK ? a.allowed + row * a.allowed_ld : nullptr;
  const int tid = threadIdx.x;
  const int64_t t = target_of(a.targets, a.wide_targets, row);
  const float lse = a.lse[row];
  const bool none = lse == -INFINITY;            // nothing allowed: no gradient
  const float g0 = t < 0 || none ? 0.0f : a.dlogp[row];
  const float g = g0 * a.inv_t;
  // d is in units of log 2
  const float h = ENT && !none ? a.dentropy[row] * a.inv_t * kLn2 : 0.0f;
  const float ent2 = ENT && !none ? a.entropy[row] * kLog2e : 0.0f;

  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int64_t head = min(a.classes, static_cast<int64_t>(shift ? V - shift : 0));
  const int64_t vecs = (a.classes - head) / V;
  const int64_t tail = head + vecs * V;
  const bool wide_out = ((reinterpret_cast<uintptr_t>(out + head)) & 15) == 0;

  const int64_t base = static_cast<int64_t>(piece) * kBwdThreads * kBwdUnroll;
  uint4 w[kBwdUnroll];
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int64_t i = base + u * kBwdThreads + tid;
    if (i < vecs) w[u] = __ldcs(reinterpret_cast<const uint4*>(z + head + i * V));
  }
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int64_t i = base + u * kBwdThreads + tid;
    if (i >= vecs) continue;
    float v[V];
    unpack<T>(w[u], v);
    const int64_t at = head + i * V;
    if (MASK) apply_mask<V>(v, ok + at);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float x = none ? 0.0f : grad_of<T, ENT>(v[k], a.inv_t, lse, g, h, ent2);
      v[k] = at + k == t && v[k] > kNone ? x + g : x;
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
      for (int k = 0; k < V; ++k) out[at + k] = Elem<T>::down(v[k]);
    }
  }
  if (piece == 0) {
    int64_t i = -1;
    if (tid < head) i = tid;
    if (tid >= 32 && tail + tid - 32 < a.classes) i = tail + tid - 32;
    if (i >= 0) {
      const float z1 = MASK && !ok[i] ? -INFINITY : Elem<T>::up(z[i]);
      const float x = none ? 0.0f : grad_of<T, ENT>(z1, a.inv_t, lse, g, h, ent2);
      out[i] = Elem<T>::down(i == t && z1 > kNone ? x + g : x);
    }
  }
}

// CTAs a row: enough that all rows fill the GPU twice (152 SMs), as long as each keeps
// at least two rounds of loads.
int cluster_size(int64_t rows, int64_t bytes) {
  int parts = 1;
  while (parts < kMaxCluster && rows * parts < 304 && bytes / (2 * parts) >= kThreads * 16) parts *= 2;
  return parts;
}

template <typename T, bool TOP, bool MASK>
cudaError_t launch_forward(const FwdArgs& a, cudaStream_t s) {
  const int parts = cluster_size(a.rows, a.classes * static_cast<int64_t>(sizeof(T)));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows * parts));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = TOP ? sizeof(TopState) : 0;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_logprobs<T, TOP, MASK>, a);
}

template <typename T>
cudaError_t forward_type(const FwdArgs& a, cudaStream_t s) {
  if (a.top)
    return a.allowed ? launch_forward<T, true, true>(a, s) : launch_forward<T, true, false>(a, s);
  return a.allowed ? launch_forward<T, false, true>(a, s) : launch_forward<T, false, false>(a, s);
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
  if (a.dentropy)
    return a.allowed ? launch_backward<T, true, true>(a, s) : launch_backward<T, true, false>(a, s);
  return a.allowed ? launch_backward<T, false, true>(a, s) : launch_backward<T, false, false>(a, s);
}

bool shape_ok(int type, int64_t rows, int64_t classes, int64_t ld, const void* logits,
              const void* targets, int target_bytes, int64_t allowed_ld, float temperature) {
  return type_ok(type) && rows >= 0 && classes >= 1 && classes <= 0x7FFFFFFF && ld >= classes &&
         (target_bytes == 4 || target_bytes == 8) && (allowed_ld == 0 || allowed_ld >= classes) &&
         temperature > 0 && std::isfinite(temperature) && (rows == 0 || (logits && targets)) &&
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
