// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Row i of a sequence has p_i = softmax(logits_i / temperature) over the allowed classes and, for i < K, the
// draft x_i, which was drawn from q_i (without draft probabilities q is 1 at x_i).  With uniform numbers u:
//   draft i is accepted while u_i q_i(x_i) < p_i(x_i);  n is the first that is not, or the first row without a draft;
//   the next token is argmax_j r_j / noise_j with r = max(p_n - q_n, 0) after a rejection (p_n where that
//   leaves nothing), else r = p_n.  With exponential noise that is a draw from r.
//
// Two kernels: one takes every row's largest logit and the sum of its exponentials, and says whether its draft
// would be accepted; the other finds n and looks for the next token.  A row is shared by the CTAs of a cluster.
// Sums and scores are in fp32, with a bound of what that may be off; a decision within the bound is made
// again by one CTA in 64 bits, so that the tokens are those of the formulas in 64 bits.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kMaxCluster = 8;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kUnroll = 4;

// The relative error of a probability e^((z - m) / t) / S with d = (z - m) log2(e) / t, in steps of 2^-22: d takes
// three roundings of 2^-24 of itself each (times ln 2: |d| / 2), 2^d one step, S the same for a mean |d| that is at most
// log2 of the classes, 31, and a quarter step for each addition of a sum's chain.
float slack(int classes, int elements_a_load) { return 20.0f + (classes / (kThreads * elements_a_load) + 16) * 0.25f; }
__device__ __forceinline__ float bound(float d, float slack) { return 0x1p-22f * (slack + fabsf(d)); }

struct Row {                              // of the workspace
  float m, S;                             // largest logit; sum of e^((z - m) / t), 0: no class, NaN: a bad row
  float logp;                             // of the draft
  int accepted;
};

struct VerifyArgs {
  const void* logits;
  int64_t z_seq, z_row;
  const void* drafts;
  const float* uniform;
  const float* noise;
  int64_t noise_ld;
  const void* probs;
  int64_t q_seq, q_row;
  const uint8_t* allowed;
  int64_t ok_seq, ok_row;
  int *tokens, *accepted;
  float* logp;
  Row* rows;
  double temperature;
  float c;                                // log2(e) / temperature
  float inv_t;
  float slack;                            // of bound()
  int K, classes;
  bool wide_drafts;
  int probs_type;                         // -1: none
};

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_parts() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// The same place of shared memory in CTA `rank` of the cluster.
template <typename V>
__device__ __forceinline__ V from_cta(const V* p, int rank) {
  static_assert(sizeof(V) == 4, "a word");
  const uint32_t la = static_cast<uint32_t>(__cvta_generic_to_shared(p));
  uint32_t ra, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(la), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(ra) : "memory");
  return *reinterpret_cast<V*>(&v);
}

__device__ __forceinline__ int64_t draft_of(const VerifyArgs& a, int64_t seq, int i) {
  const int64_t e = seq * a.K + i;
  return a.wide_drafts ? static_cast<const int64_t*>(a.drafts)[e] : static_cast<const int*>(a.drafts)[e];
}
__device__ __forceinline__ float prob_at(const VerifyArgs& a, int64_t e) {
  if (a.probs_type == HA_TYPE_FP32) return static_cast<const float*>(a.probs)[e];
  if (a.probs_type == HA_TYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(a.probs)[e]);
  return __half2float(static_cast<const __half*>(a.probs)[e]);
}

// A row's logit, kNone where the class is not allowed.
template <typename T>
__device__ __forceinline__ float logit(const T* z, const uint8_t* ok, int j) {
  const float v = max_nan(Elem<T>::up(z[j]), kNone<T>);
  return ok && !ok[j] ? kNone<T> : v;
}

struct Sum {
  float m, S;
};
__device__ __forceinline__ Sum join(Sum s, float c) {
  const float m = from_ordered(__reduce_max_sync(~0u, ordered(s.m)));
  Sum r = {m, s.S * exp2_fast(max_nan((s.m - m) * c, -200.0f))};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.S += __shfl_xor_sync(~0u, r.S, o);
  return r;
}

// log of the sum of e^(z / t), in 64 bits, by one CTA; every thread has it.
template <typename T>
__device__ __noinline__ double exact_lse(const VerifyArgs& a, const T* z, const uint8_t* ok, float m, double* part) {
  const double top = static_cast<double>(m) / a.temperature;
  double s = 0.0;
  for (int j = threadIdx.x; j < a.classes; j += kThreads) {
    const float v = logit(z, ok, j);
    if (v > kNone<T>) s += exp(static_cast<double>(v) / a.temperature - top);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < kWarps; ++w) s += part[w];
  return top + log(s);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_verify_rows(const __grid_constant__ VerifyArgs a) {
  __shared__ Sum warp_sum[kWarps];
  __shared__ Sum cta_sum, row_sum;
  __shared__ double part[kWarps];
  __shared__ bool unsure;
  constexpr int V = kVec<T>;
  const uint32_t rank = cluster_rank(), parts = cluster_parts();
  const int64_t row = blockIdx.x / parts, seq = row / (a.K + 1);
  const int i = static_cast<int>(row % (a.K + 1)), tid = threadIdx.x, lane = tid & 31;
  const T* z = static_cast<const T*>(a.logits) + seq * a.z_seq + i * a.z_row;
  const uint8_t* ok = a.allowed ? a.allowed + seq * a.ok_seq + i * a.ok_row : nullptr;
  const float c = a.c;
  let_next_start();

  // The vectors start at the row's first 16-byte boundary; the entries before and after them are taken one by one.
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T));
  const int head = min(a.classes, shift ? V - shift : 0), vecs = (a.classes - head) / V, tail = head + vecs * V;
  const int v0 = static_cast<int>(static_cast<int64_t>(vecs) * rank / parts);
  const int v1 = static_cast<int>(static_cast<int64_t>(vecs) * (rank + 1) / parts);
  Sum s = {kNone<T>, 0.0f};
  int one = -1;
  if (rank == 0 && tid < head) one = tid;
  if (rank == parts - 1 && tid >= 32 && tail + tid - 32 < a.classes) one = tail + tid - 32;
  if (one >= 0) {
    s.m = logit(z, ok, one);
    s.S = s.m > kNone<T> ? 1.0f : s.m == s.m ? 0.0f : s.m;
    if (s.m != s.m) s.m = kNone<T>;
  }
  for (int r = v0 + tid; r < v1; r += kThreads * kUnroll) {
    uint4 w[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (r + u * kThreads < v1) w[u] = __ldg(reinterpret_cast<const uint4*>(z + head) + r + u * kThreads);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (r + u * kThreads >= v1) break;
      float v[V];
      unpack<T>(w[u], v);
      const int at = head + (r + u * kThreads) * V;
      float top = s.m;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[e] = max_nan(v[e], kNone<T>);
        if (ok && !ok[at + e]) v[e] = kNone<T>;
        top = fmaxf(top, v[e]);
      }
      if (top > s.m) {
        s.S *= exp2_fast(max_nan((s.m - top) * c, -200.0f));
        s.m = top;
      }
      // what is not allowed adds 0: the largest is above it, or all are not
      if (s.m > kNone<T>) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = exp2_fast((v[e] - s.m) * c);
#pragma unroll
        for (int o = V / 2; o > 0; o >>= 1) {
#pragma unroll
          for (int e = 0; e < o; ++e) v[e] += v[e + o];
        }
        s.S += v[0];
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (v[e] != v[e]) s.S = v[e];
      }
    }
  }
  s = join(s, c);
  if (lane == 0) warp_sum[tid >> 5] = s;
  __syncthreads();
  if (tid < 32) {
    s = join(tid < kWarps ? warp_sum[tid] : Sum{kNone<T>, 0.0f}, c);
    if (tid == 0) cta_sum = s;
  }
  if (parts > 1) {
    cluster_barrier();
    if (rank == 0 && tid < 32) {
      s = {kNone<T>, 0.0f};
      if (tid < static_cast<int>(parts)) s = {from_cta(&cta_sum.m, tid), from_cta(&cta_sum.S, tid)};
      s = join(s, c);
    }
    cluster_barrier();
    if (rank != 0) return;
  }
  if (tid == 0) {
    const int64_t x = i < a.K ? draft_of(a, seq, i) : -1;
    Row out = {s.m, s.S, 0.0f, 0};
    unsure = false;
    if (x >= 0 && x < a.classes && s.S > 0.0f) {            // not where there is no class, or a NaN
      const float zx = logit(z, ok, static_cast<int>(x)), d = (zx - s.m) * c;
      const double q = a.probs ? static_cast<double>(prob_at(a, seq * a.q_seq + i * a.q_row + x)) : 1.0;
      const double left = static_cast<double>(a.uniform[seq * a.K + i]) * q;
      if (zx > kNone<T>) {
        const double p = static_cast<double>(exp2_fast(d)) / s.S, off = bound(d, a.slack) * p;
        out.accepted = left < p;
        unsure = fabs(left - p) <= off || (p < 1e-30 && left < 1e-30);
        out.logp = fmaf(zx - s.m, a.inv_t, -logf(s.S));
      }
    }
    a.rows[row] = out;
    row_sum = s;
  }
  __syncthreads();
  if (!unsure) return;
  const double lse = exact_lse(a, z, ok, row_sum.m, part);
  if (tid == 0) {
    const int64_t x = draft_of(a, seq, i);
    const double q = a.probs ? static_cast<double>(prob_at(a, seq * a.q_seq + i * a.q_row + x)) : 1.0;
    const double p = exp(static_cast<double>(logit(z, ok, static_cast<int>(x))) / a.temperature - lse);
    a.rows[row].accepted = static_cast<double>(a.uniform[seq * a.K + i]) * q < p;
  }
}

// The best class so far: its score, what that may be off, and the most that any other's may be.
struct Best {
  float score, off, others;
  int index;
};
__device__ __forceinline__ Best better(const Best& a, const Best& b) {
  const bool first = a.score > b.score || (a.score == b.score && static_cast<uint32_t>(a.index) < static_cast<uint32_t>(b.index));
  const Best &w = first ? a : b, &l = first ? b : a;
  return {w.score, w.off, fmaxf(fmaxf(a.others, b.others), l.index < 0 ? 0.0f : l.score + l.off), w.index};
}
__device__ __forceinline__ Best warp_best(Best b) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Best x = {__shfl_xor_sync(~0u, b.score, o), __shfl_xor_sync(~0u, b.off, o), __shfl_xor_sync(~0u, b.others, o),
                    __shfl_xor_sync(~0u, b.index, o)};
    b = better(b, x);
  }
  return b;
}

__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The next token in 64 bits, by one CTA.
template <typename T>
__device__ __noinline__ int exact_token(const VerifyArgs& a, const T* z, const uint8_t* ok, const float* noise, float m,
                                        int64_t q0, int x, bool rejected, double* part, int* part_index) {
  const double lse = exact_lse(a, z, ok, m, part);
  int best = -1;
  for (int pass = rejected ? 0 : 1; pass < 2 && best < 0; ++pass) {
    double score = -1.0;
    bool any = false;
    best = -1;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) {
      const float v = logit(z, ok, j);
      if (!(v > kNone<T>)) continue;
      double r = exp(static_cast<double>(v) / a.temperature - lse);
      if (pass == 0) r = a.probs ? fmax(r - static_cast<double>(prob_at(a, q0 + j)), 0.0) : j == x ? 0.0 : r;
      const double s = r / static_cast<double>(noise[j]);
      any = any || r > 0.0;
      if (r > 0.0 && s >= 0.0 && s > score) {
        score = s;
        best = j;
      }
    }
    const int some = __syncthreads_or(any);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double s = __shfl_xor_sync(~0u, score, o);
      const int j = __shfl_xor_sync(~0u, best, o);
      if (s > score || (s == score && static_cast<uint32_t>(j) < static_cast<uint32_t>(best))) {
        score = s;
        best = j;
      }
    }
    if ((threadIdx.x & 31) == 0) {
      part[threadIdx.x >> 5] = score;
      part_index[threadIdx.x >> 5] = best;
    }
    __syncthreads();
    score = -1.0;
    best = -1;
    for (int w = 0; w < kWarps; ++w)
      if (part[w] > score || (part[w] == score && static_cast<uint32_t>(part_index[w]) < static_cast<uint32_t>(best))) {
        score = part[w];
        best = part_index[w];
      }
    __syncthreads();
    if (some) break;
  }
  return best;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_verify_next(const __grid_constant__ VerifyArgs a) {
  __shared__ Best warp_bests[kWarps];
  __shared__ Best cta_best;
  __shared__ double part[kWarps];
  __shared__ int part_index[kWarps], row_n, token_shared;
  __shared__ bool unsure;
  const uint32_t rank = cluster_rank(), parts = cluster_parts();
  const int64_t seq = blockIdx.x / parts;
  const int tid = threadIdx.x, lane = tid & 31, K = a.K;
  wait_for_previous();
  const Row* rows = a.rows + seq * (K + 1);
  if (tid < 32) {                                            // the first draft that is not accepted
    int n = K;
    for (int i0 = 0; i0 < K && n == K; i0 += 32) {
      const uint32_t bad = __ballot_sync(~0u, i0 + lane < K && !rows[i0 + lane].accepted);
      if (bad) n = i0 + __ffs(bad) - 1;
    }
    if (lane == 0) row_n = n;
  }
  __syncthreads();
  const int n = row_n;
  const int64_t x64 = n < K ? draft_of(a, seq, n) : -1;
  const bool rejected = x64 >= 0;
  const int x = x64 < a.classes ? static_cast<int>(x64) : -1;
  const T* z = static_cast<const T*>(a.logits) + seq * a.z_seq + n * a.z_row;
  const uint8_t* ok = a.allowed ? a.allowed + seq * a.ok_seq + n * a.ok_row : nullptr;
  const float* noise = a.noise + seq * a.noise_ld;
  const int64_t q0 = seq * a.q_seq + n * a.q_row;
  const Row st = rows[n];
  const bool dead = !(st.S > 0.0f);                          // no class, or a NaN
  Best best = {0.0f, 0.0f, 0.0f, -1};
  if (!dead) {
    const float c = a.c, inv_s = 1.0f / st.S;
    const bool minus_q = rejected && a.probs;
    const int hole = rejected && !a.probs ? x : -1;
    const int step = static_cast<int>(parts) * kThreads;
    for (int j0 = static_cast<int>(rank) * kThreads + tid; j0 < a.classes; j0 += step * kUnroll) {
      float v[kUnroll], q[kUnroll], e[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t j = j0 + static_cast<int64_t>(u) * step;
        v[u] = kNone<T>;
        q[u] = 0.0f;
        if (j < a.classes) {
          v[u] = logit(z, ok, static_cast<int>(j));
          e[u] = noise[j];
          if (minus_q) q[u] = prob_at(a, q0 + j);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int j = j0 + u * step;
        if (!(v[u] > kNone<T>) || j == hole) continue;
        const float d = (v[u] - st.m) * c, p = exp2_fast(d) * inv_s, rn = rcp_fast(e[u]);
        const Best one = {fmaxf(p - q[u], 0.0f) * rn, fmaf(bound(d, a.slack), p, FLT_MIN) * rn, 0.0f, j};
        if (!(one.score + one.off <= best.others)) best = better(best, one);
      }
    }
  }
  best = warp_best(best);
  if (lane == 0) warp_bests[tid >> 5] = best;
  __syncthreads();
  if (tid < 32) {
    best = warp_best(tid < kWarps ? warp_bests[tid] : Best{0.0f, 0.0f, 0.0f, -1});
    if (tid == 0) cta_best = best;
  }
  if (parts > 1) {
    cluster_barrier();
    if (rank == 0 && tid < 32) {
      best = {0.0f, 0.0f, 0.0f, -1};
      if (tid < static_cast<int>(parts))
        best = {from_cta(&cta_best.score, tid), from_cta(&cta_best.off, tid), from_cta(&cta_best.others, tid),
                from_cta(&cta_best.index, tid)};
      best = warp_best(best);
    }
    cluster_barrier();
    if (rank != 0) return;
  }
  if (tid == 0) {
    token_shared = best.index;
    unsure = !dead && !(best.score - best.off > best.others);
  }
  __syncthreads();
  int token = token_shared;
  if (unsure) token = exact_token(a, z, ok, noise, st.m, q0, x, rejected, part, part_index);
  for (int i = tid; i <= K; i += kThreads) {
    int t = -1;
    float lp = 0.0f;
    if (i < n) {
      t = static_cast<int>(draft_of(a, seq, i));
      lp = rows[i].logp;
    } else if (i == n) {
      t = dead ? -1 : token;
      if (dead) lp = st.S == 0.0f ? -INFINITY : NAN;
      else if (t >= 0) lp = fmaf(logit(z, ok, t) - st.m, a.inv_t, -logf(st.S));
    }
    a.tokens[seq * (K + 1) + i] = t;
    a.logp[seq * (K + 1) + i] = lp;
  }
  if (tid == 0) a.accepted[seq] = n;
}

// CTAs a row: until all rows' fill the GPU (152 SMs), as long as each has a round of loads.
int cluster_size(int64_t rows, int64_t bytes) {
  int parts = 1;
  while (parts < kMaxCluster && rows * parts < 152 && bytes / (2 * parts) >= kThreads * 16) parts *= 2;
  return parts;
}

template <typename K>
cudaError_t launch(K kernel, const VerifyArgs& a, int64_t rows, int parts, bool early, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows * parts));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (parts > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = parts;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  if (early) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T>
cudaError_t verify_type(const VerifyArgs& a, int64_t sequences, cudaStream_t s) {
  const int64_t rows = sequences * (a.K + 1), bytes = a.classes * static_cast<int64_t>(sizeof(T));
  const cudaError_t e = launch(k_verify_rows<T>, a, rows, cluster_size(rows, bytes), false, s);
  if (e != cudaSuccess) return e;
  return launch(k_verify_next<T>, a, sequences, cluster_size(sequences, a.classes * int64_t(8)), true, s);
}

bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_verify_workspace(int64_t sequences, int drafts, int64_t* bytes) {
  if (!bytes || sequences < 0 || drafts < 0) return HA_EINVAL;
  if (drafts >= 0x7FFFFFFF / kMaxCluster || sequences > 0x7FFFFFFF / kMaxCluster / (drafts + 1)) return HA_EUNSUPPORTED;
  *bytes = sequences * (drafts + 1) * static_cast<int64_t>(sizeof(Row));
  return HA_OK;
}

extern "C" int hier_avg_verify_drafts(const void* logits_dev, int type, int64_t sequences, int drafts, int64_t classes,
                                      int64_t logits_seq, int64_t logits_row, const void* drafts_dev, int draft_bytes,
                                      const float* uniform_dev, const float* noise_dev, int64_t noise_ld,
                                      const void* probs_dev, int probs_type, int64_t probs_seq, int64_t probs_row,
                                      const uint8_t* allowed_dev, int64_t allowed_seq, int64_t allowed_row,
                                      double temperature, int32_t* tokens_dev, int32_t* accepted_dev, float* logp_dev,
                                      void* workspace_dev, int64_t workspace_bytes, void* stream) {
  if (!type_ok(type) || sequences < 0 || drafts < 0 || classes < 1 || classes > 0x7FFFFFFF - (1 << 20) || logits_seq < 0 ||
      logits_row < 0 || noise_ld < 0 || (draft_bytes != 4 && draft_bytes != 8) ||
      !(temperature >= FLT_MIN && temperature <= 1e27) || misaligned(logits_dev, type_size(type)) ||
      misaligned(workspace_dev, 16))
    return HA_EINVAL;
  if (probs_dev && (!type_ok(probs_type) || probs_seq < 0 || probs_row < 0 || misaligned(probs_dev, type_size(probs_type))))
    return HA_EINVAL;
  if (allowed_dev && (allowed_seq < 0 || allowed_row < 0)) return HA_EINVAL;
  int64_t need;
  if (const int e = hier_avg_verify_workspace(sequences, drafts, &need)) return e;
  if (sequences == 0) return HA_OK;
  if (!logits_dev || !noise_dev || (drafts > 0 && (!drafts_dev || !uniform_dev)) || !tokens_dev || !accepted_dev || !logp_dev)
    return HA_EINVAL;
  if (!workspace_dev || workspace_bytes < need) return HA_ENOMEM;
  VerifyArgs a = {};
  a.logits = logits_dev;
  a.z_seq = logits_seq;
  a.z_row = logits_row;
  a.drafts = drafts_dev;
  a.uniform = uniform_dev;
  a.noise = noise_dev;
  a.noise_ld = noise_ld;
  a.probs = probs_dev;
  a.q_seq = probs_seq;
  a.q_row = probs_row;
  a.allowed = allowed_dev;
  a.ok_seq = allowed_seq;
  a.ok_row = allowed_row;
  a.tokens = tokens_dev;
  a.accepted = accepted_dev;
  a.logp = logp_dev;
  a.rows = static_cast<Row*>(workspace_dev);
  a.temperature = temperature;
  a.c = static_cast<float>(1.4426950408889634 / temperature);
  a.inv_t = static_cast<float>(1.0 / temperature);
  a.slack = slack(static_cast<int>(classes), 16 / type_size(type));
  a.K = drafts;
  a.classes = static_cast<int>(classes);
  a.wide_drafts = draft_bytes == 8;
  a.probs_type = probs_dev ? probs_type : -1;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = type == HA_TYPE_FP32   ? verify_type<float>(a, sequences, s)
                        : type == HA_TYPE_BF16 ? verify_type<__nv_bfloat16>(a, sequences, s)
                                               : verify_type<__half>(a, sequences, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}
