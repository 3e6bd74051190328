// The norm of all gradients together, the factor that clips them, and clipping in place:
//   norm = sqrt(sum over the tensors of their elements' squares),  scale = max_norm / norm where norm > max_norm, else 1,
// one of each for a learner where the tensors' first dimension is the learner's.
//
// A CTA takes 32 KB, or a warp 2 KB of small tensors, and sums its squares in fp32; a second kernel adds the sums in 64 bits,
// in a fixed order.  Squares that pass fp32's range, or are so small that it loses them, show in a chunk's sum,
// which is then taken again in 64 bits from the values, still in registers.  Clipping reads the gradients a
// second time, the last ones first, since those are still in L2.
// 285 M bf16 elements: 83 us, 6.9 TB/s; 300 fp32 tensors of 4.4 M elements, clipped: 14.2 us with a factor, 8.8
// where none is needed, most of it two launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <utility>
#include <vector>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kThreads = 256;
template <int THREADS> constexpr int kLoads = THREADS > 32 ? 8 : 4;       // 16-byte loads of a thread
// A chunk is a CTA's or, where tensors are small, a warp's.
template <int THREADS> constexpr int kChunkBytes = THREADS * kLoads<THREADS> * 16;
constexpr int kSmallPiece = 8192;         // bytes of a learner's part of a tensor, on average, below which they are small
constexpr int kOneThreads = 1024, kOneLearners = 152;
constexpr int kFew = 64, kSome = 384, kMany = 1400;      // tensors of a launch; its arguments are at most 32,764 bytes
constexpr int kMaxRanges = 32;
constexpr float kSmallSum = 0x1p-100f;    // a chunk's lost squares, 2^14 times 2^-150, are 2^-36 of it

template <int N> struct Table {
  const void* p[N];
  int64_t n[N];                           // elements of a learner
  int first[N + 1];                       // chunks of a learner before each tensor
  uint8_t type[N];
  int tensors;
};
struct Ranges {
  int64_t base[kMaxRanges];               // a launch's first sum
  int chunks[kMaxRanges];                 // and its chunks of each learner
  int n;
};

// A chunk: its elements and, from the first 16-byte boundary on, whole vectors.
template <typename T, int THREADS> struct Span {
  T* p;
  int n, head, vecs;
  __device__ __forceinline__ Span(const void* base, int64_t at, int64_t left) {
    constexpr int kElements = kChunkBytes<THREADS> / sizeof(T);
    p = static_cast<T*>(const_cast<void*>(base)) + at;
    n = static_cast<int>(left < kElements ? left : kElements);
    const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    head = min(n, shift ? kVec<T> - shift : 0);
    vecs = (n - head) / kVec<T>;
  }
  // The elements outside the vectors, at most 2 (kVec - 1): one a thread; -1 for the others.
  __device__ __forceinline__ int single() const {
    const int tid = threadIdx.x % THREADS, tail = head + vecs * kVec<T>;
    if (tid < head) return tid;
    return tid >= 16 && tail + tid - 16 < n ? tail + tid - 16 : -1;
  }
};

// The sum over a chunk's threads, in each of them (of 64 bits: in the first).  64-bit additions are few: this GPU does two a cycle
// and SM.
template <int THREADS, typename F>
__device__ __forceinline__ F chunk_sum(F x, F* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  if constexpr (THREADS > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = part[0];
    if (sizeof(F) == 4 || threadIdx.x == 0) {
#pragma unroll
      for (int w = 1; w < THREADS / 32; ++w) x += part[w];
    }
  }
  return x;
}

template <typename T, int THREADS>
__device__ __forceinline__ double sum_of_squares(const Span<T, THREADS>& c, float* part, double* wide) {
  const int tid = threadIdx.x % THREADS;
  uint4 w[kLoads<THREADS>];
#pragma unroll
  for (int u = 0; u < kLoads<THREADS>; ++u) {
    const int i = u * THREADS + tid;
    w[u] = i < c.vecs ? __ldg(reinterpret_cast<const uint4*>(c.p + c.head) + i) : make_uint4(0, 0, 0, 0);
  }
  const int one = c.single();
  const float x = one >= 0 ? Elem<T>::up(c.p[one]) : 0.0f;
  Pair s[2] = {pair(x * x, 0.0f), pair(0.0f, 0.0f)};
#pragma unroll
  for (int u = 0; u < kLoads<THREADS>; ++u) {
    float v[kVec<T>];
    unpack<T>(w[u], v);
#pragma unroll
    for (int e = 0; e < kVec<T>; e += 2) {
      const Pair q = pair(v[e], v[e + 1]);
      s[e / 2 & 1] = fma2(q, q, s[e / 2 & 1]);
    }
  }
  float a, b;
  halves(add2(s[0], s[1]), a, b);
  const float sum = chunk_sum<THREADS>(a + b, part);
  if (sum >= kSmallSum && sum < INFINITY) return sum;
  uint32_t any = __float_as_uint(x) & 0x7FFFFFFFu;
#pragma unroll
  for (int u = 0; u < kLoads<THREADS>; ++u) {
    constexpr uint32_t kSigns = sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu;
    any |= (w[u].x | w[u].y | w[u].z | w[u].w) & kSigns;
  }
  if (!(THREADS > 32 ? __syncthreads_or(any != 0) : __any_sync(~0u, any != 0))) return 0.0;
  double d = static_cast<double>(x) * x;
#pragma unroll 1
  for (int u = 0; u < kLoads<THREADS>; ++u) {
    float v[kVec<T>];
    uint4 q = w[0];
#pragma unroll
    for (int i = 1; i < kLoads<THREADS>; ++i)
      if (i == u) q = w[i];
    unpack<T>(q, v);
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) d += static_cast<double>(v[e]) * v[e];
  }
  return chunk_sum<THREADS>(d, wide);
}

template <typename T, int THREADS>
__device__ __forceinline__ void scale_by(const Span<T, THREADS>& c, float f) {
  const int tid = threadIdx.x % THREADS;
  uint4* at = reinterpret_cast<uint4*>(c.p + c.head);
  uint4 w[kLoads<THREADS>];
#pragma unroll
  for (int u = 0; u < kLoads<THREADS>; ++u) {
    const int i = u * THREADS + tid;
    if (i < c.vecs) w[u] = at[i];
  }
#pragma unroll
  for (int u = 0; u < kLoads<THREADS>; ++u) {
    const int i = u * THREADS + tid;
    float v[kVec<T>];
    unpack<T>(w[u], v);
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) v[e] *= f;
    if (i < c.vecs) at[i] = pack<T>(v);
  }
  const int one = c.single();
  if (one >= 0) c.p[one] = Elem<T>::down(Elem<T>::up(c.p[one]) * f);
}

// The chunk `c` of learner `p`: f(span).
template <int THREADS, int N, typename F>
__device__ __forceinline__ void with_chunk(const Table<N>& t, int p, int c, F f) {
  int low = 0, high = t.tensors - 1;      // the last tensor whose first chunk is not behind c
  while (low < high) {
    const int mid = (low + high + 1) / 2;
    if (t.first[mid] <= c) low = mid;
    else high = mid - 1;
  }
  const int64_t size = t.type[low] == HA_TYPE_FP32 ? 4 : 2, skip = static_cast<int64_t>(c - t.first[low]) * (kChunkBytes<THREADS> / size);
  const int64_t at = p * t.n[low] + skip, left = t.n[low] - skip;
  if (t.type[low] == HA_TYPE_FP32) f(Span<float, THREADS>(t.p[low], at, left));
  else if (t.type[low] == HA_TYPE_BF16) f(Span<__nv_bfloat16, THREADS>(t.p[low], at, left));
  else f(Span<__half, THREADS>(t.p[low], at, left));
}

// CTAs of a learner, each with a chunk, or one a warp.
template <int THREADS> __host__ __device__ constexpr int ctas_of(int chunks) { return (chunks + kThreads / THREADS - 1) / (kThreads / THREADS); }

template <int N, int THREADS>
__global__ void __launch_bounds__(kThreads) k_squares(const __grid_constant__ Table<N> t, double* sums) {
  __shared__ float part[kThreads / 32];
  __shared__ double wide[kThreads / 32];
  const int chunks = t.first[t.tensors], ctas = ctas_of<THREADS>(chunks), p = blockIdx.x / ctas;
  const int c = blockIdx.x % ctas * (kThreads / THREADS) + threadIdx.x / THREADS;
  let_next_start();
  if (c >= chunks) return;
  with_chunk<THREADS>(t, p, c, [&](auto span) {
    const double s = sum_of_squares(span, part, wide);
    if (threadIdx.x % THREADS == 0) sums[static_cast<int64_t>(p) * chunks + c] = s;
  });
}

// Few chunks' sum, by one warp: 64-bit additions are slow, and each CTA that clips does them by itself.  (The sums are no __restrict__
// const here and below: the kernel may start while the one before it still writes them, and reads them behind its wait.)
constexpr int kFewChunks = 1024;
__device__ __forceinline__ double warp_total(const double* sums, int n) {
  double s = 0.0;
#pragma unroll 8
  for (int c = threadIdx.x & 31; c < n; c += 32) s += sums[c];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
  return s;
}
__device__ __forceinline__ float scale_of(double norm, double max_norm) {
  return norm > max_norm ? static_cast<float>(max_norm / norm) : 1.0f;
}

// A CTA a learner.
__global__ void __launch_bounds__(kThreads) k_norm(const double* sums, const __grid_constant__ Ranges r, double max_norm, float* norm,
                                                   float* scale) {
  __shared__ double part[kThreads / 32];
  let_next_start();
  wait_for_previous();
  const int p = blockIdx.x;
  double s = 0.0;
  if (r.n == 1 && r.chunks[0] <= kFewChunks) {
    if (threadIdx.x < 32) s = warp_total(sums + static_cast<int64_t>(p) * r.chunks[0], r.chunks[0]);
  } else {
    for (int i = 0; i < r.n; ++i) {
      const double* from = sums + r.base[i] + static_cast<int64_t>(p) * r.chunks[i];
#pragma unroll 8
      for (int c = threadIdx.x; c < r.chunks[i]; c += kThreads) s += from[c];
    }
    s = chunk_sum<kThreads>(s, part);
  }
  if (threadIdx.x == 0) {
    s = sqrt(s);
    norm[p] = static_cast<float>(s);
    if (scale) scale[p] = scale_of(s, max_norm);
  }
}

// With sums, few chunks': their norm is taken here, as k_norm takes it, and written by a learner's first chunk (300 tensors of 4.4 M
// elements: a launch less, 21.6 to 18.9 us a call, the host's time included).
template <int N, int THREADS>
__global__ void __launch_bounds__(kThreads) k_clip(const __grid_constant__ Table<N> t, const double* sums, double max_norm, float* norm,
                                                   float* scale) {
  __shared__ float factor;
  const int chunks = t.first[t.tensors], ctas = ctas_of<THREADS>(chunks), b = static_cast<int>(gridDim.x - 1 - blockIdx.x), p = b / ctas;
  const int c = b % ctas * (kThreads / THREADS) + threadIdx.x / THREADS;
  let_next_start();
  wait_for_previous();
  if (sums) {
    if (threadIdx.x < 32) {
      double s = warp_total(sums + static_cast<int64_t>(p) * chunks, chunks);
      if (threadIdx.x == 0) {
        s = sqrt(s);
        factor = scale_of(s, max_norm);
        if (c == 0) {
          norm[p] = static_cast<float>(s);
          scale[p] = factor;
        }
      }
    }
    __syncthreads();
  }
  const float f = sums ? factor : scale[p];
  if (f == 1.0f || c >= chunks) return;
  with_chunk<THREADS>(t, p, c, [&](auto span) { scale_by(span, f); });
}

// Few and small tensors: a CTA a learner does it all, a chunk a warp at a time.
template <int N>
__global__ void __launch_bounds__(kOneThreads) k_norm_one(const __grid_constant__ Table<N> t, double max_norm, bool clip, float* norm,
                                                          float* scale) {
  constexpr int kWarps = kOneThreads / 32;
  __shared__ double part[kWarps];
  __shared__ float factor;
  const int chunks = t.first[t.tensors], p = blockIdx.x, warp = threadIdx.x / 32;
  double s = 0.0;
  for (int c = warp; c < chunks; c += kWarps) with_chunk<32>(t, p, c, [&](auto span) { s += sum_of_squares(span, nullptr, nullptr); });
  if (threadIdx.x % 32 == 0) part[warp] = s;
  __syncthreads();
  if (warp == 0) {
    s = warp_total(part, kWarps);
    if (threadIdx.x == 0) {
      s = sqrt(s);
      norm[p] = static_cast<float>(s);
      factor = scale_of(s, max_norm);
      if (scale) scale[p] = factor;
    }
  }
  if (!clip) return;
  __syncthreads();
  if (factor == 1.0f) return;
  for (int c = warp; c < chunks; c += kWarps) with_chunk<32>(t, p, c, [&](auto span) { scale_by(span, factor); });
}

// Chunks of one learner's part of a tensor.
int64_t chunks_of(int64_t n, int type, int threads) {
  static_assert(kChunkBytes<32> == 1 << 11 && kChunkBytes<kThreads> == 1 << 15, "");
  const int shift = (threads == 32 ? 11 : 15) - (type == HA_TYPE_FP32 ? 2 : 1);
  return (n + (int64_t(1) << shift) - 1) >> shift;
}

struct Call {
  const void* const* grads;
  const int* types;
  const int64_t* n;
  int learners, threads;
  double* sums;
  double max_norm;
  float *norm, *scale;
  cudaStream_t s;
};
enum Pass { kSquares, kClip, kNormAndClip, kOne, kOneAndClip };

template <int N>
cudaError_t launch_range(const Call& a, int t0, int t1, int64_t base, Pass pass, int& chunks) {
  Table<N> t;
  t.tensors = t1 - t0;
  int64_t at = 0;
  const int threads = pass >= kOne ? 32 : a.threads;
  for (int i = t0; i < t1; ++i) {
    t.p[i - t0] = a.grads[i];
    t.n[i - t0] = a.learners == 1 ? a.n[i] : a.n[i] / a.learners;
    t.type[i - t0] = static_cast<uint8_t>(a.types[i]);
    t.first[i - t0] = static_cast<int>(at);
    at += chunks_of(t.n[i - t0], a.types[i], threads);
  }
  t.first[t.tensors] = static_cast<int>(at);
  chunks = static_cast<int>(at);
  if (pass >= kOne) {
    k_norm_one<N><<<a.learners, kOneThreads, 0, a.s>>>(t, a.max_norm, pass == kOneAndClip, a.norm, a.scale);
    return cudaGetLastError();
  }
  if (at == 0) return cudaSuccess;
  const unsigned grid = static_cast<unsigned>(a.learners) * (threads == 32 ? ctas_of<32>(chunks) : ctas_of<kThreads>(chunks));
  if (pass != kSquares)
    return launch_early(threads == 32 ? k_clip<N, 32> : k_clip<N, kThreads>, grid, kThreads, 0, a.s, t,
                        static_cast<const double*>(pass == kNormAndClip ? a.sums : nullptr), a.max_norm, a.norm, a.scale);
  if (threads == 32) k_squares<N, 32><<<grid, kThreads, 0, a.s>>>(t, a.sums + base);
  else k_squares<N, kThreads><<<grid, kThreads, 0, a.s>>>(t, a.sums + base);
  return cudaGetLastError();
}
cudaError_t launch_all(const Call& a, int tensors, Pass pass, Ranges& r) {
  r.n = 0;
  int64_t base = 0;
  const int each = tensors <= kFew ? kFew : tensors <= kSome ? kSome : kMany;
  for (int t = 0; t < tensors; t += each) {
    const int end = std::min(t + each, tensors);
    int chunks = 0;
    const cudaError_t e = each == kFew    ? launch_range<kFew>(a, t, end, base, pass, chunks)
                          : each == kSome ? launch_range<kSome>(a, t, end, base, pass, chunks)
                                          : launch_range<kMany>(a, t, end, base, pass, chunks);
    if (e != cudaSuccess) return e;
    r.base[r.n] = base;
    r.chunks[r.n++] = chunks;
    base += static_cast<int64_t>(chunks) * a.learners;
  }
  return cudaSuccess;
}

// How a call is done.  One CTA a learner takes a chunk for each of its warps: 10 tensors of 17 thousand 16-bit elements 4.0 us, by two
// kernels 3.9 and 2 us of the host's; 111 tensors of 213 thousand 13.8 and 4.6.  Small tensors' chunks are a warp's: clipping
// 335 tensors of 5 learners, 1 KB each, 5.8 us, 15 with a CTA each.
constexpr int kOneChunks = kOneThreads / 32;
struct Plan {
  int threads;
  int64_t sums;                           // below 0: a status
  bool one;
};
Plan plan_of(int tensors, const int* types, const int64_t* n, int learners) {
  if (tensors < 1 || learners < 1 || !types || !n) return {0, HA_EINVAL, false};
  if (tensors > kMaxRanges * kMany) return {0, HA_EUNSUPPORTED, false};
  int64_t cta = 0, warp = 0, bytes = 0, pieces = 0;         // chunks of a learner
  for (int i = 0; i < tensors; ++i) {
    if (!type_ok(types[i]) || n[i] < 0 || (learners > 1 && n[i] % learners)) return {0, HA_EINVAL, false};
    if (n[i] > int64_t(1) << 46) return {0, HA_EUNSUPPORTED, false};
    const int64_t mine = learners == 1 ? n[i] : n[i] / learners;
    cta += chunks_of(mine, types[i], kThreads);
    warp += chunks_of(mine, types[i], 32);
    bytes += mine * type_size(types[i]);
    pieces += n[i] > 0;
  }
  const bool small = bytes < kSmallPiece * pieces;
  const int64_t chunks = small ? warp : cta;
  if (chunks > 0x7FFFFFFF / learners) return {0, HA_EUNSUPPORTED, false};
  return {small ? 32 : kThreads, chunks * learners, warp <= kOneChunks && tensors <= kMany && learners <= kOneLearners};
}

// Do the gradients share memory?  They are usually in the order of their addresses.
bool overlap(int tensors, const void* const* grads, const int* types, const int64_t* n) {
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  spans.reserve(tensors);
  for (int i = 0; i < tensors; ++i)
    if (n[i]) {
      const uintptr_t p = reinterpret_cast<uintptr_t>(grads[i]);
      spans.push_back({p, p + static_cast<uintptr_t>(n[i]) * type_size(types[i])});
    }
  if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].first < spans[i - 1].second) return true;
  return false;
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_grad_norm_workspace(int tensors, const int* types, const int64_t* n, int learners, int64_t* bytes) {
  if (!bytes) return HA_EINVAL;
  const Plan plan = plan_of(tensors, types, n, learners);
  if (plan.sums < 0) return static_cast<int>(plan.sums);
  *bytes = std::max<int64_t>(plan.sums, 1) * static_cast<int64_t>(sizeof(double));
  return HA_OK;
}

extern "C" int hier_avg_grad_norm(int tensors, void* const* grads_dev, const int* types, const int64_t* n, int learners,
                                  double max_norm, int clip, float* norm_dev, float* scale_dev, void* workspace_dev,
                                  int64_t workspace_bytes, void* stream) {
  const Plan plan = plan_of(tensors, types, n, learners);
  if (plan.sums < 0) return static_cast<int>(plan.sums);
  if (!grads_dev || !norm_dev || (clip && !scale_dev) || (scale_dev && !(max_norm >= 0.0 && std::isfinite(max_norm))))
    return HA_EINVAL;
  for (int i = 0; i < tensors; ++i)
    if (n[i] && (!grads_dev[i] || reinterpret_cast<uintptr_t>(grads_dev[i]) % type_size(types[i]))) return HA_EINVAL;
  if (!workspace_dev || workspace_bytes < plan.sums * static_cast<int64_t>(sizeof(double))) return HA_ENOMEM;
  if (reinterpret_cast<uintptr_t>(workspace_dev) % sizeof(double)) return HA_EINVAL;
  try {
    if (clip && overlap(tensors, grads_dev, types, n)) return HA_EINVAL;
  } catch (const std::bad_alloc&) {
    return HA_ENOMEM;
  }
  const Call a = {grads_dev, types, n, learners, plan.threads, static_cast<double*>(workspace_dev), max_norm, norm_dev, scale_dev,
                  static_cast<cudaStream_t>(stream)};
  Ranges r;
  std::memset(&r, 0, sizeof r);
  if (plan.one) return launch_all(a, tensors, clip ? kOneAndClip : kOne, r) == cudaSuccess ? HA_OK : HA_ECUDA;
  cudaError_t e = launch_all(a, tensors, kSquares, r);
  const bool few = clip && r.n == 1 && r.chunks[0] > 0 && r.chunks[0] <= kFewChunks;
  if (e == cudaSuccess && !few)
    e = launch_early(k_norm, static_cast<unsigned>(learners), kThreads, 0, a.s, a.sums, r, max_norm, norm_dev, scale_dev);
  if (e == cudaSuccess && clip) e = launch_all(a, tensors, few ? kNormAndClip : kClip, r);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}
