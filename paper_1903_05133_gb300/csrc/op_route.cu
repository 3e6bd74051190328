// The router of rows to experts, the sort of rows by their group, and the router's gradient.
//
// For a row z over E experts: the k largest logits (equal ones by index), lse = log sum_i e^(z_i), and
//   over the chosen: w_j = e^(z_j) / sum over the chosen of e^z,   over all: w_j = e^(z_j - lse).
// The entries (row, j) are then sorted by group, in their order within a group: a counting sort.
// Each warp takes rows that follow one another and counts them by group in shared memory, where a
// group's count is the next entry's rank; the CTA's warps, then the CTAs add up their counts in order.  A CTA an SM, so
// that with few groups the second kernel's CTAs can each add up all CTAs' counts by themselves.
//
//   over the chosen: dz_j = w_j (dw_j - s) at the chosen, 0 elsewhere;  s = sum over the chosen of w dw
//   over all:        dz_i = [i chosen] w_i dw_i - p_i s,                p_i = e^(z_i - lse)
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kMaxExperts = 1024, kMaxGroups = 1024, kMaxChosen = 32;
constexpr int kCtas = 152;                // of a sort
constexpr int kWarps = 32;                // of a CTA
template <int L, int R> constexpr int kRouteWarps = L == 32 && R > 8 ? kWarps / 2 : kWarps;   // their logits fill the registers
constexpr int kBackWarps = 8;             // of a CTA of the gradient
constexpr int kSumGroups = 128;           // groups whose counts each CTA adds up by itself
constexpr int kRankBits = 21;             // an entry in work: its group above, its rank below
constexpr int kStaged = 2048;             // entries of a CTA that are kept in shared memory meanwhile
constexpr int64_t kMaxChunk = int64_t(1) << (kRankBits - 1);

struct SortArgs {
  int* offsets;                           // [groups + 1]
  int* place;                             // [entries]
  int* source;                            // [entries]
  int* counts;                            // of group g in chunk c: [g * g_step + c * c_step]
  int* totals;                            // [groups]
  int64_t entries;
  int64_t per;                            // entries of a chunk
  int groups, chunks;
  int g_step, c_step;                     // chunk after chunk, or group after group where a kernel of its own adds them up
};

// Exclusive sums of value[0, n) in place and their total behind them.
__device__ __forceinline__ void block_scan(int* value, int n, int* warp_sum) {
  const int tid = threadIdx.x, lane = tid & 31, warps = blockDim.x >> 5;
  const int each = (n + blockDim.x - 1) / blockDim.x, at = tid * each;
  int sum = 0;
  for (int i = at; i < min(at + each, n); ++i) sum += value[i];
  int run = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(~0u, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) warp_sum[tid >> 5] = run;
  __syncthreads();
  if (tid < 32) {
    int w = tid < warps ? warp_sum[tid] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(~0u, w, o);
      if (lane >= o) w += x;
    }
    if (tid < warps) warp_sum[tid] = w;
  }
  __syncthreads();
  int before = run - sum + (tid >= 32 ? warp_sum[(tid >> 5) - 1] : 0);
  for (int i = at; i < min(at + each, n); ++i) {
    const int v = value[i];
    value[i] = before;
    before += v;
  }
  if (tid == 0) value[n] = warp_sum[warps - 1];
  __syncthreads();
}

// The end of a chunk's first pass: hist [warps, groups] holds each warp's counts, stage the entries with
// their rank in their warp.  The ranks become those in the chunk, or with ONE the places.
template <bool ONE>
__device__ __forceinline__ void end_chunk(const SortArgs& a, int* hist, int* total, const int* stage, int64_t e0, int n) {
  __shared__ int warp_sum[32];
  const int warps = blockDim.x >> 5;
  __syncthreads();
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    int run = 0;
#pragma unroll 8
    for (int w = 0; w < warps; ++w) {
      const int c = hist[w * a.groups + g];
      hist[w * a.groups + g] = run;
      run += c;
    }
    if (ONE) total[g] = run;
    else a.counts[static_cast<int64_t>(g) * a.g_step + static_cast<int64_t>(blockIdx.x) * a.c_step] = run;
  }
  __syncthreads();
  if (ONE) {
    block_scan(total, a.groups, warp_sum);
    for (int g = threadIdx.x; g <= a.groups; g += blockDim.x) a.offsets[g] = total[g];
  }
}

// ---------------------------------------------------------------- the router
struct RouteArgs {
  const void* logits;
  int64_t rows, ld;
  const int* learners;                    // nullptr: one
  int n_learners, experts, k;
  bool all;
  int* expert;
  float* weight;
  float* lse;
  SortArgs sort;
};

template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  if constexpr (L == 32) {
    return __reduce_max_sync(~0u, x);
  } else {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) x = max(x, __shfl_xor_sync(~0u, x, o));
    return x;
  }
}
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}

// A logit's key, its order among the row's.  A 16-bit logit's key has its index below, so that no two are equal; equal ones of
// fp32 have equal keys.  v: the logit, raised to kNone where it is below; +0 makes zeros of both signs the same.
template <typename T> constexpr bool kUnique = sizeof(T) == 2;
template <typename T>
__device__ __forceinline__ uint32_t key_of(float v, int index) {
  if constexpr (kUnique<T>) {
    // 16 bits of the type in their order: bf16 is the upper half of an fp32
    uint32_t u = __float_as_uint(v + 0.0f);
    if constexpr (!std::is_same<T, __nv_bfloat16>::value) u = static_cast<uint32_t>(__half_as_ushort(__float2half_rn(v + 0.0f))) << 16;
    const uint32_t flip = (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u) & 0xFFFF0000u;
    return (u ^ flip) | static_cast<uint32_t>(0xFFFF - index);
  } else {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u);
  }
}
template <typename T>
__device__ __forceinline__ float value_of(uint32_t key) {
  const uint32_t o = kUnique<T> ? key & 0xFFFF0000u : key;
  uint32_t u = o & 0x80000000u ? o ^ 0x80000000u : ~o;
  if constexpr (kUnique<T>) u &= 0xFFFF0000u;
  if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half(static_cast<unsigned short>(u >> 16)));
  return __uint_as_float(u);
}
// The keys of what is masked are at most this (fp16 has nothing at kNone but minus infinity).
template <typename T>
__device__ __forceinline__ uint32_t key_none() {
  return std::is_same<T, __half>::value ? 0x03FFFFFFu : key_of<T>(kNone<T>, 0) | (kUnique<T> ? 0xFFFFu : 0u);
}

// L lanes take a row, at least as many as it has chosen ones; lane l of them holds the logits l, l + L, ...  The chosen
// are found from the largest down: of a lane's keys below the last, less the last, the largest is that of the keys, since
// differences of unsigned numbers wrap, in one instruction a key.  Several rows a warp share the latencies.
template <typename T, int L, int R, bool ONE>
__global__ void __launch_bounds__(32 * kRouteWarps<L, R>) k_route(const __grid_constant__ RouteArgs a) {
  extern __shared__ int dyn[];
  constexpr int kRows = 32 / L;                               // of a warp at a time
  __shared__ uint32_t slot_key[kUnique<T> ? 1 : kRouteWarps<L, R>][32];
  __shared__ int slot_index[kUnique<T> ? 1 : kRouteWarps<L, R>][32];
  constexpr uint32_t kLanes = L == 32 ? ~0u : (1u << L) - 1;
  const int lane = threadIdx.x & 31, l = lane % L, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int G = a.sort.groups, k = a.k;
  int* hist = dyn;                                            // [warps, groups]
  int* total = hist + warps * G;                              // [groups + 1] (ONE)
  const int64_t per_rows = a.sort.per / k, r0 = blockIdx.x * per_rows;
  const int n_rows = static_cast<int>(min(per_rows, a.rows - r0));
  int* stage = a.sort.per <= kStaged ? total + G + 1 : a.sort.place + r0 * k;
  let_next_start();
  for (int i = threadIdx.x; i < warps * G; i += blockDim.x) hist[i] = 0;
  __syncthreads();

  // a multiple of kRows for every warp but the last, so that none is idle beside another's rows
  const int each = ((n_rows + warps - 1) / warps + kRows - 1) / kRows * kRows;
  const int first = min(warp * each, n_rows), last = min(first + each, n_rows);
  int learner = 0;
  if (a.learners && first < last) {                           // learners that end at or before the warp's first row
    int high = a.n_learners;
    while (learner < high) {
      const int mid = (learner + high) / 2;
      if (a.learners[mid + 1] <= r0 + first) learner = mid + 1;
      else high = mid;
    }
  }
  for (int r1 = first; r1 < last; r1 += kRows) {
    const int r = r1 + lane / L;
    const bool mine = r < last;
    const int64_t row = r0 + (mine ? r : r1);                 // lanes without a row repeat the first's
    const T* z = static_cast<const T*>(a.logits) + row * a.ld;
    const uint32_t none = key_none<T>();
    uint32_t key[R], most = 0;
    float v[R];
#pragma unroll
    for (int u = 0; u < R; ++u) v[u] = u * L + l < a.experts ? Elem<T>::up(z[u * L + l]) : -INFINITY;
#pragma unroll
    for (int u = 0; u < R; ++u) {
      v[u] = max_nan(v[u], kNone<T>);
      key[u] = key_of<T>(v[u], u * L + l);
      most = max(most, key[u]);
    }
    const uint32_t top = lanes_max<L>(most);
    const float m = value_of<T>(top);
    Pair S2 = pair(0.0f, 0.0f);
#pragma unroll
    for (int u = 0; u < R; u += 2) {
      float x, y;
      halves(mul2(add2(pair(v[u], v[u + 1]), pair(-m, -m)), pair(kLog2e, kLog2e)), x, y);
      S2 = add2(S2, pair(exp2_fast(x), exp2_fast(y)));
    }
    float x, y;
    halves(S2, x, y);
    const float S = lanes_sum<L>(x + y);                      // NaN where a logit is NaN, or infinite: inf - inf
    const bool bad = !(S == S);

    uint32_t slot = l == 0 && top > none ? top : 0, best = max(top, none);     // lane j's is the j-th
    for (int j = 1; j < k; ++j) {
      uint32_t t = 0;
#pragma unroll
      for (int u = 0; u < R; ++u) t = __viaddmax_u32(key[u], 0u - best, t);
      const uint32_t next = lanes_max<L>(t) + best;
      best = next < best ? max(next, none) : none;            // (none is below it)
      if (l == j) slot = best > none ? best : 0;
    }
    int index = -1;
    if constexpr (kUnique<T>) {
      if (slot) index = 0xFFFF - static_cast<int>(slot & 0xFFFFu);
    } else {
      // Which are they?  As many as there are slots, unless logits are equal.
      uint32_t held = 0;
      const uint32_t least = max(best, none + 1);
#pragma unroll
      for (int u = 0; u < R; ++u) held |= key[u] >= least ? 1u << u : 0;
      int n = __popc(held);
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) n += __shfl_xor_sync(~0u, n, o);
      const int slots = __popc(__ballot_sync(~0u, slot != 0) >> (lane - l) & kLanes);
      if (__any_sync(~0u, n != slots)) {                      // then one by one, the lowest index first
        slot = 0;
        for (int j = 0; j < k; ++j) {
          uint32_t mine_most = 0;
          int at = 0;
#pragma unroll
          for (int u = 0; u < R; ++u)
            if (key[u] > mine_most) {
              mine_most = key[u];
              at = u;
            }
          const uint32_t first = lanes_max<L>(mine_most);
          const uint32_t i = mine_most == first ? static_cast<uint32_t>(at * L + l) : ~0u;
          const uint32_t lowest = ~lanes_max<L>(~i);
          if (first <= none) continue;                        // of this row; others' lanes go on
          if (l == j) {
            slot = first;
            index = static_cast<int>(lowest);
          }
          if (static_cast<int>(lowest) % L == l) {
#pragma unroll
            for (int u = 0; u < R; ++u)
              if (u * L + l == static_cast<int>(lowest)) key[u] = 0;
          }
        }
      } else {
        slot_key[warp][lane] = slot;
        __syncwarp();
        while (held) {
          const int i = (__ffs(held) - 1) * L + l;
          held &= held - 1;
          const uint32_t mine_key = key_of<T>(Elem<T>::up(z[i]), i);
          for (int j = 0; j < k; ++j)
            if (slot_key[warp][lane - l + j] == mine_key) slot_index[warp][lane - l + j] = i;
        }
        __syncwarp();
        if (slot) index = slot_index[warp][lane];
      }
    }
    if (bad) index = -1;
    const float e = index >= 0 ? expf(value_of<T>(slot) - m) : 0.0f;
    const float sum = a.all ? S : lanes_sum<L>(e);
    if (mine && l < k) {
      a.expert[row * k + l] = index;
      a.weight[row * k + l] = bad ? NAN : index >= 0 ? e / sum : 0.0f;
    }
    if (mine && l == 0) a.lse[row] = bad ? NAN : top <= none ? -INFINITY : m + logf(S);

    int group = mine && l < k ? index : -1;
    if (a.learners) {
      int p = learner;
      while (p < a.n_learners && a.learners[p + 1] <= row) ++p;
      if (p >= a.n_learners || row < a.learners[p]) group = -1;
      else if (group >= 0) group += p * a.experts;
      learner = __shfl_sync(~0u, p, 0);                       // the first row's is not behind the others'
    }
    int packed = -1;
    if constexpr (kRows == 1) {
      if (group >= 0) {                                       // a row's experts differ
        const int rank = hist[warp * G + group];
        hist[warp * G + group] = rank + 1;
        packed = group << kRankBits | rank;
      }
    } else {
      const uint32_t same = __match_any_sync(~0u, group);
      int rank = 0;
      if (group >= 0) {
        rank = hist[warp * G + group];
        packed = group << kRankBits | (rank + __popc(same & ((1u << lane) - 1)));
      }
      __syncwarp();
      if (group >= 0 && lane == __ffs(same) - 1) hist[warp * G + group] = rank + __popc(same);
    }
    if (mine && l < k) stage[r * k + l] = packed;
    __syncwarp();
  }
  end_chunk<ONE>(a.sort, hist, total, stage, r0 * k, n_rows * k);
  const int64_t e0 = r0 * k;
  for (int i = first * k + lane; i < last * k; i += 32) {
    int p = stage[i];
    if (p >= 0) {
      p += hist[warp * G + (p >> kRankBits)];
      if (ONE) {
        p = (p & ((1 << kRankBits) - 1)) + total[p >> kRankBits];
        a.sort.source[p] = i;
      }
    }
    a.sort.place[e0 + i] = p;
  }
  if (ONE)
    for (int p = total[G] + threadIdx.x; p < n_rows * k; p += blockDim.x) a.sort.source[p] = -1;
}

// ---------------------------------------------------------------- the sort of given groups
template <bool ONE>
__global__ void __launch_bounds__(32 * kWarps) k_group(const int* __restrict__ ids, const __grid_constant__ SortArgs a) {
  extern __shared__ int dyn[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, G = a.groups;
  int* hist = dyn;
  int* total = hist + warps * G;
  const int64_t e0 = blockIdx.x * a.per;
  const int n = static_cast<int>(min(a.per, a.entries - e0));
  int* stage = a.per <= kStaged ? total + G + 1 : a.place + e0;
  let_next_start();
  for (int i = threadIdx.x; i < warps * G; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  const int each = (n + warps - 1) / warps, first = min(warp * each, n), last = min(first + each, n);
  for (int i0 = first; i0 < last; i0 += 32) {
    const int i = i0 + lane;
    int g = i < last ? ids[e0 + i] : -1;
    if (g >= G) g = -1;
    const uint32_t same = __match_any_sync(~0u, g);
    int packed = -1, count = 0;
    if (g >= 0) {
      count = hist[warp * G + g];
      packed = g << kRankBits | (count + __popc(same & ((1u << lane) - 1)));
    }
    __syncwarp();
    if (g >= 0 && lane == __ffs(same) - 1) hist[warp * G + g] = count + __popc(same);
    if (i < last) stage[i] = packed;
    __syncwarp();
  }
  end_chunk<ONE>(a, hist, total, stage, e0, n);
  for (int i = first + lane; i < last; i += 32) {
    int p = stage[i];
    if (p >= 0) {
      p += hist[warp * G + (p >> kRankBits)];
      if (ONE) {
        p = (p & ((1 << kRankBits) - 1)) + total[p >> kRankBits];
        a.source[p] = i;
      }
    }
    a.place[e0 + i] = p;
  }
  if (ONE)
    for (int p = total[G] + threadIdx.x; p < n; p += blockDim.x) a.source[p] = -1;
}

// A warp a group: the chunks' counts become what comes before each chunk.
__global__ void __launch_bounds__(kBackWarps * 32) k_chunks(const __grid_constant__ SortArgs a) {
  const int lane = threadIdx.x & 31, g = blockIdx.x * kBackWarps + (threadIdx.x >> 5);
  let_next_start();
  wait_for_previous();
  if (g >= a.groups) return;
  int* c = a.counts + static_cast<int64_t>(g) * a.chunks;
  int carry = 0;
  for (int i0 = 0; i0 < a.chunks; i0 += 128) {
    int v[4], sum = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + lane * 4 + u;
      v[u] = i < a.chunks ? c[i] : 0;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) sum += v[u];
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(~0u, run, o);
      if (lane >= o) run += x;
    }
    int before = carry + run - sum;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + lane * 4 + u;
      if (i < a.chunks) c[i] = before;
      before += v[u];
    }
    carry += __shfl_sync(~0u, run, 31);
  }
  if (lane == 0) a.totals[g] = carry;
}

// Ranks in a chunk become places.  SUM, for at most kSumGroups groups: the counts of all chunks are added up here, by as many threads
// a group as there are, all loads at once, and one warp makes places of them.
template <bool SUM>
__global__ void __launch_bounds__(kWarps * 32) k_place(const __grid_constant__ SortArgs a) {
  __shared__ int base[kMaxGroups + 1], mine[kMaxGroups];
  __shared__ int warp_sum[32];
  const int chunk = blockIdx.x, tid = threadIdx.x;
  const int64_t e0 = chunk * a.per, e1 = min(e0 + a.per, a.entries);
  int next = -1;
  if (SUM) {
    for (int i = tid; i < a.groups; i += blockDim.x) base[i] = mine[i] = 0;
    __syncthreads();
    wait_for_previous();
    if (e0 + tid < e1) next = a.place[e0 + tid];              // on its way meanwhile
    int shift = 5;                                            // threads of a part, a power of two
    while (1 << shift < a.groups) ++shift;
    const int g = tid & ((1 << shift) - 1), parts = static_cast<int>(blockDim.x) >> shift;
    if (g < a.groups) {
      constexpr int kAtOnce = 20;                             // 152 chunks by 8 threads a group
      for (int c0 = tid >> shift; c0 < a.chunks; c0 += parts * kAtOnce) {
        int n[kAtOnce], all = 0, before = 0;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int c = c0 + u * parts;
          n[u] = c < a.chunks ? a.counts[c * a.groups + g] : 0;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          all += n[u];
          before += c0 + u * parts < chunk ? n[u] : 0;
        }
        atomicAdd(base + g, all);                             // whole numbers: their order changes nothing
        atomicAdd(mine + g, before);
      }
    }
    __syncthreads();
    if (tid < 32) {
      constexpr int kEach = kSumGroups / 32;
      int v[kEach], sum = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        v[i] = tid * kEach + i < a.groups ? base[tid * kEach + i] : 0;
        sum += v[i];
      }
      int run = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(~0u, run, o);
        if (tid >= o) run += x;
      }
      int before = run - sum;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = tid * kEach + i;
        if (at < a.groups) {
          base[at] = before + mine[at];
          if (chunk == 0) a.offsets[at] = before;
        }
        before += v[i];
      }
      if (tid == 31) {
        base[a.groups] = run;
        if (chunk == 0) a.offsets[a.groups] = run;
      }
    }
  } else {
    wait_for_previous();
    if (e0 + tid < e1) next = a.place[e0 + tid];
    for (int g = tid; g < a.groups; g += blockDim.x) {
      base[g] = a.totals[g];
      mine[g] = a.counts[static_cast<int64_t>(g) * a.chunks + chunk];
    }
    __syncthreads();
    block_scan(base, a.groups, warp_sum);
    if (chunk == 0)
      for (int g = tid; g <= a.groups; g += blockDim.x) a.offsets[g] = base[g];
    __syncthreads();
    for (int g = tid; g < a.groups; g += blockDim.x) base[g] += mine[g];
  }
  __syncthreads();
  const int count = base[a.groups];
  for (int64_t e = e0 + tid; e < e1; e += blockDim.x) {
    int p = next;
    if (e + blockDim.x < e1) next = a.place[e + blockDim.x];
    if (p >= 0) {
      p = (p & ((1 << kRankBits) - 1)) + base[p >> kRankBits];
      a.place[e] = p;
      a.source[p] = static_cast<int>(e);
    }
    if (e >= count) a.source[e] = -1;
  }
}

// ---------------------------------------------------------------- the gradient
struct RouteBwdArgs {
  const void* logits;
  const float *dweight, *weight, *lse;
  const int* expert;
  void* out;
  int64_t rows, ld, out_ld;
  int experts, k;
  bool all;
};

// L lanes a row, at least as many as it has chosen ones, whose lanes write theirs after the row's others.  R of a lane's
// logits are loaded before the first use.
template <typename T, int L, bool ALL>
__global__ void __launch_bounds__(kBackWarps * 32) k_route_backward(const __grid_constant__ RouteBwdArgs a) {
  constexpr int R = 8;
  const int lane = threadIdx.x & 31, l = lane % L;
  constexpr uint32_t kLanes = L == 32 ? ~0u : (1u << L) - 1;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kBackWarps * (32 / L);
  for (int64_t r0 = (blockIdx.x * static_cast<int64_t>(kBackWarps) + (threadIdx.x >> 5)) * (32 / L); r0 < a.rows; r0 += step) {
    const bool mine = r0 + lane / L < a.rows;
    const int64_t row = mine ? r0 + lane / L : r0;           // lanes without a row repeat the first's
    const T* z = ALL ? static_cast<const T*>(a.logits) + row * a.ld : nullptr;
    T* out = static_cast<T*>(a.out) + row * a.out_ld;
    int i = -1;
    float w = 0.0f, dw = 0.0f, lse = 0.0f;
    if (l < a.k) {
      i = a.expert[row * a.k + l];
      w = a.weight[row * a.k + l];
      dw = a.dweight[row * a.k + l];
    }
    T x[R];
    if constexpr (ALL) {
      lse = a.lse[row];
#pragma unroll
      for (int u = 0; u < R; ++u)
        if (u * L + l < a.experts) x[u] = z[u * L + l];
    }
    if (i < 0 || i >= a.experts) i = -1;
    float zi = -INFINITY;
    if (ALL && i >= 0) zi = Elem<T>::up(z[i]);
    const bool bad = (__ballot_sync(~0u, w != w) >> (lane - l) & kLanes) != 0;
    float g = i >= 0 ? w * dw : 0.0f;
    const float s = lanes_sum<L>(g);
    // an expert that is named twice has the sum of both
    int before = 0;
    for (int j = 0; j < a.k; ++j) {
      const int other = __shfl_sync(~0u, i, j, L);           // by all lanes
      before += j < l && other == i;
    }
    if (__any_sync(~0u, i >= 0 && before)) {
      float g2 = 0.0f, w2 = 0.0f;
      for (int j = 0; j < a.k; ++j) {
        const float gj = __shfl_sync(~0u, g, j, L), wj = __shfl_sync(~0u, w, j, L);
        if (__shfl_sync(~0u, i, j, L) == i) {
          g2 += gj;
          w2 += wj;
        }
      }
      g = g2;
      w = w2;
    }
    if constexpr (ALL) {
      if (lse == -INFINITY) lse = INFINITY;                  // nothing allowed: every p is 0
      auto p = [&](float v) { return v > kNone<T> ? exp2_fast((v - lse) * kLog2e) : v == v ? 0.0f : v; };
      for (int j0 = 0; j0 < a.experts; j0 += R * L) {
        if (j0 > 0) {
#pragma unroll
          for (int u = 0; u < R; ++u)
            if (j0 + u * L + l < a.experts) x[u] = z[j0 + u * L + l];
        }
#pragma unroll
        for (int u = 0; u < R; ++u)
          if (j0 + u * L + l < a.experts && mine) out[j0 + u * L + l] = Elem<T>::down(bad ? NAN : -p(Elem<T>::up(x[u])) * s);
      }
      __syncwarp();
      if (i >= 0 && mine) out[i] = Elem<T>::down(bad ? NAN : fmaf(-p(zi), s, g));
    } else {
      if (mine)
        for (int j = l; j < a.experts; j += L) out[j] = Elem<T>::down(bad ? NAN : 0.0f);
      __syncwarp();
      if (i >= 0 && mine) out[i] = Elem<T>::down(bad ? NAN : fmaf(-w, s, g));
    }
  }
}

// ---------------------------------------------------------------- launches
// Units (rows) of a sort's chunk: one for each SM, of a warp's rows at least, more chunks where their ranks would not fit.
int64_t chunk_units(int64_t units, int64_t entries_each) {
  const int64_t per = std::max<int64_t>((units + kCtas - 1) / kCtas, 32);
  return std::min(per, kMaxChunk / entries_each);
}
int64_t workspace_ints(int64_t entries, int unit, int groups) {
  const int64_t units = entries / unit, per = chunk_units(units, unit);
  return (static_cast<int64_t>(groups)) * ((units + per - 1) / per) + groups;
}
// The entries that one CTA sorts by itself, a warp a row: 8 rows of 64 experts 4.3 us, 32 rows about as long as two kernels; 128 rows
// would take 11.1 us, by two kernels 6.1.
constexpr int64_t kOneRows = 32, kOneEntries = 1024;

size_t sort_smem(int warps, int groups, int64_t per) {
  return sizeof(int) * (static_cast<size_t>(warps) * groups + groups + 1 + (per <= kStaged ? per : 0));
}

// With few groups the places' kernel adds up the counts, else a third one.  A route of 8 chosen fp32 so and with three kernels: 1000
// rows of 64 experts 8.7 and 9.5 us, 16384 of 128 14.4 and 15.4, of 200 19.2 both, of 1024 46.7 and 36.3.
cudaError_t end_sort(const SortArgs& a, cudaStream_t s) {
  const unsigned chunks = static_cast<unsigned>(a.chunks);
  if (a.c_step > 1) return launch_early(k_place<true>, chunks, kWarps * 32, 0, s, a);
  const cudaError_t e = launch_early(k_chunks, (a.groups + kBackWarps - 1) / kBackWarps, kBackWarps * 32, 0, s, a);
  if (e != cudaSuccess) return e;
  return launch_early(k_place<false>, chunks, kWarps * 32, 0, s, a);
}

template <typename T, int L, int R, bool ONE>
cudaError_t route_rows(const RouteArgs& a, cudaStream_t s) {
  static bool ok[kMaxDevices];
  const int warps = ONE ? static_cast<int>(std::min<int64_t>(a.rows, kRouteWarps<L, R>)) : kRouteWarps<L, R>;
  const size_t smem = sort_smem(warps, a.sort.groups, a.sort.per);
  const auto kernel = k_route<T, L, R, ONE>;
  cudaError_t e = allow_smem(kernel, 200 << 10, ok);
  if (e != cudaSuccess) return e;
  kernel<<<static_cast<unsigned>(a.sort.chunks), warps * 32, smem, s>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess || ONE) return e;
  return end_sort(a.sort, s);
}

template <typename T>
cudaError_t route_type(const RouteArgs& a, bool one, cudaStream_t s) {
  if (one) {                                                  // a warp a row: few rows, whose latency counts
    if (a.experts <= 64) return route_rows<T, 32, 2, true>(a, s);
    if (a.experts <= 256) return route_rows<T, 32, 8, true>(a, s);
    return route_rows<T, 32, 32, true>(a, s);
  }
  if (a.k <= 8 && a.experts <= 32) return route_rows<T, 8, 4, false>(a, s);
  if (a.k <= 8 && a.experts <= 64) return route_rows<T, 8, 8, false>(a, s);
  if (a.k <= 8 && a.experts <= 128) return route_rows<T, 8, 16, false>(a, s);
  if (a.k <= 16 && a.experts <= 32) return route_rows<T, 16, 2, false>(a, s);
  if (a.k <= 16 && a.experts <= 128) return route_rows<T, 16, 8, false>(a, s);
  if (a.k <= 16 && a.experts <= 256) return route_rows<T, 16, 16, false>(a, s);
  if (a.experts <= 128) return route_rows<T, 32, 4, false>(a, s);
  if (a.experts <= 512) return route_rows<T, 32, 16, false>(a, s);
  return route_rows<T, 32, 32, false>(a, s);
}

template <typename T, int L>
cudaError_t backward_rows(const RouteBwdArgs& a, cudaStream_t s) {
  const int64_t per = kBackWarps * (32 / L), ctas = std::min<int64_t>((a.rows + per - 1) / per, 152 * 8 * 8);
  const auto kernel = a.all ? k_route_backward<T, L, true> : k_route_backward<T, L, false>;
  kernel<<<static_cast<unsigned>(ctas), kBackWarps * 32, 0, s>>>(a);
  return cudaGetLastError();
}
template <typename T>
cudaError_t backward_type(const RouteBwdArgs& a, cudaStream_t s) {
  if (a.k <= 8 && a.experts <= 128) return backward_rows<T, 8>(a, s);
  if (a.k <= 16 && a.experts <= 256) return backward_rows<T, 16>(a, s);
  return backward_rows<T, 32>(a, s);
}

bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// Fills in a sort's chunks; false where the workspace is too small.
bool plan_sort(SortArgs& a, int unit, bool one, void* ws, int64_t bytes) {
  const int64_t units = a.entries / unit, per = one ? units : chunk_units(units, unit);
  a.per = per * unit;
  a.chunks = static_cast<int>((units + per - 1) / per);
  if (one) return true;
  const int64_t need = sizeof(int) * (static_cast<int64_t>(a.groups) * a.chunks + a.groups);
  if (!ws || bytes < need) return false;
  a.counts = static_cast<int*>(ws);
  a.totals = a.counts + static_cast<int64_t>(a.groups) * a.chunks;
  // (one group: the strides are the same)
  const bool sum = a.groups > 1 && a.groups <= kSumGroups && a.chunks <= 2 * kCtas;
  a.g_step = sum ? 1 : a.chunks;
  a.c_step = sum ? a.groups : 1;
  return true;
}
bool one_cta(int64_t units, int64_t entries) { return units <= kOneRows && entries <= kOneEntries; }

// offsets[0 .. groups] = 0 where there are no rows
cudaError_t no_entries(int* offsets, int groups, cudaStream_t s) {
  return cudaMemsetAsync(offsets, 0, sizeof(int) * (groups + 1), s);
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_sort_workspace(int64_t rows, int per_row, int groups, int64_t* bytes) {
  if (!bytes || rows < 0 || per_row < 1 || groups < 1) return HA_EINVAL;
  if (groups > kMaxGroups || per_row > kMaxChosen || rows > 0x7FFFFFFF / per_row) return HA_EUNSUPPORTED;
  *bytes = one_cta(rows, rows * per_row) ? 0 : sizeof(int) * workspace_ints(rows * per_row, per_row, groups);
  return HA_OK;
}

extern "C" int hier_avg_route(const void* logits_dev, int type, int64_t rows, int experts, int64_t ld, int k,
                              int over_all, const int32_t* learners_dev, int learners, int32_t* expert_dev,
                              float* weight_dev, float* lse_dev, int32_t* offsets_dev, int32_t* place_dev,
                              int32_t* source_dev, void* workspace_dev, int64_t workspace_bytes, void* stream) {
  if (!type_ok(type) || rows < 0 || experts < 1 || ld < experts || k < 1 || k > experts || workspace_bytes < 0 ||
      (learners_dev ? learners < 1 : learners != 0) || misaligned(logits_dev, type_size(type)) ||
      misaligned(workspace_dev, 4) || !offsets_dev)
    return HA_EINVAL;
  if (k > kMaxChosen || experts > kMaxExperts ||
      static_cast<int64_t>(experts) * std::max(learners, 1) > kMaxGroups || rows > 0x7FFFFFFF / k)
    return HA_EUNSUPPORTED;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int groups = experts * std::max(learners, 1);
  if (rows == 0) return no_entries(offsets_dev, groups, s) == cudaSuccess ? HA_OK : HA_ECUDA;
  if (!logits_dev || !expert_dev || !weight_dev || !lse_dev || !place_dev || !source_dev) return HA_EINVAL;
  RouteArgs a = {logits_dev, rows, ld, learners_dev, learners, experts, k, over_all != 0, expert_dev, weight_dev, lse_dev,
                 {offsets_dev, place_dev, source_dev, nullptr, nullptr, rows * k, 0, groups, 0}};
  const bool one = one_cta(rows, rows * k);
  if (!plan_sort(a.sort, k, one, workspace_dev, workspace_bytes)) return HA_ENOMEM;
  const cudaError_t e = type == HA_TYPE_FP32   ? route_type<float>(a, one, s)
                        : type == HA_TYPE_BF16 ? route_type<__nv_bfloat16>(a, one, s)
                                               : route_type<__half>(a, one, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}

extern "C" int hier_avg_sort_by_group(const int32_t* group_dev, int64_t rows, int per_row, int groups,
                                      int32_t* offsets_dev, int32_t* place_dev, int32_t* source_dev,
                                      void* workspace_dev, int64_t workspace_bytes, void* stream) {
  if (rows < 0 || per_row < 1 || groups < 1 || workspace_bytes < 0 || misaligned(workspace_dev, 4) || !offsets_dev)
    return HA_EINVAL;
  if (groups > kMaxGroups || per_row > kMaxChosen || rows > 0x7FFFFFFF / per_row) return HA_EUNSUPPORTED;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) return no_entries(offsets_dev, groups, s) == cudaSuccess ? HA_OK : HA_ECUDA;
  if (!group_dev || !place_dev || !source_dev) return HA_EINVAL;
  SortArgs a = {offsets_dev, place_dev, source_dev, nullptr, nullptr, rows * per_row, 0, groups, 0};
  const bool one = one_cta(rows, rows * per_row);
  if (!plan_sort(a, per_row, one, workspace_dev, workspace_bytes)) return HA_ENOMEM;
  const int warps = one ? static_cast<int>(std::min<int64_t>((a.entries + 31) / 32, kWarps)) : kWarps;
  static bool one_ok[kMaxDevices], ok[kMaxDevices];
  const auto kernel = one ? k_group<true> : k_group<false>;
  cudaError_t e = allow_smem(kernel, 200 << 10, one ? one_ok : ok);
  if (e == cudaSuccess) {
    kernel<<<static_cast<unsigned>(a.chunks), warps * 32, sort_smem(warps, groups, a.per), s>>>(group_dev, a);
    e = cudaGetLastError();
  }
  if (e == cudaSuccess && !one) e = end_sort(a, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}

extern "C" int hier_avg_route_backward(const float* dweight_dev, const void* logits_dev, int type, int64_t rows,
                                       int experts, int64_t ld, int k, int over_all, const int32_t* expert_dev,
                                       const float* weight_dev, const float* lse_dev, void* dlogits_dev,
                                       int64_t dlogits_ld, void* stream) {
  if (!type_ok(type) || rows < 0 || experts < 1 || k < 1 || k > experts || dlogits_ld < experts ||
      misaligned(dlogits_dev, type_size(type)))
    return HA_EINVAL;
  if (over_all && (ld < experts || misaligned(logits_dev, type_size(type)))) return HA_EINVAL;
  if (k > kMaxChosen || experts > kMaxExperts || rows > 0x7FFFFFFF / k) return HA_EUNSUPPORTED;
  if (rows == 0) return HA_OK;
  if (!dweight_dev || !expert_dev || !weight_dev || !dlogits_dev || (over_all && (!logits_dev || !lse_dev))) return HA_EINVAL;
  RouteBwdArgs a = {logits_dev, dweight_dev, weight_dev, lse_dev, expert_dev, dlogits_dev, rows, ld, dlogits_ld,
                    experts, k, over_all != 0};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = type == HA_TYPE_FP32   ? backward_type<float>(a, s)
                        : type == HA_TYPE_BF16 ? backward_type<__nv_bfloat16>(a, s)
                                               : backward_type<__half>(a, s);
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}
