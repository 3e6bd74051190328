// Rows to their groups and back.  Token t has k entries; entry (t, j) stands at row place[t, j] of the
// sorted rows (-1: nowhere).
//
//   dispatch           xs[place[t, j]] = x[t]; zero for the rows that no entry has
//   dispatch_backward  dx[t] = sum over j of dxs[place[t, j]]
//   combine            out[t] = sum over j of w[t, j] y[place[t, j]], 0 for the y of no place
//   combine_backward   dy[place[t, j]] = w[t, j] dout[t],  dw[t, j] = <dout[t], y[place[t, j]]>
//
// All are bound by the bytes of the sorted rows.  The work goes by tokens: what belongs to a token is
// read once, and its entries' rows, which nobody else has, by 16 bytes a thread with as many loads in
// flight as a token has entries.  Sums are in fp32, in the order of j.  8192 tokens of 4 entries of 4096 bf16:
// dispatch 51.3 us, combine 52.5 (336 MB: 6.5 and 6.4 TB/s, the copy's rate is 6.75), its gradient 89.6 (604 MB, 6.7).
#include <algorithm>
#include <climits>
#include <type_traits>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kThreads = 256;
// Parts of a row that a thread has in flight at a time, for 16-byte parts and for single elements.  8192 tokens of 4 entries of
// 4096 bf16: combine takes 55.1 us with 2 parts (four CTAs an SM; 76 with five, whose registers spill), 57.1 with one and 53.5
// with four, which fewer tokens do not fill the GPU with.  Rows that are read once do not stay in L2 (58.1 where they do).  (52.5 with
// two since the weights' loads do not wait for the places.)
constexpr int kWide = 2, kSingle = 8;
constexpr int kSingleSums = 4;            // of combine's gradient: 3001 tokens of 4 odd entries of 1111 fp32 25 us, 33 with 8

struct RowArgs {
  const void* token;                      // x or dout
  const void* sorted;                     // y or dxs
  const int* place;
  const float* weight;
  const int* count;                       // entries that have a place: offsets[groups]
  void* out_token;
  void* out_sorted;
  float* dweight;
  int64_t tokens, entries, token_ld, sorted_ld, out_token_ld, out_sorted_ld;
  int k, width;
  int lanes;                              // threads of a token
};

// V elements of a row as they are held in memory: 16 bytes, or fp32 beside a 16-bit type's eight, or one
// element where rows are not aligned.  Rows are widened when they are added, so that the loads in flight take
// no more registers than their bytes.
template <typename T, int V> struct Part {
  static constexpr int kWords = V == 1 ? 1 : V / kVec<T>;
  uint4 w[kWords];
  T one;
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V == 1) {
      one = *p;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
  }
  __device__ __forceinline__ void load_once(const T* p) {   // what nobody reads again soon
    if constexpr (V == 1) {
      one = *p;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    }
  }
  __device__ __forceinline__ void clear() {
    if constexpr (V == 1) {
      one = Elem<T>::down(0.0f);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (V == 1) {
      *p = one;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
    }
  }
  __device__ __forceinline__ void up(float* v) const {
    if constexpr (V == 1) {
      v[0] = Elem<T>::up(one);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) unpack<T>(w[i], v + i * kVec<T>);
    }
  }
  __device__ __forceinline__ void down(const float* v) {
    if constexpr (V == 1) {
      one = Elem<T>::down(v[0]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = pack<T>(v + i * kVec<T>);
    }
  }
};

// An entry's row, or -1.
__device__ __forceinline__ int64_t place_of(const RowArgs& a, int64_t entry) {
  const int p = a.place[entry];
  return p >= 0 && p < a.entries ? p : -1;
}

// A thread's token and its first part of the rows; the next is a.lanes parts on.
struct Item {
  int64_t token;
  int first;
};
__device__ __forceinline__ Item item_of(const RowArgs& a) {
  const int64_t at = blockIdx.x * static_cast<int64_t>(kThreads);
  if (a.entries * a.lanes <= 0x7FFFFFFF - kThreads) {       // a division of 32 bits
    const int i = static_cast<int>(at) + static_cast<int>(threadIdx.x);
    return {i / a.lanes, i % a.lanes};
  }
  const int64_t i = at + threadIdx.x;
  return {i / a.lanes, static_cast<int>(i % a.lanes)};
}

// f(part) for U parts of a row at a time, `lanes` apart; a row's last elements, which fill no part, go to g one by one.
template <int V, int U, typename F, typename G>
__device__ __forceinline__ void each_part(int first, int lanes, int width, F f, G g) {
  const int parts = width / V;
  for (int i = first; i < parts; i += lanes * U) f(i);
  if constexpr (V > 1)
    for (int c = parts * V + first; c < width; c += lanes) g(c);
}

template <typename T, int V, int U>
__device__ __forceinline__ void dispatch_at(const RowArgs& a, int64_t token, int i, int parts) {
  Part<T, V> x[U], none;
  const T* from = static_cast<const T*>(a.token) + token * a.token_ld;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (i + u * a.lanes < parts) x[u].load(from + (i + u * a.lanes) * V);
  none.clear();
  const int64_t count = *a.count;
  for (int j = 0; j < a.k; ++j) {
    const int64_t e = token * a.k + j, p = place_of(a, e);
    T* out = static_cast<T*>(a.out_sorted);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = (i + u * a.lanes) * V;
      if (i + u * a.lanes >= parts) break;
      if (p >= 0) x[u].store(out + p * a.out_sorted_ld + c);
      if (e >= count) none.store(out + e * a.out_sorted_ld + c);
    }
  }
}
template <typename T, int V, int U>
__global__ void __launch_bounds__(kThreads) k_dispatch(const __grid_constant__ RowArgs a) {
  const Item it = item_of(a);
  if (it.token >= a.tokens) return;
  each_part<V, U>(it.first, a.lanes, a.width, [&](int i) { dispatch_at<T, V, U>(a, it.token, i, a.width / V); },
                  [&](int c) { dispatch_at<T, 1, 1>(a, it.token, c, a.width); });
}

// out[t] = sum of w y; without weights their sum.  AT entries' loads of U parts are in flight together.
template <typename T, typename O, int V, int U, int AT, bool WEIGHTS>
__device__ __forceinline__ void combine_at(const RowArgs& a, int64_t token, int i, int parts) {
  float sum[U][V];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < V; ++e) sum[u][e] = 0.0f;
  for (int j0 = 0; j0 < a.k; j0 += AT) {
    Part<T, V> y[AT][U];
    float w[AT];
#pragma unroll
    for (int q = 0; q < AT; ++q) {
      const int64_t p = j0 + q < a.k ? place_of(a, token * a.k + j0 + q) : -1;
      w[q] = WEIGHTS && j0 + q < a.k ? a.weight[token * a.k + j0 + q] : 0.0f;   // of no place too: a router's NaN shows
      const T* row = static_cast<const T*>(a.sorted) + p * a.sorted_ld;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p >= 0 && i + u * a.lanes < parts) y[q][u].load_once(row + (i + u * a.lanes) * V);
        else y[q][u].clear();
      }
    }
#pragma unroll
    for (int q = 0; q < AT; ++q)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[V];
        y[q][u].up(v);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[u][e] = WEIGHTS ? fmaf(w[q], v[e], sum[u][e]) : sum[u][e] + v[e];
      }
  }
  O* out = static_cast<O*>(a.out_token) + token * a.out_token_ld;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (i + u * a.lanes < parts) {
      Part<O, V> o;
      o.down(sum[u]);
      o.store(out + (i + u * a.lanes) * V);
    }
}
template <typename T, typename O, int V, int U, int AT, bool WEIGHTS>
__global__ void __launch_bounds__(kThreads, 4) k_combine(const __grid_constant__ RowArgs a) {
  const Item it = item_of(a);
  if (it.token >= a.tokens) return;
  each_part<V, U>(it.first, a.lanes, a.width, [&](int i) { combine_at<T, O, V, U, AT, WEIGHTS>(a, it.token, i, a.width / V); },
                  [&](int c) { combine_at<T, O, 1, 1, AT, WEIGHTS>(a, it.token, c, a.width); });
}

// The sum over a group of lanes, a power of two; a CTA's over each of its warps.
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  if (lanes >= 32) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  } else {
    for (int o = lanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  }
  return x;
}

// A CTA, a warp or some lanes a token, a power of two: the weights' gradients are sums over the whole row.
template <typename T, typename O, int V, int U, int AT>
__device__ __forceinline__ void combine_backward_at(const RowArgs& a, int64_t token, int i, int parts, int lanes, const int64_t* p,
                                                    const float* w, float* dot) {
  Part<O, V> d[U];
  Part<T, V> y[AT][U];
  const O* from = static_cast<const O*>(a.token) + token * a.token_ld;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (i + u * lanes < parts) d[u].load(from + (i + u * lanes) * V);
    else d[u].clear();
  }
#pragma unroll
  for (int q = 0; q < AT; ++q)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p[q] >= 0 && i + u * lanes < parts)
        y[q][u].load(static_cast<const T*>(a.sorted) + p[q] * a.sorted_ld + (i + u * lanes) * V);
      else
        y[q][u].clear();
    }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float dv[V];
    d[u].up(dv);
#pragma unroll
    for (int q = 0; q < AT; ++q) {
      float v[V];
      y[q][u].up(v);
      if (p[q] < 0) continue;                               // dout may be infinite
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dot[q] = fmaf(dv[e], v[e], dot[q]);
        v[e] = w[q] * dv[e];
      }
      if (i + u * lanes < parts) {
        Part<T, V> dy;
        dy.down(v);
        dy.store(static_cast<T*>(a.out_sorted) + p[q] * a.out_sorted_ld + (i + u * lanes) * V);
      }
    }
  }
}
template <typename T, typename O, int V, int U, int AT, bool CTA>
__global__ void __launch_bounds__(kThreads) k_combine_backward(const __grid_constant__ RowArgs a) {
  __shared__ float part[kThreads / 32][AT];
  const int lanes = CTA ? kThreads : a.lanes;
  const Item it = CTA ? Item{blockIdx.x, static_cast<int>(threadIdx.x)} : item_of(a);
  const bool mine = CTA || it.token < a.tokens;             // all take part in the sums
  const int64_t token = mine ? it.token : 0;
  const int first = it.first, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t count = *a.count;
  for (int j0 = 0; j0 < a.k; j0 += AT) {
    int64_t p[AT];
    float w[AT], dot[AT];
#pragma unroll
    for (int q = 0; q < AT; ++q) {
      const int64_t e = token * a.k + j0 + q;
      p[q] = mine && j0 + q < a.k ? place_of(a, e) : -1;
      w[q] = j0 + q < a.k ? a.weight[e] : 0.0f;
      dot[q] = 0.0f;
    }
    if (mine) each_part<V, U>(first, lanes, a.width,
                    [&](int i) { combine_backward_at<T, O, V, U, AT>(a, token, i, a.width / V, lanes, p, w, dot); },
                    [&](int c) { combine_backward_at<T, O, 1, 1, AT>(a, token, c, a.width, lanes, p, w, dot); });
#pragma unroll
    for (int q = 0; q < AT; ++q) dot[q] = lanes_sum(dot[q], lanes);
    if (CTA) {
      if (lane == 0) {
#pragma unroll
        for (int q = 0; q < AT; ++q) part[warp][q] = dot[q];
      }
      __syncthreads();
      if (threadIdx.x < AT && j0 + threadIdx.x < a.k) {
        float s = 0.0f;
        for (int q = 0; q < kThreads / 32; ++q) s += part[q][threadIdx.x];
        a.dweight[token * a.k + j0 + threadIdx.x] = s;
      }
      __syncthreads();
    } else if (first == 0 && mine) {
#pragma unroll
      for (int q = 0; q < AT; ++q)
        if (j0 + q < a.k) a.dweight[token * a.k + j0 + q] = dot[q];
    }
  }
  // the rows that no entry has
  for (int64_t e = max(count, token * a.k); mine && e < (token + 1) * a.k; ++e) {
    T* dy = static_cast<T*>(a.out_sorted) + e * a.out_sorted_ld;
    each_part<V, 1>(first, lanes, a.width, [&](int i) {
      Part<T, V> none;
      none.clear();
      none.store(dy + i * V);
    }, [&](int c) { dy[c] = Elem<T>::down(0.0f); });
  }
}

// ---------------------------------------------------------------- rows that are not aligned
// 16 bytes from any element on: the two aligned 16 bytes around them, shifted.  The second ones are a neighbour's first, so
// that they come from L1.  What is read beside the element's own bytes is the rows' too: see Aligned::inside.
template <typename T> struct Shifted {
  uint4 a, b;
  uint32_t shift;                         // bytes
  __device__ __forceinline__ void load(const T* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    shift = static_cast<uint32_t>(at & 15);
    const uint4* q = reinterpret_cast<const uint4*>(at - shift);
    a = q[0];
    b = q[1];
  }
  __device__ __forceinline__ void clear() {
    a = b = make_uint4(0, 0, 0, 0);
    shift = 0;
  }
  __device__ __forceinline__ uint4 get() const {
    const bool two = shift & 8, one = shift & 4;
    uint32_t t[6] = {two ? a.z : a.x, two ? a.w : a.y, two ? b.x : a.z, two ? b.y : a.w, two ? b.z : b.x, two ? b.w : b.y};
#pragma unroll
    for (int i = 0; i < 5; ++i) t[i] = one ? t[i + 1] : t[i];
    if constexpr (sizeof(T) == 4) return make_uint4(t[0], t[1], t[2], t[3]);
    const uint32_t bits = 8 * (shift & 3);
    return make_uint4(__funnelshift_r(t[0], t[1], bits), __funnelshift_r(t[1], t[2], bits), __funnelshift_r(t[2], t[3], bits),
                      __funnelshift_r(t[3], t[4], bits));
  }
};

// A row that is written: its elements before the first 16-byte boundary, and the parts of V from there on.
struct Aligned {
  int head, parts;
  // Rows that are read beside it begin or end the memory of all rows (`edge`): there the first and the last part, around
  // which a shifted load reads up to 15 bytes before and 16 behind, are taken element by element.
  template <int V>
  __device__ __forceinline__ void inside(bool edge) {
    if (!edge) return;
    if (parts > 0) head += V;
    parts = max(parts - 2, 0);
  }
};
template <typename O, int V>
__device__ __forceinline__ Aligned aligned(const O* row, int width) {
  const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / static_cast<int>(sizeof(O));
  const int head = min(width, off ? kVec<O> - off : 0);
  return {head, (width - head) / V};
}
// f(part, number of parts) for U parts of a row at a time, `lanes` apart; g(column) for the elements outside of them.
template <int V, int U, typename F, typename G>
__device__ __forceinline__ void each_aligned(Aligned r, int first, int lanes, int width, F f, G g) {
  for (int i = first; i < r.parts; i += lanes * U) f(i);
  for (int c = first; c < r.head; c += lanes) g(c);
  for (int c = r.head + r.parts * V + first; c < width; c += lanes) g(c);
}

// By entries, since the rows of a token's entries are aligned each in its own way.
template <typename T, int U>
__global__ void __launch_bounds__(kThreads) k_dispatch_shifted(const __grid_constant__ RowArgs a) {
  constexpr int V = kVec<T>;
  const Item it = item_of(a);                               // its token is an entry
  if (it.token >= a.entries) return;
  const int64_t p = place_of(a, it.token);
  const T* from = static_cast<const T*>(a.token) + it.token / a.k * a.token_ld;
  if (p >= 0) {
    T* out = static_cast<T*>(a.out_sorted) + p * a.out_sorted_ld;
    Aligned r = aligned<T, V>(out, a.width);
    r.template inside<V>(it.token < a.k || it.token >= a.entries - a.k);
    each_aligned<V, U>(r, it.first, a.lanes, a.width, [&](int i) {
      Shifted<T> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * a.lanes < r.parts) x[u].load(from + r.head + (i + u * a.lanes) * V);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * a.lanes < r.parts) *reinterpret_cast<uint4*>(out + r.head + (i + u * a.lanes) * V) = x[u].get();
    }, [&](int c) { out[c] = from[c]; });
  }
  if (it.token >= *a.count) {
    T* out = static_cast<T*>(a.out_sorted) + it.token * a.out_sorted_ld;
    const Aligned r = aligned<T, V>(out, a.width);
    each_aligned<V, 1>(r, it.first, a.lanes, a.width,
                       [&](int i) { *reinterpret_cast<uint4*>(out + r.head + i * V) = make_uint4(0, 0, 0, 0); },
                       [&](int c) { out[c] = Elem<T>::down(0.0f); });
  }
}

template <typename T, typename O, int U, int AT, bool WEIGHTS>
__global__ void __launch_bounds__(kThreads, 4) k_combine_shifted(const __grid_constant__ RowArgs a) {
  constexpr int V = kVec<T>;
  const Item it = item_of(a);
  if (it.token >= a.tokens) return;
  O* out = static_cast<O*>(a.out_token) + it.token * a.out_token_ld;
  Aligned r = aligned<O, V>(out, a.width);
  bool edge = false;
  for (int j = 0; j < a.k; ++j) {
    const int64_t p = place_of(a, it.token * a.k + j);
    edge = edge || p == 0 || p == a.entries - 1;
  }
  r.template inside<V>(edge);
  each_aligned<V, U>(r, it.first, a.lanes, a.width, [&](int i) {
    float sum[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) sum[u][e] = 0.0f;
    for (int j0 = 0; j0 < a.k; j0 += AT) {
      Shifted<T> y[AT][U];
      float w[AT];
#pragma unroll
      for (int q = 0; q < AT; ++q) {
        const int64_t p = j0 + q < a.k ? place_of(a, it.token * a.k + j0 + q) : -1;
        w[q] = WEIGHTS && j0 + q < a.k ? a.weight[it.token * a.k + j0 + q] : 0.0f;
        const T* row = static_cast<const T*>(a.sorted) + p * a.sorted_ld + r.head;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (p >= 0 && i + u * a.lanes < r.parts) y[q][u].load(row + (i + u * a.lanes) * V);
          else y[q][u].clear();
        }
      }
#pragma unroll
      for (int q = 0; q < AT; ++q)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float v[V];
          unpack<T>(y[q][u].get(), v);
#pragma unroll
          for (int e = 0; e < V; ++e) sum[u][e] = WEIGHTS ? fmaf(w[q], v[e], sum[u][e]) : sum[u][e] + v[e];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * a.lanes < r.parts) {
        Part<O, V> o;
        o.down(sum[u]);
        o.store(out + r.head + (i + u * a.lanes) * V);
      }
  }, [&](int c) { combine_at<T, O, 1, 1, AT, WEIGHTS>(a, it.token, c, a.width); });
}

// Some lanes, a warp or a CTA an entry.
template <typename T, typename O, int U>
__global__ void __launch_bounds__(kThreads, 5) k_combine_backward_shifted(const __grid_constant__ RowArgs a) {
  constexpr int V = kVec<T>, kWords = V / kVec<O>;
  __shared__ float part[kThreads / 32];
  const Item it = item_of(a);                               // its token is an entry
  const bool mine = it.token < a.entries;                   // all take part in the sums
  const int64_t entry = mine ? it.token : 0, p = mine ? place_of(a, entry) : -1;
  const O* d = static_cast<const O*>(a.token) + entry / a.k * a.token_ld;
  float dot = 0.0f;
  if (p >= 0) {
    const float w = a.weight[entry];
    const T* y = static_cast<const T*>(a.sorted) + p * a.sorted_ld;
    T* dy = static_cast<T*>(a.out_sorted) + p * a.out_sorted_ld;
    Aligned r = aligned<T, V>(dy, a.width);
    r.template inside<V>(p == 0 || p == a.entries - 1 || entry < a.k || entry >= a.entries - a.k);
    each_aligned<V, U>(r, it.first, a.lanes, a.width, [&](int i) {
      Shifted<T> ys[U];
      Shifted<O> ds[U][kWords];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = r.head + (i + u * a.lanes) * V;
        if (i + u * a.lanes < r.parts) {
          ys[u].load(y + c);
#pragma unroll
          for (int x = 0; x < kWords; ++x) ds[u][x].load(d + c + x * kVec<O>);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u * a.lanes >= r.parts) break;
        float yv[V], dv[V];
        unpack<T>(ys[u].get(), yv);
#pragma unroll
        for (int x = 0; x < kWords; ++x) unpack<O>(ds[u][x].get(), dv + x * kVec<O>);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dot = fmaf(dv[e], yv[e], dot);
          dv[e] *= w;
        }
        *reinterpret_cast<uint4*>(dy + r.head + (i + u * a.lanes) * V) = pack<T>(dv);
      }
    }, [&](int c) {
      const float dv = Elem<O>::up(d[c]);
      dot = fmaf(dv, Elem<T>::up(y[c]), dot);
      dy[c] = Elem<T>::down(w * dv);
    });
  }
  if (mine && entry >= *a.count) {
    T* dy = static_cast<T*>(a.out_sorted) + entry * a.out_sorted_ld;
    const Aligned r = aligned<T, V>(dy, a.width);
    each_aligned<V, 1>(r, it.first, a.lanes, a.width,
                       [&](int i) { *reinterpret_cast<uint4*>(dy + r.head + i * V) = make_uint4(0, 0, 0, 0); },
                       [&](int c) { dy[c] = Elem<T>::down(0.0f); });
  }
  dot = lanes_sum(dot, a.lanes);
  if (a.lanes == kThreads) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = dot;
    __syncthreads();
    dot = 0.0f;
    for (int q = 0; q < kThreads / 32; ++q) dot += part[q];
  }
  if (mine && it.first == 0) a.dweight[entry] = dot;
}

// ---------------------------------------------------------------- launches
// A pointer and a stride of rows that allow 16 bytes at a time.
bool wide(const void* p, int64_t ld, int type) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld) * type_size(type)) & 15) == 0;
}
// Rows of a 16-bit type of at least this many 16 bytes are read by 16 bytes where they are not aligned.  (Of fp32 a warp's
// single elements are 128 bytes already.)
// 8192 tokens of 4 entries of 4095 bf16 so and by single elements: dispatch 78 and 148 us, its gradient 76 and 118, combine 84 and
// 112, its gradient 117 and 209; 16384 of 65: 7.2 and 7.3, 6.6 and 6.1, 8.1 and 6.1, 9.8 and 23.7.
template <typename T>
bool shifted(const RowArgs& a, int parts) { return sizeof(T) == 2 && a.width >= parts * kVec<T>; }
constexpr int kShiftedParts = 16, kShiftedSums = 4;
// A power of two of lanes for rows of so many parts: a warp at most, and a CTA for long rows where they are few, or longer than
// `most` parts.  Tokens of 4 entries, bf16, a CTA and a warp each: 8192 of 4096 89.9 and 94.7 us, 3001 of 1112 10.1 and 8.4, 100 of
// 4096 3.3 and 10.5; odd entries 8192 x 4 of 4095 143 and 117, 3001 x 4 of 1111 32 and 13, 400 x 4 of 4095 8.9 and 8.8, 100 x 4 4.3 and 7.7.
constexpr int kFewRows = 2000;
int lanes_for(int64_t rows, int parts, int most) {
  if (parts > 128 && (rows < kFewRows || parts > most)) return kThreads;
  int lanes = 1;
  while (lanes < 32 && lanes < parts) lanes *= 2;
  return lanes;
}

// Threads of a token (or an entry): U parts each where rows are long.
cudaError_t plan_flat(RowArgs& a, int64_t items, int v, int u, unsigned& grid) {
  const int parts = std::max(a.width / v, 1);
  a.lanes = (parts + u - 1) / u;
  const int64_t ctas = (items * a.lanes + kThreads - 1) / kThreads;
  grid = static_cast<unsigned>(ctas);
  return ctas > 0x7FFFFFFF ? cudaErrorInvalidConfiguration : cudaSuccess;
}

template <typename T, int V, int U>
cudaError_t launch_dispatch(RowArgs a, cudaStream_t s) {
  unsigned grid;
  const cudaError_t e = plan_flat(a, a.tokens, V, U, grid);
  if (e != cudaSuccess) return e;
  k_dispatch<T, V, U><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}
template <typename T>
cudaError_t dispatch_type(const RowArgs& a, bool vec, cudaStream_t s) {
  if (vec) return launch_dispatch<T, kVec<T>, 1>(a, s);
  if (!shifted<T>(a, kShiftedParts)) return launch_dispatch<T, 1, 4>(a, s);
  if constexpr (sizeof(T) == 2) {
    RowArgs b = a;
    unsigned grid;
    const cudaError_t e = plan_flat(b, b.entries, kVec<T>, 4, grid);
    if (e != cudaSuccess) return e;
    k_dispatch_shifted<T, 4><<<grid, kThreads, 0, s>>>(b);
  }
  return cudaGetLastError();
}

template <typename T, typename O, int V, int U, int AT, bool WEIGHTS>
cudaError_t launch_combine(RowArgs a, cudaStream_t s) {
  unsigned grid;
  const cudaError_t e = plan_flat(a, a.tokens, V, U, grid);
  if (e != cudaSuccess) return e;
  k_combine<T, O, V, U, AT, WEIGHTS><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}
template <typename T, typename O, int U, int AT, bool WEIGHTS>
cudaError_t launch_combine_shifted(RowArgs a, cudaStream_t s) {
  unsigned grid;
  const cudaError_t e = plan_flat(a, a.tokens, kVec<T>, U, grid);
  if (e != cudaSuccess) return e;
  k_combine_shifted<T, O, U, AT, WEIGHTS><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}
template <typename T, typename O, bool WEIGHTS>
cudaError_t combine_type(const RowArgs& a, bool vec, cudaStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (!vec && shifted<T>(a, kShiftedParts)) return launch_combine_shifted<T, O, 2, 2, WEIGHTS>(a, s);
  if (a.k <= 4) return vec ? launch_combine<T, O, kVec<T>, kWide, 4, WEIGHTS>(a, s) : launch_combine<T, O, 1, kSingle, 4, WEIGHTS>(a, s);
  return vec ? launch_combine<T, O, kVec<T>, 1, 8, WEIGHTS>(a, s) : launch_combine<T, O, 1, kSingle / 2, 8, WEIGHTS>(a, s);
}

template <typename T, typename O, int V, int U, int AT>
cudaError_t launch_combine_backward(RowArgs a, cudaStream_t s) {
  a.lanes = lanes_for(a.tokens, std::max(a.width / V, 1), 256);
  const int64_t ctas = (a.tokens * a.lanes + kThreads - 1) / kThreads;
  if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
  const auto kernel = a.lanes == kThreads ? k_combine_backward<T, O, V, U, AT, true> : k_combine_backward<T, O, V, U, AT, false>;
  kernel<<<static_cast<unsigned>(ctas), kThreads, 0, s>>>(a);
  return cudaGetLastError();
}
template <typename T, typename O>
cudaError_t combine_backward_type(const RowArgs& a, bool vec, cudaStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (!vec && shifted<T>(a, kShiftedSums)) {
      RowArgs b = a;
      b.lanes = lanes_for(a.entries, a.width / kVec<T>, INT_MAX);
      const int64_t ctas = (a.entries * b.lanes + kThreads - 1) / kThreads;
      if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
      k_combine_backward_shifted<T, O, 1><<<static_cast<unsigned>(ctas), kThreads, 0, s>>>(b);
      return cudaGetLastError();
    }
  if (a.k <= 4) return vec ? launch_combine_backward<T, O, kVec<T>, 1, 4>(a, s) : launch_combine_backward<T, O, 1, kSingleSums, 4>(a, s);
  return vec ? launch_combine_backward<T, O, kVec<T>, 1, 8>(a, s) : launch_combine_backward<T, O, 1, kSingleSums / 2, 8>(a, s);
}

// A thread's next column, which is up to a row and a share of one on, has to fit 32 bits.
constexpr int kMaxWidth = 1 << 30;
int shape_status(int type, int64_t rows, int width, int k) {
  if (!type_ok(type) || rows < 0 || width < 1 || k < 1) return HA_EINVAL;
  return width > kMaxWidth || rows > 0x7FFFFFFF / k ? HA_EUNSUPPORTED : HA_OK;
}
bool rows_ok(const void* p, int64_t ld, int width, int type) {
  return ld >= width && reinterpret_cast<uintptr_t>(p) % type_size(type) == 0;
}
int status(cudaError_t e) { return e == cudaSuccess ? HA_OK : HA_ECUDA; }

int combine_any(RowArgs a, int type, int out_type, cudaStream_t s) {
  const bool vec = wide(a.sorted, a.sorted_ld, type) && wide(a.out_token, a.out_token_ld, out_type);
  const auto go = [&](auto weights) {
    constexpr bool W = decltype(weights)::value;
    if (type == HA_TYPE_FP32) return combine_type<float, float, W>(a, vec, s);
    if (type == HA_TYPE_BF16)
      return out_type == type ? combine_type<__nv_bfloat16, __nv_bfloat16, W>(a, vec, s) : combine_type<__nv_bfloat16, float, W>(a, vec, s);
    return out_type == type ? combine_type<__half, __half, W>(a, vec, s) : combine_type<__half, float, W>(a, vec, s);
  };
  return status(a.weight ? go(std::true_type()) : go(std::false_type()));
}

}  // namespace
}  // namespace ha

using namespace ha;

extern "C" int hier_avg_dispatch(const void* x_dev, int type, int64_t rows, int width, int64_t x_ld,
                                 const int32_t* place_dev, int per_row, const int32_t* offsets_dev, int groups,
                                 void* xs_dev, int64_t xs_ld, void* stream) {
  if (const int e = shape_status(type, rows, width, per_row)) return e;
  if (!rows_ok(x_dev, x_ld, width, type) || !rows_ok(xs_dev, xs_ld, width, type) || groups < 1) return HA_EINVAL;
  if (rows == 0) return HA_OK;
  if (!x_dev || !place_dev || !offsets_dev || !xs_dev) return HA_EINVAL;
  RowArgs a = {};
  a.token = x_dev;
  a.place = place_dev;
  a.count = offsets_dev + groups;
  a.out_sorted = xs_dev;
  a.tokens = rows;
  a.entries = rows * per_row;
  a.token_ld = x_ld;
  a.out_sorted_ld = xs_ld;
  a.k = per_row;
  a.width = width;
  const bool vec = wide(x_dev, x_ld, type) && wide(xs_dev, xs_ld, type);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return status(type == HA_TYPE_FP32   ? dispatch_type<float>(a, vec, s)
                : type == HA_TYPE_BF16 ? dispatch_type<__nv_bfloat16>(a, vec, s)
                                       : dispatch_type<__half>(a, vec, s));
}

extern "C" int hier_avg_combine(const void* y_dev, int type, int64_t rows, int width, int64_t y_ld,
                                const int32_t* place_dev, int per_row, const float* weight_dev, void* out_dev,
                                int64_t out_ld, int out_type, void* stream) {
  if (const int e = shape_status(type, rows, width, per_row)) return e;
  if ((out_type != type && out_type != HA_TYPE_FP32) || !rows_ok(y_dev, y_ld, width, type) ||
      !rows_ok(out_dev, out_ld, width, out_type))
    return HA_EINVAL;
  if (rows == 0) return HA_OK;
  if (!y_dev || !place_dev || !out_dev) return HA_EINVAL;
  RowArgs a = {};
  a.sorted = y_dev;
  a.place = place_dev;
  a.weight = weight_dev;
  a.out_token = out_dev;
  a.tokens = rows;
  a.entries = rows * per_row;
  a.sorted_ld = y_ld;
  a.out_token_ld = out_ld;
  a.k = per_row;
  a.width = width;
  return combine_any(a, type, out_type, static_cast<cudaStream_t>(stream));
}

extern "C" int hier_avg_combine_backward(const void* dout_dev, int dout_type, int64_t dout_ld, const void* y_dev, int type,
                                         int64_t rows, int width, int64_t y_ld, const int32_t* place_dev, int per_row,
                                         const float* weight_dev, const int32_t* offsets_dev, int groups, void* dy_dev,
                                         int64_t dy_ld, float* dweight_dev, void* stream) {
  if (const int e = shape_status(type, rows, width, per_row)) return e;
  if ((dout_type != type && dout_type != HA_TYPE_FP32) || groups < 1 || !rows_ok(y_dev, y_ld, width, type) ||
      !rows_ok(dout_dev, dout_ld, width, dout_type) || !rows_ok(dy_dev, dy_ld, width, type))
    return HA_EINVAL;
  if (rows == 0) return HA_OK;
  if (!dout_dev || !y_dev || !place_dev || !weight_dev || !offsets_dev || !dy_dev || !dweight_dev) return HA_EINVAL;
  RowArgs a = {};
  a.token = dout_dev;
  a.sorted = y_dev;
  a.place = place_dev;
  a.weight = weight_dev;
  a.count = offsets_dev + groups;
  a.out_sorted = dy_dev;
  a.dweight = dweight_dev;
  a.tokens = rows;
  a.entries = rows * per_row;
  a.token_ld = dout_ld;
  a.sorted_ld = y_ld;
  a.out_sorted_ld = dy_ld;
  a.k = per_row;
  a.width = width;
  const bool vec = wide(dout_dev, dout_ld, dout_type) && wide(y_dev, y_ld, type) && wide(dy_dev, dy_ld, type);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (type == HA_TYPE_FP32) return status(combine_backward_type<float, float>(a, vec, s));
  if (type == HA_TYPE_BF16)
    return status(dout_type == type ? combine_backward_type<__nv_bfloat16, __nv_bfloat16>(a, vec, s)
                                    : combine_backward_type<__nv_bfloat16, float>(a, vec, s));
  return status(dout_type == type ? combine_backward_type<__half, __half>(a, vec, s)
                                  : combine_backward_type<__half, float>(a, vec, s));
}
