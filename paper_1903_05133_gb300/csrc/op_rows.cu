// Rows to their groups and back.  Token t has k entries; entry (t, j) stands at row place[t, j] of the
// sorted rows (-1: nowhere).
//
//   dispatch           xs[place[t, j]] = x[t]; zero for the rows that no entry has
//   dispatch_backward  dx[t] = sum over j of dxs[place[t, j]]
//   combine            out[t] = sum over j of w[t, j] y[place[t, j]]
//   combine_backward   dy[place[t, j]] = w[t, j] dout[t],  dw[t, j] = <dout[t], y[place[t, j]]>
//
// All are bound by the bytes of the sorted rows.  The work goes by tokens: what belongs to a token is
// read once, and its entries' rows, which nobody else has, by 16 bytes a thread with as many loads in
// flight as a token has entries.  Sums are in fp32, in the order of j.
#include <algorithm>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 8;                // entries of a token whose loads are in flight together

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
  int lanes;                              // threads of an item
  int slices;                             // items of a token
};

// V elements at once, or one where rows are not aligned.
template <typename T, int V> struct Part {
  float v[V];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V == 1) {
      v[0] = Elem<T>::up(*p);
    } else if constexpr (V == kVec<T>) {
      unpack<T>(*reinterpret_cast<const uint4*>(p), v);
    } else {                              // fp32 beside a 16-bit type's eight
      unpack<T>(reinterpret_cast<const uint4*>(p)[0], v);
      unpack<T>(reinterpret_cast<const uint4*>(p)[1], v + 4);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (V == 1) {
      *p = Elem<T>::down(v[0]);
    } else if constexpr (V == kVec<T>) {
      *reinterpret_cast<uint4*>(p) = pack<T>(v);
    } else {
      reinterpret_cast<uint4*>(p)[0] = pack<T>(v);
      reinterpret_cast<uint4*>(p)[1] = pack<T>(v + 4);
    }
  }
};

// An entry's row, or -1.
__device__ __forceinline__ int64_t place_of(const RowArgs& a, int64_t entry) {
  const int p = a.place[entry];
  return p >= 0 && p < a.entries ? p : -1;
}

// The item's columns: part i of each row for i in [lane, parts) by steps, of a token's slice.
struct Item {
  int64_t token;
  int first, step, parts;
};
template <int V>
__device__ __forceinline__ Item item_of(const RowArgs& a) {
  const int64_t item = blockIdx.x * static_cast<int64_t>(kThreads / a.lanes) + threadIdx.x / a.lanes;
  const int parts = (a.width + V - 1) / V;
  return {item / a.slices, static_cast<int>(item % a.slices) * a.lanes + static_cast<int>(threadIdx.x) % a.lanes,
          a.slices * a.lanes, parts};
}

// A row's last part may be short: its elements are then taken one by one.
template <int V, typename F, typename G>
__device__ __forceinline__ void each_part(const Item& it, int width, F whole, G single) {
  for (int i = it.first; i < it.parts; i += it.step) {
    const int c = i * V;
    if (c + V <= width) whole(c);
    else
      for (int e = c; e < width; ++e) single(e);
  }
}

template <typename T, int V>
__device__ __forceinline__ void dispatch_at(const RowArgs& a, int64_t token, int c) {
  Part<T, V> x, none;
#pragma unroll
  for (int e = 0; e < V; ++e) none.v[e] = 0.0f;
  x.load(static_cast<const T*>(a.token) + token * a.token_ld + c);
  T* out = static_cast<T*>(a.out_sorted) + c;
  const int64_t count = *a.count;
  for (int j = 0; j < a.k; ++j) {
    const int64_t e = token * a.k + j, p = place_of(a, e);
    if (p >= 0) x.store(out + p * a.out_sorted_ld);
    if (e >= count) none.store(out + e * a.out_sorted_ld);
  }
}
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) k_dispatch(const __grid_constant__ RowArgs a) {
  const Item it = item_of<V>(a);
  if (it.token >= a.tokens) return;
  each_part<V>(it, a.width, [&](int c) { dispatch_at<T, V>(a, it.token, c); },
               [&](int c) { dispatch_at<T, 1>(a, it.token, c); });
}

// out[t] = sum of w y; without weights their sum.
template <typename T, typename O, int V, bool WEIGHTS>
__device__ __forceinline__ void combine_at(const RowArgs& a, int64_t token, int c) {
  const T* rows = static_cast<const T*>(a.sorted) + c;
  Part<O, V> sum;
#pragma unroll
  for (int e = 0; e < V; ++e) sum.v[e] = 0.0f;
  for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
    Part<T, V> y[kAtOnce];
    float w[kAtOnce];
    bool has[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int64_t p = j0 + u < a.k ? place_of(a, token * a.k + j0 + u) : -1;
      has[u] = p >= 0;
      if (has[u]) {
        y[u].load(rows + p * a.sorted_ld);
        w[u] = WEIGHTS ? a.weight[token * a.k + j0 + u] : 1.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (has[u]) {
#pragma unroll
        for (int e = 0; e < V; ++e) sum.v[e] = WEIGHTS ? fmaf(w[u], y[u].v[e], sum.v[e]) : sum.v[e] + y[u].v[e];
      }
  }
  sum.store(static_cast<O*>(a.out_token) + token * a.out_token_ld + c);
}
template <typename T, typename O, int V, bool WEIGHTS>
__global__ void __launch_bounds__(kThreads) k_combine(const __grid_constant__ RowArgs a) {
  const Item it = item_of<V>(a);
  if (it.token >= a.tokens) return;
  each_part<V>(it, a.width, [&](int c) { combine_at<T, O, V, WEIGHTS>(a, it.token, c); },
               [&](int c) { combine_at<T, O, 1, WEIGHTS>(a, it.token, c); });
}

// A CTA a token (or a warp, a.lanes = 32): the weights' gradients are sums over the whole row.
template <typename T, typename O, int V>
__device__ __forceinline__ void combine_backward_at(const RowArgs& a, int64_t token, int j0, int c, const int64_t* p,
                                                    const float* w, float* dot) {
  Part<O, V> d;
  d.load(static_cast<const O*>(a.token) + token * a.token_ld + c);
  Part<T, V> y[kAtOnce];
#pragma unroll
  for (int u = 0; u < kAtOnce; ++u)
    if (p[u] >= 0) y[u].load(static_cast<const T*>(a.sorted) + p[u] * a.sorted_ld + c);
#pragma unroll
  for (int u = 0; u < kAtOnce; ++u)
    if (p[u] >= 0) {
      Part<T, V> dy;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dot[u] = fmaf(d.v[e], y[u].v[e], dot[u]);
        dy.v[e] = w[u] * d.v[e];
      }
      dy.store(static_cast<T*>(a.out_sorted) + p[u] * a.out_sorted_ld + c);
    }
}
template <typename T, typename O, int V>
__global__ void __launch_bounds__(kThreads) k_combine_backward(const __grid_constant__ RowArgs a) {
  __shared__ float part[kThreads / 32][kAtOnce];
  const Item it = item_of<V>(a);
  const bool cta = a.lanes == kThreads;
  if (it.token >= a.tokens) return;                         // whole warps, or whole CTAs
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t count = *a.count;
  for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
    int64_t p[kAtOnce];
    float w[kAtOnce], dot[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int64_t e = it.token * a.k + j0 + u;
      p[u] = j0 + u < a.k ? place_of(a, e) : -1;
      w[u] = j0 + u < a.k ? a.weight[e] : 0.0f;
      dot[u] = 0.0f;
    }
    each_part<V>(it, a.width, [&](int c) { combine_backward_at<T, O, V>(a, it.token, j0, c, p, w, dot); },
                 [&](int c) { combine_backward_at<T, O, 1>(a, it.token, j0, c, p, w, dot); });
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot[u] += __shfl_xor_sync(~0u, dot[u], o);
    }
    if (cta) {
      if (lane == 0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) part[warp][u] = dot[u];
      }
      __syncthreads();
      if (threadIdx.x < kAtOnce && j0 + threadIdx.x < a.k) {
        float s = 0.0f;
        for (int q = 0; q < kThreads / 32; ++q) s += part[q][threadIdx.x];
        a.dweight[it.token * a.k + j0 + threadIdx.x] = s;
      }
      __syncthreads();
    } else if (lane == 0) {
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (j0 + u < a.k) a.dweight[it.token * a.k + j0 + u] = dot[u];
    }
  }
  // the rows that no entry has
  for (int64_t e = max(count, it.token * a.k); e < (it.token + 1) * a.k; ++e) {
    T* dy = static_cast<T*>(a.out_sorted) + e * a.out_sorted_ld;
    each_part<V>(it, a.width, [&](int c) {
      Part<T, V> none;
#pragma unroll
      for (int x = 0; x < V; ++x) none.v[x] = 0.0f;
      none.store(dy + c);
    }, [&](int c) { dy[c] = Elem<T>::down(0.0f); });
  }
}

// ---------------------------------------------------------------- launches
// A pointer and a stride of rows that allow 16 bytes at a time.
bool wide(const void* p, int64_t ld, int type) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld) * type_size(type)) & 15) == 0;
}
int64_t parts_of(int width, int v) { return (width + v - 1) / v; }

// Threads of an item: no more than a row has parts, a power of two.
int lanes_for(int64_t parts, int least) {
  int lanes = least;
  while (lanes < kThreads && lanes < parts) lanes *= 2;
  return lanes;
}
// A part a thread: items of at most a CTA, as many as a row takes.
cudaError_t plan_flat(RowArgs& a, int v, unsigned& grid) {
  const int64_t parts = parts_of(a.width, v);
  a.lanes = lanes_for(parts, 1);
  a.slices = static_cast<int>((parts + a.lanes - 1) / a.lanes);
  const int64_t per = kThreads / a.lanes, ctas = (a.tokens * a.slices + per - 1) / per;
  grid = static_cast<unsigned>(ctas);
  return ctas > 0x7FFFFFFF ? cudaErrorInvalidConfiguration : cudaSuccess;
}

template <typename T>
cudaError_t dispatch_type(RowArgs a, bool vec, cudaStream_t s) {
  unsigned grid;
  const cudaError_t e = plan_flat(a, vec ? kVec<T> : 1, grid);
  if (e != cudaSuccess) return e;
  if (vec) k_dispatch<T, kVec<T>><<<grid, kThreads, 0, s>>>(a);
  else k_dispatch<T, 1><<<grid, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T, typename O>
cudaError_t combine_type(RowArgs a, bool vec, cudaStream_t s) {
  unsigned grid;
  const cudaError_t e = plan_flat(a, vec ? kVec<T> : 1, grid);
  if (e != cudaSuccess) return e;
  if (a.weight) {
    if (vec) k_combine<T, O, kVec<T>, true><<<grid, kThreads, 0, s>>>(a);
    else k_combine<T, O, 1, true><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (vec) k_combine<T, O, kVec<T>, false><<<grid, kThreads, 0, s>>>(a);
    else k_combine<T, O, 1, false><<<grid, kThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

template <typename T, typename O>
cudaError_t combine_backward_type(RowArgs a, bool vec, cudaStream_t s) {
  a.lanes = parts_of(a.width, vec ? kVec<T> : 1) <= 128 ? 32 : kThreads;
  a.slices = 1;
  const int64_t per = kThreads / a.lanes, ctas = (a.tokens + per - 1) / per;
  if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
  if (vec) k_combine_backward<T, O, kVec<T>><<<static_cast<unsigned>(ctas), kThreads, 0, s>>>(a);
  else k_combine_backward<T, O, 1><<<static_cast<unsigned>(ctas), kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

int shape_status(int type, int64_t rows, int width, int k) {
  if (!type_ok(type) || rows < 0 || width < 1 || k < 1) return HA_EINVAL;
  return rows > 0x7FFFFFFF / k ? HA_EUNSUPPORTED : HA_OK;
}
bool rows_ok(const void* p, int64_t ld, int width, int type) {
  return ld >= width && reinterpret_cast<uintptr_t>(p) % type_size(type) == 0;
}
int status(cudaError_t e) { return e == cudaSuccess ? HA_OK : HA_ECUDA; }

int combine_any(RowArgs a, int type, int out_type, cudaStream_t s) {
  const bool vec = wide(a.sorted, a.sorted_ld, type) && wide(a.out_token, a.out_token_ld, out_type);
  if (type == HA_TYPE_FP32) return status(combine_type<float, float>(a, vec, s));
  if (type == HA_TYPE_BF16)
    return status(out_type == type ? combine_type<__nv_bfloat16, __nv_bfloat16>(a, vec, s)
                                   : combine_type<__nv_bfloat16, float>(a, vec, s));
  return status(out_type == type ? combine_type<__half, __half>(a, vec, s) : combine_type<__half, float>(a, vec, s));
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
