// AdamW over many tensors in one launch, states in 32 or 8 bits.
//
//   m <- b1 m + (1 - b1) g          v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Everything is computed in 32 bits; the states are rounded when they are stored.  In 8
// bits m and sqrt(v) are held as e4m3 floats with one fp32 scale for each block of 256
// elements (scale = largest magnitude / 448).  sqrt(v) rather than v, because e4m3 spans
// 2^18 and v the square of that; and sqrt(v) is rounded up or down at random, with
// probabilities that keep its mean: with b2 = 0.999 a step moves sqrt(v) by about 0.05 %,
// which rounding to nearest (steps of 6 to 12 %) would always take back.  The random bits
// come from the element's place and the caller's seed, so a step is reproducible.
#include <cfloat>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <vector>

#include <cuda_fp8.h>

#include "op_common.cuh"

namespace ha {
namespace {

constexpr int kBlock = 256;         // elements that share a scale: one warp, 8 a lane
constexpr int kChunk = 1024;        // elements of one CTA: a block for each warp
constexpr int kThreads = 128;
constexpr int64_t kMaxElements = int64_t(1) << 37;        // of a plan: twice a GPU's memory of parameters
constexpr float kTop = 448.0f;      // largest e4m3 value
constexpr float kTiny = 1e-30f;     // a block whose largest magnitude is below is stored as 0

struct Chunk {
  float* p;
  void* copy;                       // 16-bit copy of p or nullptr
  int64_t state;                    // first element in the state arrays (a multiple of kBlock)
  int64_t grad;                     // first element in the tensor's gradient
  int tensor;
  int n;                            // elements, <= kChunk
  float decay;
  int pad;
};

template <int N> struct Grads { const void* p[N]; };

struct StepArgs {
  const Chunk* chunks;
  int first_tensor;
  int copy_type;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  const float* grad_scale;
  float b1, omb1, b2, omb2, eps, lr, step, inv_c2;
  uint32_t seed;
};

__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// sqrt(x) of two numbers, rounded to nearest: the residual of x * (1 / sqrt(x)) corrects its last bit
// (Markstein 1990).  For fp32 numbers from 2^-102 on, and for NaN, it gives __fsqrt_rn's result
// (compared one by one); below, the residual underflows, and of 0 and infinity it makes NaN.
__device__ __forceinline__ Pair sqrt_near(Pair x) {
  float a, b, ya, yb;
  halves(x, a, b);
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(ya) : "f"(a));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(yb) : "f"(b));
  const Pair y = pair(ya, yb), s = mul2(x, y), n = mul2(y, pair(-0.5f, -0.5f));
  return fma2(fma2(s, s, mul2(x, pair(-1.0f, -1.0f))), n, s);      // (x - s s) y / 2 + s
}
// The same for all numbers: small ones are taken up by 2^64, their root down by 2^32, both exactly.
__device__ __forceinline__ Pair sqrt_any(Pair x) {
  float a, b, ra, rb;
  halves(x, a, b);
  const bool la = a < 0x1p-38f, lb = b < 0x1p-38f;
  halves(sqrt_near(pair(la ? a * 0x1p64f : a, lb ? b * 0x1p64f : b)), ra, rb);
  return pair(a == 0.0f || a == INFINITY ? a : la ? ra * 0x1p-32f : ra,
              b == 0.0f || b == INFINITY ? b : lb ? rb * 0x1p-32f : rb);
}

// 20 random bits for place j: a multiplicative hash with the fractions of the golden
// ratio, sqrt(2) and sqrt(3) as multipliers.
__device__ __forceinline__ uint32_t random20(uint32_t j, uint32_t seed) {
  uint32_t x = (j + seed * 0xBB67AE85u) * 0x9E3779B9u;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return (x >> 12) ^ (x >> 25);        // (x ^ x >> 13) >> 12
}

// a >= 0 rounded to a value of e4m3's grid, up or down by the 20 random bits.  From 2^-6 on
// the grid keeps 3 mantissa bits of fp32's 23; below it is even with step 2^-9, which is the
// same truncation after adding 2^-6.  What is not 0 stays so.
__device__ __forceinline__ float round_random_normal(float a, uint32_t r) {
  return __uint_as_float((__float_as_uint(a) + r) & 0xFFF00000u);
}
__device__ __forceinline__ float round_random(float a, uint32_t r) {
  const float low = a < 0.015625f ? 0.015625f : 0.0f;
  const float t = round_random_normal(a + low, r) - low;
  return a == 0.0f ? 0.0f : fmaxf(t, 0.001953125f);
}

__device__ __forceinline__ uint32_t to_e4m3x4(const float* x) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[0], x[1]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[2], x[3]), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
__device__ __forceinline__ void from_e4m3x4(uint32_t w, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(
        static_cast<__nv_fp8x2_storage_t>((w >> (16 * i)) & 0xFFFFu), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

template <typename G>
__device__ __forceinline__ void load_grad4(const G* g, float* x);
template <>
__device__ __forceinline__ void load_grad4<float>(const float* g, float* x) {
  const float4 f = *reinterpret_cast<const float4*>(g);
  x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
}
template <typename G>
__device__ __forceinline__ void load_grad4(const G* g, float* x) {
  const uint2 w = *reinterpret_cast<const uint2*>(g);
  widen2<G>(w.x, x[0], x[1]);
  widen2<G>(w.y, x[2], x[3]);
}

// Largest magnitude of the block held by a warp, NaN and infinity above all numbers: the
// magnitudes' bit patterns order as unsigned integers.
__device__ __forceinline__ float warp_abs_max(float a) {
  return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(a) & 0x7FFFFFFFu));
}

// A warp's block of 256 elements, 8 a lane.  32-bit states: two groups of four consecutive
// ones, so that every 16-byte access of a warp is contiguous.  8-bit states: 8 consecutive ones,
// which takes half the instructions for the narrow arrays.
struct Block {
  const Chunk& c;
  int b0;              // first element of the block in the chunk
  int64_t s0;          // and in the state arrays
  bool full;           // whole, and aligned for wide accesses
};
template <int BITS>
__device__ __forceinline__ int element(int i) {           // of the lane's i-th in the block
  const int lane = threadIdx.x & 31;
  return BITS == 32 ? (i >> 2) * 128 + lane * 4 + (i & 3) : lane * 8 + i;
}

template <int BITS, typename G>
__device__ __forceinline__ bool is_wide(const Chunk& c, const G* g) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(c.p), q = reinterpret_cast<uintptr_t>(g),
                  r = reinterpret_cast<uintptr_t>(c.copy);
  if (BITS == 32) return ((p & 15) | (q & (4 * sizeof(G) - 1)) | (r & 7)) == 0;
  return ((p & 31) | (q & 15) | (r & 15)) == 0;
}

// One by one, where a block is short or not aligned.
template <int BITS, typename G>
__device__ __forceinline__ void load_single(const Block& b, const G* g, float* p, float* gr) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = b.b0 + element<BITS>(i);
    p[i] = e < b.c.n ? b.c.p[e] : 0.0f;
    gr[i] = e < b.c.n ? Elem<G>::up(g[e]) : 0.0f;
  }
}

// a + b, each rounded: a product of two pairs and a sum of them would be contracted to one
// operation (by the assembler, whatever the rounding modifiers and -fmad=false say).
__device__ __forceinline__ Pair add_products(Pair a, Pair b) {
  float a0, a1, b0, b1;
  halves(a, a0, a1);
  halves(b, b0, b1);
  return pair(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
}

__device__ __forceinline__ void store_256(float* to, const float* x) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(x[0]), "f"(x[1]),
               "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
               : "memory");
}

// The step of a block and the stores of everything it changes.
template <int BITS>
__device__ __forceinline__ void update(const StepArgs& a, const Block& b, float gs, float* p, const float* gr,
                                       float* m, float* v) {
  const int lane = threadIdx.x & 31, b0 = b.b0;
  const int64_t s0 = b.s0;
  const bool full = b.full;
  const Chunk& c = b.c;
  const float keep = 1.0f - a.lr * c.decay;
  float root[8];
  float m_top = 0.0f, r_top = 0.0f;
  // The states are rounded operation by operation, so that what is stored in 8 bits can be
  // reproduced exactly: one unit in the 24th place can move a code by 1/8 of its value.  Two
  // elements an instruction: in 8 bits the arithmetic is as long as the memory takes.
  auto both = [](float x) { return pair(x, x); };
  float least = INFINITY, most = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const Pair g2 = mul2(pair(gr[i], gr[i + 1]), both(gs));
    const Pair m2 = add_products(mul2(both(a.b1), pair(m[i], m[i + 1])), mul2(both(a.omb1), g2));
    const Pair v2 = add_products(mul2(both(a.b2), pair(v[i], v[i + 1])), mul2(mul2(both(a.omb2), g2), g2));
    halves(m2, m[i], m[i + 1]);
    halves(v2, v[i], v[i + 1]);
    least = fminf(least, fminf(v[i], v[i + 1]));
    most = fmaxf(most, fmaxf(v[i], v[i + 1]));
  }
  // One look at a warp's second moments: with zeros among them, numbers close to zero, or squares
  // that have passed fp32's range, they take the longer root (it for all of them: 316 us for 71.2 M
  // elements of 32-bit states and 694 for 285 M of 8-bit states, this 307 and 688).
  if (__any_sync(~0u, least < 0x1p-102f || most == INFINITY)) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) halves(sqrt_any(pair(v[i], v[i + 1])), root[i], root[i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 2) halves(sqrt_near(pair(v[i], v[i + 1])), root[i], root[i + 1]);
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float da, db;
    halves(fma2(pair(root[i], root[i + 1]), both(a.inv_c2), both(a.eps)), da, db);
    const Pair u = mul2(pair(m[i], m[i + 1]), pair(rcp_fast(da), rcp_fast(db)));
    halves(fma2(u, both(-a.step), mul2(pair(p[i], p[i + 1]), both(keep))), p[i], p[i + 1]);
    if constexpr (BITS == 8) {
      m_top = max_nan(m_top, max_nan(fabsf(m[i]), fabsf(m[i + 1])));
      r_top = max_nan(r_top, max_nan(root[i], root[i + 1]));
    }
  }
  if (full) {
    uint32_t w[4];
    if (c.copy) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = a.copy_type == HA_TYPE_BF16 ? narrow2<__nv_bfloat16>(p[2 * i], p[2 * i + 1])
                                           : narrow2<__half>(p[2 * i], p[2 * i + 1]);
    }
    uint16_t* copy = static_cast<uint16_t*>(c.copy);
    if constexpr (BITS == 32) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int e = b0 + q * 128 + lane * 4;
        __stcs(reinterpret_cast<float4*>(c.p + e), make_float4(p[4 * q], p[4 * q + 1], p[4 * q + 2], p[4 * q + 3]));
        if (copy) __stcs(reinterpret_cast<uint2*>(copy + e), make_uint2(w[2 * q], w[2 * q + 1]));
      }
    } else {
      store_256(c.p + b0 + lane * 8, p);
      if (copy) __stcs(reinterpret_cast<uint4*>(copy + b0 + lane * 8), make_uint4(w[0], w[1], w[2], w[3]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = b0 + element<BITS>(i);
      if (e >= c.n) continue;
      c.p[e] = p[i];
      if (c.copy) {
        if (a.copy_type == HA_TYPE_BF16)
          static_cast<__nv_bfloat16*>(c.copy)[e] = __float2bfloat16_rn(p[i]);
        else
          static_cast<__half*>(c.copy)[e] = __float2half_rn(p[i]);
      }
    }
  }
  uint32_t m8[2], r8[2];
  if constexpr (BITS == 8) {
    m_top = warp_abs_max(m_top);
    r_top = warp_abs_max(r_top);
    if (m_top < kTiny) m_top = 0.0f;
    if (r_top < kTiny) r_top = 0.0f;
    const float mi = m_top == 0.0f ? 0.0f : __fmul_rn(__frcp_rn(m_top), kTop);
    const float ri = r_top == 0.0f ? 0.0f : __fmul_rn(__frcp_rn(r_top), kTop);
    least = INFINITY;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      halves(mul2(pair(m[i], m[i + 1]), both(mi)), m[i], m[i + 1]);
      halves(mul2(pair(root[i], root[i + 1]), both(ri)), root[i], root[i + 1]);
      least = fminf(least, fminf(root[i], root[i + 1]));
    }
    const uint32_t j = static_cast<uint32_t>(s0) + lane * 8;
    if (__all_sync(~0u, least >= 0.015625f)) {       // nearly always: no value below 2^-6
#pragma unroll
      for (int i = 0; i < 8; ++i)
        root[i] = round_random_normal(root[i], random20(j + i, a.seed));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        root[i] = round_random(root[i], random20(j + i, a.seed));
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      m8[q] = to_e4m3x4(m + 4 * q);
      r8[q] = to_e4m3x4(root + 4 * q);
    }
    if (lane == 0) {
      a.m_scale[s0 / kBlock] = m_top * (1.0f / kTop);
      a.v_scale[s0 / kBlock] = r_top * (1.0f / kTop);
    }
  }
  if constexpr (BITS == 32) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int64_t s = s0 + q * 128 + lane * 4;
      __stcs(reinterpret_cast<float4*>(static_cast<float*>(a.m) + s),
             make_float4(m[4 * q], m[4 * q + 1], m[4 * q + 2], m[4 * q + 3]));
      __stcs(reinterpret_cast<float4*>(static_cast<float*>(a.v) + s),
             make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]));
    }
  } else {
    const int64_t s = s0 + lane * 8;
    __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.m) + s), make_uint2(m8[0], m8[1]));
    __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.v) + s), make_uint2(r8[0], r8[1]));
  }
}

// One CTA a chunk.  States of 32 bits: the stream of 30 bytes an element keeps the memory busy
// by itself (71.2 M elements with a 16-bit copy: 307 us, 7.0 TB/s).
template <typename G, int NG>
__global__ void __launch_bounds__(kThreads, 10) k_adamw32(const __grid_constant__ Grads<NG> grads,
                                                         const __grid_constant__ StepArgs a) {
  const Chunk c = a.chunks[blockIdx.x];
  const G* g = static_cast<const G*>(grads.p[c.tensor - a.first_tensor]) + c.grad;
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const int lane = threadIdx.x & 31, b0 = (threadIdx.x >> 5) * kBlock;
  if (b0 >= c.n) return;
  const Block b = {c, b0, c.state + b0, is_wide<32>(c, g) && b0 + kBlock <= c.n};
  float p[8], gr[8], m[8], v[8];
  if (b.full) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int e = b0 + q * 128 + lane * 4;
      const float4 f = __ldcs(reinterpret_cast<const float4*>(c.p + e));
      p[4 * q] = f.x; p[4 * q + 1] = f.y; p[4 * q + 2] = f.z; p[4 * q + 3] = f.w;
      load_grad4<G>(g + e, gr + 4 * q);
    }
  } else {
    load_single<32>(b, g, p, gr);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int64_t s = b.s0 + q * 128 + lane * 4;
    const float4 fm = __ldcs(reinterpret_cast<const float4*>(static_cast<float*>(a.m) + s));
    const float4 fv = __ldcs(reinterpret_cast<const float4*>(static_cast<float*>(a.v) + s));
    m[4 * q] = fm.x; m[4 * q + 1] = fm.y; m[4 * q + 2] = fm.z; m[4 * q + 3] = fm.w;
    v[4 * q] = fv.x; v[4 * q + 1] = fv.y; v[4 * q + 2] = fv.z; v[4 * q + 3] = fv.w;
  }
  update<32>(a, b, gs, p, gr, m, v);
}

// States of 8 bits: half the bytes and twice the arithmetic.  Small CTAs in the order of the
// memory, many of them at once (285 M elements with bf16 gradients and a bf16 copy: 688 us, 6.6
// TB/s; CTAs of 256 threads 710; CTAs that stay and take every 608th chunk, with loads three
// blocks ahead in shared memory, 831: they drift apart, and the memory's pages with them).
__device__ __forceinline__ void load_256(float* x, const float* from) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
               : "l"(from));
}
template <typename G, int NG>
__global__ void __launch_bounds__(kThreads, 10) k_adamw8(const __grid_constant__ Grads<NG> grads,
                                                        const __grid_constant__ StepArgs a) {
  const Chunk c = a.chunks[blockIdx.x];
  const G* g = static_cast<const G*>(grads.p[c.tensor - a.first_tensor]) + c.grad;
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const int lane = threadIdx.x & 31, b0 = (threadIdx.x >> 5) * kBlock;
  if (b0 >= c.n) return;
  const Block b = {c, b0, c.state + b0, is_wide<8>(c, g) && b0 + kBlock <= c.n};
  float p[8], gr[8], m[8], v[8];
  const uint2 mc = __ldcs(reinterpret_cast<const uint2*>(static_cast<uint8_t*>(a.m) + b.s0 + lane * 8));
  const uint2 rc = __ldcs(reinterpret_cast<const uint2*>(static_cast<uint8_t*>(a.v) + b.s0 + lane * 8));
  const float ms = a.m_scale[b.s0 / kBlock], vs = a.v_scale[b.s0 / kBlock];
  if (b.full) {
    load_256(p, c.p + b0 + lane * 8);
    load_grad4<G>(g + b0 + lane * 8, gr);
    load_grad4<G>(g + b0 + lane * 8 + 4, gr + 4);
  } else {
    load_single<8>(b, g, p, gr);
  }
  from_e4m3x4(mc.x, m);
  from_e4m3x4(mc.y, m + 4);
  from_e4m3x4(rc.x, v);
  from_e4m3x4(rc.y, v + 4);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    halves(mul2(pair(m[i], m[i + 1]), pair(ms, ms)), m[i], m[i + 1]);
    const Pair r2 = mul2(pair(v[i], v[i + 1]), pair(vs, vs));
    halves(mul2(r2, r2), v[i], v[i + 1]);
  }
  update<8>(a, b, gs, p, gr, m, v);
}

}  // namespace
}  // namespace ha

struct hier_avg_adamw {
  int bits = 0, n_tensors = 0, copy_type = 0;
  int64_t elements = 0;                       // of each state array, padded pieces
  std::vector<ha::Chunk> chunks;
  std::vector<int64_t> first_chunk;           // per tensor, and the end
  const ha::Chunk* table = nullptr;
  void *m = nullptr, *v = nullptr;
  float *m_scale = nullptr, *v_scale = nullptr;
};

namespace {

using namespace ha;

// The gradients' addresses travel in the kernel's arguments (at most 32,764 bytes), so a
// step needs no copy to the device.  Few tensors take a small argument block.
template <int BITS, typename G, int NG>
cudaError_t launch_range(const hier_avg_adamw* h, const void* const* grads, int t0, int t1,
                         StepArgs a, cudaStream_t s) {
  const int64_t c0 = h->first_chunk[t0], c1 = h->first_chunk[t1];
  if (c0 == c1) return cudaSuccess;
  Grads<NG> g;
  std::memset(&g, 0, sizeof g);
  for (int t = t0; t < t1; ++t) g.p[t - t0] = grads[t];
  a.chunks = h->table + c0;
  a.first_tensor = t0;
  if constexpr (BITS == 32) {
    k_adamw32<G, NG><<<static_cast<unsigned>(c1 - c0), kThreads, 0, s>>>(g, a);
  } else {
    k_adamw8<G, NG><<<static_cast<unsigned>(c1 - c0), kThreads, 0, s>>>(g, a);
  }
  return cudaGetLastError();
}

template <int BITS, typename G>
cudaError_t launch_all(const hier_avg_adamw* h, const void* const* grads, const StepArgs& a,
                       cudaStream_t s) {
  constexpr int kFew = 64, kSome = 512, kMany = 3968;
  if (h->n_tensors <= kFew) return launch_range<BITS, G, kFew>(h, grads, 0, h->n_tensors, a, s);
  if (h->n_tensors <= kSome) return launch_range<BITS, G, kSome>(h, grads, 0, h->n_tensors, a, s);
  for (int t = 0; t < h->n_tensors; t += kMany) {
    const int end = t + kMany < h->n_tensors ? t + kMany : h->n_tensors;
    const cudaError_t e = launch_range<BITS, G, kMany>(h, grads, t, end, a, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <int BITS>
cudaError_t launch_type(const hier_avg_adamw* h, const void* const* grads, int grad_type,
                        const StepArgs& a, cudaStream_t s) {
  switch (grad_type) {
    case HA_TYPE_FP32: return launch_all<BITS, float>(h, grads, a, s);
    case HA_TYPE_BF16: return launch_all<BITS, __nv_bfloat16>(h, grads, a, s);
    default: return launch_all<BITS, __half>(h, grads, a, s);
  }
}

}  // namespace

extern "C" int hier_avg_adamw_create(int bits, int n_tensors, int64_t n_pieces, const int* tensor,
                                     float* const* p_dev, void* const* copy_dev, int copy_type,
                                     const int64_t* n, const int64_t* grad_offset,
                                     const float* decay, hier_avg_adamw** out) {
  if (!out) return HA_EINVAL;
  *out = nullptr;
  if ((bits != 8 && bits != 32) || n_tensors < 1 || n_pieces < 0) return HA_EINVAL;
  if (n_pieces > 0 && (!tensor || !p_dev || !n || !grad_offset || !decay)) return HA_EINVAL;
  if (copy_dev && copy_type != HA_TYPE_BF16 && copy_type != HA_TYPE_FP16) return HA_EINVAL;
  try {
    auto plan = std::make_unique<hier_avg_adamw>();
    hier_avg_adamw* h = plan.get();
    h->bits = bits;
    h->n_tensors = n_tensors;
    h->copy_type = copy_type;
    int last = 0;
    bool ok = true;
    for (int64_t i = 0; i < n_pieces && ok; ++i) {
      ok = tensor[i] >= last && tensor[i] < n_tensors && n[i] >= 0 && grad_offset[i] >= 0 &&
           (n[i] == 0 || p_dev[i]) && std::isfinite(decay[i]) &&
           n[i] <= kMaxElements - h->elements;            // before the plan takes the host's memory
      if (!ok) break;
      while (static_cast<int>(h->first_chunk.size()) <= tensor[i])
        h->first_chunk.push_back(static_cast<int64_t>(h->chunks.size()));
      last = tensor[i];
      for (int64_t at = 0; at < n[i]; at += kChunk) {
        Chunk c = {};
        c.p = p_dev[i] + at;
        c.copy = copy_dev && copy_dev[i] ? static_cast<uint16_t*>(copy_dev[i]) + at : nullptr;
        c.state = h->elements + at;
        c.grad = grad_offset[i] + at;
        c.tensor = tensor[i];
        c.n = static_cast<int>(n[i] - at < kChunk ? n[i] - at : kChunk);
        c.decay = decay[i];
        h->chunks.push_back(c);
      }
      h->elements += (n[i] + kBlock - 1) / kBlock * kBlock;
    }
    while (static_cast<int>(h->first_chunk.size()) <= n_tensors)
      h->first_chunk.push_back(static_cast<int64_t>(h->chunks.size()));
    if (!ok || h->chunks.size() > 0x7FFFFFFFu) return HA_EINVAL;
    *out = plan.release();
  } catch (const std::bad_alloc&) {
    return HA_ENOMEM;
  }
  return HA_OK;
}

extern "C" void hier_avg_adamw_destroy(hier_avg_adamw* h) { delete h; }

extern "C" int hier_avg_adamw_sizes(const hier_avg_adamw* h, int64_t* elements, int64_t* table_bytes) {
  if (!h) return HA_EINVAL;
  if (elements) *elements = h->elements;
  if (table_bytes) *table_bytes = static_cast<int64_t>(h->chunks.size() * sizeof(Chunk));
  return HA_OK;
}

extern "C" int hier_avg_adamw_bind(hier_avg_adamw* h, void* table_dev, int64_t table_bytes,
                                   void* m_dev, void* v_dev, float* m_scale_dev,
                                   float* root_scale_dev, void* stream) {
  if (!h) return HA_EINVAL;
  const int64_t need = static_cast<int64_t>(h->chunks.size() * sizeof(Chunk));
  if (need > 0) {
    if (!table_dev || !m_dev || !v_dev || (h->bits == 8 && (!m_scale_dev || !root_scale_dev)))
      return HA_EINVAL;
    if ((reinterpret_cast<uintptr_t>(m_dev) | reinterpret_cast<uintptr_t>(v_dev) |
         reinterpret_cast<uintptr_t>(table_dev)) & 15)
      return HA_EINVAL;
    if (table_bytes < need) return HA_ENOMEM;
    if (cudaMemcpyAsync(table_dev, h->chunks.data(), need, cudaMemcpyHostToDevice,
                        static_cast<cudaStream_t>(stream)) != cudaSuccess)
      return HA_ECUDA;
  }
  h->table = static_cast<const Chunk*>(table_dev);
  h->m = m_dev;
  h->v = v_dev;
  h->m_scale = m_scale_dev;
  h->v_scale = root_scale_dev;
  return HA_OK;
}

extern "C" int hier_avg_adamw_step(hier_avg_adamw* h, const void* const* grads_dev, int grad_type,
                                   double lr, double beta1, double beta2, double eps, int64_t t,
                                   const float* grad_scale_dev, uint32_t seed, void* stream) {
  if (!h || !grads_dev || !type_ok(grad_type) || t < 1) return HA_EINVAL;
  if (!std::isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
      !(eps >= FLT_MIN) || !std::isfinite(eps))      // below, the reciprocal of eps alone is infinite
    return HA_EINVAL;
  if (h->chunks.empty()) return HA_OK;
  if (!h->table) return HA_ESTATE;
  for (int i = 0; i < h->n_tensors; ++i)
    if (!grads_dev[i] && h->first_chunk[i] != h->first_chunk[i + 1]) return HA_EINVAL;
  StepArgs a = {};
  a.copy_type = h->copy_type;
  a.m = h->m;
  a.v = h->v;
  a.m_scale = h->m_scale;
  a.v_scale = h->v_scale;
  a.grad_scale = grad_scale_dev;
  a.b1 = static_cast<float>(beta1);
  a.omb1 = static_cast<float>(1.0 - beta1);
  a.b2 = static_cast<float>(beta2);
  a.omb2 = static_cast<float>(1.0 - beta2);
  a.eps = static_cast<float>(eps);
  a.lr = static_cast<float>(lr);
  a.step = static_cast<float>(lr / (1.0 - std::pow(beta1, static_cast<double>(t))));
  a.inv_c2 = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(beta2, static_cast<double>(t))));
  a.seed = seed;
  const cudaError_t e =
      h->bits == 32 ? launch_type<32>(h, grads_dev, grad_type, a, static_cast<cudaStream_t>(stream))
                    : launch_type<8>(h, grads_dev, grad_type, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? HA_OK : HA_ECUDA;
}
