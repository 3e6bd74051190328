// Shared by the operator translation units: element types and pairs of them, the table of
// what is done once a device, logits that count as masked and the order of floats, launches that
// overlap, and arithmetic on two floats an instruction.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "hier_avg.h"

namespace ha {

__host__ __device__ constexpr int type_size(int type) { return type == HA_TYPE_FP32 ? 4 : 2; }
inline bool type_ok(int type) { return type >= HA_TYPE_FP32 && type <= HA_TYPE_FP16; }

// The current device's slot of a table that keeps, for each kernel, what was found out or set
// once for it (-1: no device).
constexpr int kMaxDevices = 16;
inline int device_slot() {
  int d = -1;
  return cudaGetDevice(&d) == cudaSuccess && d < kMaxDevices ? d : -1;
}
// Allows the kernel `bytes` of dynamic shared memory, once a device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, bool (&done)[kMaxDevices]) {
  const int d = device_slot();
  if (d >= 0 && done[d]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && d >= 0) done[d] = true;
  return e;
}

template <typename T> struct Elem;
template <> struct Elem<float> {
  static __device__ __forceinline__ float up(float x) { return x; }
  static __device__ __forceinline__ float down(float x) { return x; }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Elem<__half> {
  static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
};

// The words of a vector load, widened: two 16-bit values in a word, the first in its low half.
template <typename T> __device__ __forceinline__ void widen2(uint32_t w, float& a, float& b);
template <> __device__ __forceinline__ void widen2<__nv_bfloat16>(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xFFFF0000u);
}
template <> __device__ __forceinline__ void widen2<__half>(uint32_t w, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  a = f.x;
  b = f.y;
}
template <typename T> __device__ __forceinline__ uint32_t narrow2(float a, float b);
template <> __device__ __forceinline__ uint32_t narrow2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t narrow2<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Exponentials are taken as the hardware's 2^x.
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
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

// The elements of a 16-byte load.
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

template <typename T>
__device__ __forceinline__ uint4 pack(const float* v) {
  if constexpr (sizeof(T) == 4)
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  else
    return make_uint4(narrow2<T>(v[0], v[1]), narrow2<T>(v[2], v[3]), narrow2<T>(v[4], v[5]), narrow2<T>(v[6], v[7]));
}

// A kernel that follows another on its stream may start while that one ends: it waits before it reads what
// the other wrote, and the other says early that it may start.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// Two floats an instruction, each rounded as by the instruction for one.
struct Pair { uint64_t w; };
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.w) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ void halves(Pair p, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.w));
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair p;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(p.w) : "l"(a.w), "l"(b.w));
  return p;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair p;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p.w) : "l"(a.w), "l"(b.w));
  return p;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair p;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(p.w) : "l"(a.w), "l"(b.w), "l"(c.w));
  return p;
}

}  // namespace ha
