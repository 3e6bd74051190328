// Shared by the operator translation units (grouped products, token log
// probabilities, AdamW): element types and pairs of them, the table of what is done
// once a device, and arithmetic on two floats an instruction.
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
