// Element types of the dense tensors (fp32, fp16, bf16): conversions to and from fp32, vectors of elements in
// registers, dispatch over MTS_DTYPE_*.  Internal to the library.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace mts {

// Kernels of the dense operators in the launch trace, behind those of the tables and caches (whose header stands in the profiler captures'
// hash and does not change with these).
enum DenseKernelId { K_RECURRENCE_FWD = K_COUNT, K_RECURRENCE_BWD, K_RELPOS_FWD, K_RELPOS_BWD, K_ADAMW, K_ADAMW_STATE, K_ALL_COUNT };

inline bool known_dtype(int32_t dtype) {
  return dtype == MTS_DTYPE_FP32 || dtype == MTS_DTYPE_FP16 || dtype == MTS_DTYPE_BF16;
}
inline int dtype_bytes(int32_t dtype) { return dtype == MTS_DTYPE_FP32 ? 4 : 2; }

// Calls fn(T()) with the element type of `dtype` (known_dtype checked by the caller).
template <typename Fn>
inline int with_dtype(int32_t dtype, Fn&& fn) {
  if (dtype == MTS_DTYPE_FP32) return fn(float());
  if (dtype == MTS_DTYPE_FP16) return fn(__half());
  return fn(__nv_bfloat16());
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Two packed 16-bit elements <-> two floats.
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Eight consecutive fp32 elements on a 32-byte boundary: one 256-bit access of sm_100.
__device__ __forceinline__ void load8_f32(const float* p, float (&v)[8]) {
  asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "l"(p));
}
__device__ __forceinline__ void store8_f32(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               :: "l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

// Eight consecutive elements on a boundary of eight elements, as fp32.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = unpack2<T>(u[k]);
    v[2 * k] = f.x;
    v[2 * k + 1] = f.y;
  }
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) { load8_f32(p, v); }

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]),
                                            pack2<T>(v[6], v[7]));
}
template <>
__device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) { store8_f32(p, v); }

template <typename T>
__device__ __forceinline__ bool aligned8(const T* p) { return (reinterpret_cast<uintptr_t>(p) & (8 * sizeof(T) - 1)) == 0; }

}  // namespace mts
