// Rows of a [N, V] tensor read by aligned vectors wherever they start, and reductions over a block.  Internal to the library.
#pragma once

#include <math.h>

#include "dense.cuh"

namespace mts {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// Least exponent that is worked with: 2 to it is 0, and a product with it is finite (an item that is ruled out has p log p = 0).
constexpr float LEAST_EXP = -16384.f;

// The exponent to work with for x: LEAST_EXP at least, NaN where x is (a NaN score, or one of +infinity less the largest).
__device__ __forceinline__ float exponent(float x) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(LEAST_EXP));
  return y;
}

// 2^x; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The elements of a row in batches of E = 16 bytes that start on 16-byte boundaries: batch b holds elements [b E - shift, b E - shift + E), of
// which those of the first and the last batch may lie outside the row.
template <typename T>
struct RowBatches {
  static constexpr int E = 16 / (int)sizeof(T);
  const T* row;
  int32_t V, shift, count;
  __device__ __forceinline__ RowBatches(const T* row_, int32_t V_) : row(row_), V(V_) {
    shift = (int32_t)((reinterpret_cast<uintptr_t>(row_) & 15) / sizeof(T));
    count = (int32_t)(((int64_t)V + shift + E - 1) / E);
  }
  __device__ __forceinline__ int32_t first(int32_t b) const { return b * E - shift; }      // may be negative; at most V + E
  __device__ __forceinline__ bool whole(int32_t b) const { const int32_t i = first(b); return i >= 0 && i <= V - E; }
  // The batch as fp32, -infinity outside the row.
  __device__ __forceinline__ void load(int32_t b, float (&v)[E]) const {
    const int32_t i = first(b);
    if (i >= 0 && i <= V - E) {
      const uint4 w = *reinterpret_cast<const uint4*>(row + i);
      unpack(w, v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = i + e >= 0 && i + e < V ? to_f32(row[i + e]) : -INFINITY;
    }
  }
  // The batch as it is stored, -infinity outside the row.
  __device__ __forceinline__ uint4 raw(int32_t b) const {
    const int32_t i = first(b);
    if (i >= 0 && i <= V - E) return __ldg(reinterpret_cast<const uint4*>(row + i));
    const uint32_t low = sizeof(T) == 4 ? 0xFF800000u : (__is_same(T, __half) ? 0xFC00FC00u : 0xFF80FF80u);
    uint4 w = make_uint4(low, low, low, low);
    if (i > -E && i < V) {
      T* const e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (i + k >= 0 && i + k < V) e[k] = row[i + k];
    }
    return w;
  }
  static __device__ __forceinline__ void unpack(const uint4& w, float (&v)[E]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        v[k] = __uint_as_float(u[k]);
      } else {
        const float2 f = unpack2<T>(u[k]);
        v[2 * k] = f.x;
        v[2 * k + 1] = f.y;
      }
    }
  }
};

// Order of scores with the lowest index first among equals, as whole numbers: the larger comes first.  -0 counts as 0; NaN comes last.
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return isnan(x) ? 0u : (b & 0x80000000u ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ uint64_t score_order(float x, int32_t index) {
  return (uint64_t)score_key(x) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int32_t order_index(uint64_t o) { return (int32_t)~(uint32_t)o; }

__device__ __forceinline__ float order_score(uint64_t o) {
  const uint32_t k = (uint32_t)(o >> 32);
  return k == 0u ? NAN : __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Pairs of fp32 numbers in one instruction.
struct Pair {
  unsigned long long bits;
  __device__ __forceinline__ Pair() {}
  __device__ __forceinline__ Pair(float x, float y) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(x), "f"(y)); }
  __device__ __forceinline__ float2 get() const {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(bits));
    return f;
  }
};
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
  return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
  return r;
}

// Largest of the elements of 16 bytes (numbers only: NaN counts as -infinity).
template <typename T>
__device__ __forceinline__ float max_of(const uint4& w) {
  if constexpr (sizeof(T) == 4) {
    return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
  } else {
    uint32_t m;
    if constexpr (sizeof(T) == 2 && !__is_same(T, __half))
      asm("{\n\t.reg .b32 a, b;\n\tmax.bf16x2 a, %1, %2;\n\tmax.bf16x2 b, %3, %4;\n\tmax.bf16x2 %0, a, b;\n\t}" : "=r"(m) : "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w));
    else
      asm("{\n\t.reg .b32 a, b;\n\tmax.f16x2 a, %1, %2;\n\tmax.f16x2 b, %3, %4;\n\tmax.f16x2 %0, a, b;\n\t}" : "=r"(m) : "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w));
    const float2 f = unpack2<T>(m);
    return fmaxf(fmaxf(f.x, f.y), -INFINITY);
  }
}

// Sum and maximum over a block of THREADS in a fixed order; every thread gets the result.  `room`: shared, [THREADS / 32]; free again at the
// next barrier of the block.
template <int THREADS>
__device__ __forceinline__ float block_sum(float x, float* room) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  if constexpr (THREADS > 32) {
    __syncthreads();
    if (lane_id() == 0) room[threadIdx.x / 32] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) x += room[w];
  }
  return x;
}
template <int THREADS>
__device__ __forceinline__ float block_max(float x, float* room) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  if constexpr (THREADS > 32) {
    __syncthreads();
    if (lane_id() == 0) room[threadIdx.x / 32] = x;
    __syncthreads();
    x = room[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) x = fmaxf(x, room[w]);
  }
  return x;
}

// Checks of a [N, columns] tensor with rows `stride` elements apart, shared by the operators over rows.
inline int check_rows(const char* what, const char* name, const void* p, int32_t dtype, int64_t N, int64_t columns, int64_t stride) {
  if (stride < columns && N > 1) return set_error(MTS_ERR_INVALID_ARG, "%s: rows of %s are %lld apart, less than %lld", what, name, (long long)stride, (long long)columns);
  if (!p && N > 0) return set_error(MTS_ERR_INVALID_ARG, "%s: null %s", what, name);
  if ((uintptr_t)p % dtype_bytes(dtype)) return set_error(MTS_ERR_ALIGNMENT, "%s: %s is no multiple of its element size", what, name);
  return MTS_OK;
}

}  // namespace mts
