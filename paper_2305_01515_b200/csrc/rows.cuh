// Rows of a [N, V] tensor read by aligned vectors wherever they start, and what softmaxes over them share.  Internal to the library.
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
// READ_ONLY: nothing writes to the row while the kernel runs (a gradient may take its place where it is false).
template <typename T, bool READ_ONLY = true>
struct RowBatches {
  static constexpr int E = 16 / (int)sizeof(T);
  static __device__ __forceinline__ uint4 load16(const T* p) {
    return READ_ONLY ? __ldg(reinterpret_cast<const uint4*>(p)) : *reinterpret_cast<const uint4*>(p);
  }
  const T* row;
  int32_t V, shift, count, whole_begin, whole_end;       // batches [whole_begin, whole_end) are whole
  __device__ __forceinline__ RowBatches(const T* row_, int32_t V_) : row(row_), V(V_) {
    shift = (int32_t)((reinterpret_cast<uintptr_t>(row_) & 15) / sizeof(T));
    count = (int32_t)(((int64_t)V + shift + E - 1) / E);
    whole_begin = shift != 0;
    whole_end = max((V + shift) / E, whole_begin);
  }
  // Of the elements before the whole batches each of E lanes has one at most, of those behind them the next E lanes; -1: none.
  __device__ __forceinline__ int32_t edge(int lane) const {
    const int32_t i = lane < E ? lane : first(whole_end) + lane - E;
    return i < (lane < E ? min(V, first(whole_begin)) : V) ? i : -1;
  }
  __device__ __forceinline__ int32_t first(int32_t b) const { return b * E - shift; }      // may be negative; at most V + E
  static constexpr uint32_t LOW = sizeof(T) == 4 ? 0xFF800000u : (__is_same(T, __half) ? 0xFC00FC00u : 0xFF80FF80u);     // -infinity
  // The batch as it is stored, -infinity outside the row.
  __device__ __forceinline__ uint4 raw(int32_t b) const {
    const int32_t i = first(b);
    if (i >= 0 && i <= V - E) return load16(row + i);
    uint4 w = make_uint4(LOW, LOW, LOW, LOW);
    if (i > -E && i < V) {
      T* const e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (i + k >= 0 && i + k < V) e[k] = row[i + k];
    }
    return w;
  }
  // A whole batch, not to be read again soon.
  static __device__ __forceinline__ void store16(T* to, const float (&v)[E]) {
    if constexpr (sizeof(T) == 4) __stcs(reinterpret_cast<float4*>(to), make_float4(v[0], v[1], v[2], v[3]));
    else __stcs(reinterpret_cast<uint4*>(to), make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])));
  }
  // Writes the batch's elements that lie in the row.
  __device__ __forceinline__ void store(int32_t b, const float (&v)[E]) const {
    const int32_t i = first(b);
    T* const to = const_cast<T*>(row) + i;
    if (i >= 0 && i <= V - E) {
      store16(to, v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (i + e >= 0 && i + e < V) to[e] = from_f32<T>(v[e]);
    }
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

// The elements of another row under the batches of `RowBatches` r (a row of scores under the row of their gradient), which need not start on boundaries: two
// aligned accesses and a shift where they do not.
template <typename T>
struct RowUnder {
  static constexpr int E = RowBatches<T>::E;
  const T* row;
  const RowBatches<T>& r;
  int32_t ahead;                 // elements from a boundary to a batch's first
  __device__ __forceinline__ RowUnder(const T* row_, const RowBatches<T>& r_) : row(row_), r(r_) {
    ahead = (int32_t)((reinterpret_cast<uintptr_t>(row_) / sizeof(T) + E - r_.shift) % E);
  }
  // Whether the accesses for batch b lie within the row.
  __device__ __forceinline__ bool within(int32_t b) const {
    const int32_t i = r.first(b) - ahead;
    return i >= 0 && i <= r.V - (ahead ? 2 * E : E);
  }
  __device__ __forceinline__ uint4 shifted(const uint4& lo, const uint4& hi) const {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const int words = ahead * (int)sizeof(T) / 4;
    uint32_t s[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      uint32_t x = w[k];
      if (words == 1) x = w[k + 1];
      if (words == 2) x = w[k + 2];
      if (words == 3 && k + 3 < 8) x = w[k + 3 < 8 ? k + 3 : 7];
      s[k] = x;
    }
    const int bits = ahead * (int)sizeof(T) * 8 % 32;
    return make_uint4(__funnelshift_r(s[0], s[1], bits), __funnelshift_r(s[1], s[2], bits), __funnelshift_r(s[2], s[3], bits), __funnelshift_r(s[3], s[4], bits));
  }
  // Batches [*from, *to) are whole and their accesses within the row.
  __device__ __forceinline__ void inner(int32_t* from, int32_t* to) const {
    *from = (r.shift + ahead + E - 1) / E;
    *to = (int32_t)(((int64_t)r.V - (ahead ? 2 * E : E) + ahead + r.shift) / E) + 1;
    if (r.V < (ahead ? 2 * E : E)) *to = *from;
  }
  __device__ __forceinline__ uint4 inside(const T* p) const {               // p: the batch's first element's access
    const uint4* const q = reinterpret_cast<const uint4*>(p);
    const uint4 lo = __ldcs(q);
    return ahead ? shifted(lo, __ldcs(q + 1)) : lo;
  }
  // The batch as it is stored, -infinity outside the row.  Not through the read-only path: the gradient may take the scores' place.
  __device__ __forceinline__ uint4 raw(int32_t b) const {
    const int32_t i = r.first(b);
    if (within(b)) return inside(row + (i - ahead));
    uint4 w = make_uint4(RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW);
    if (i > -E && i < r.V) {
      T* const e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (i + k >= 0 && i + k < r.V) e[k] = row[i + k];
    }
    return w;
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

// Largest of a warp's numbers (NaN counts as -infinity).
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(fmaxf(x, -INFINITY)));
  return y;
}
__device__ __forceinline__ float warp_min(float x) {
  float y;
  asm volatile("redux.sync.min.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
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
  __device__ __forceinline__ float sum() const { const float2 f = get(); return f.x + f.y; }
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

// Largest of the elements of 16 bytes (numbers only: NaN counts as -infinity): first as a pair of 16-bit elements or an fp32 number, which can
// be compared on, then as fp32.
template <typename T>
__device__ __forceinline__ uint32_t max_bits(uint32_t a, uint32_t b) {
  uint32_t m;
  if constexpr (sizeof(T) == 4) asm("max.f32 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  else if constexpr (__is_same(T, __half)) asm("max.f16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  else asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t max_bits(uint32_t a, const uint4& w) {
  if constexpr (sizeof(T) == 4) {                                         // three operands in one instruction
    asm("max.f32 %0, %0, %1, %2;" : "+r"(a) : "r"(w.x), "r"(w.y));
    asm("max.f32 %0, %0, %1, %2;" : "+r"(a) : "r"(w.z), "r"(w.w));
    return a;
  }
  return max_bits<T>(max_bits<T>(max_bits<T>(w.x, w.y), max_bits<T>(w.z, w.w)), a);
}
template <typename T>
__device__ __forceinline__ uint32_t max_bits(const uint4& w) {
  if constexpr (sizeof(T) == 4) {
    uint32_t a;
    asm("max.f32 %0, %1, %2, %3;" : "=r"(a) : "r"(w.x), "r"(w.y), "r"(w.z));
    return max_bits<T>(a, w.w);
  }
  return max_bits<T>(max_bits<T>(w.x, w.y), max_bits<T>(w.z, w.w));
}
template <typename T>
__device__ __forceinline__ float max_value(uint32_t m) {
  if constexpr (sizeof(T) == 4) return fmaxf(__uint_as_float(m), -INFINITY);
  const float2 f = unpack2<T>(m);
  return fmaxf(fmaxf(f.x, f.y), -INFINITY);
}

// Exponents of a softmax are taken relative to the largest score m: c x - base with base = c m rounded, which is one instruction and leaves out no more of c m than
// half a unit of base's last place; that is put right at the end.  Below 2^23 it is less than one half, so that terms are at most 2^0.5.  From there on (large scales, or
// nothing but a mask's lowest value seen so far) it could be anything, and the exponent is c (x - m).
__device__ __forceinline__ float base_of(float m, float c) { return m == -INFINITY ? 0.f : __fmul_rn(m, c); }      // never joined with a sum into one rounding
__device__ __forceinline__ bool ordinary(float base) { return fabsf(base) < 8388608.f; }
// What the logarithm of a sum of 2^(c x - base) has too much by the rounding of the base.
__device__ __forceinline__ float log_excess(float m, float base, float c) { return ordinary(base) && m != -INFINITY ? fmaf(m, c, -base) * LN2 : 0.f; }

// scale (x - y), where x - y itself need not be a number of fp32 (scores of either sign around 2e38 and more, under a small scale).
__device__ __forceinline__ float scaled_difference(float x, float y, float scale) { return fmaf(0.5f, x, -0.5f * y) * (2.f * scale); }
// Exponent of the factor that takes sums relative to `from`, in the form that goes with it, to sums relative to `to`, which is not smaller.
__device__ __forceinline__ float change_of_base(float from, float to, float c) {
  const float a = base_of(from, c), b = base_of(to, c);
  if (ordinary(b)) return ordinary(a) ? a - b : fmaf(from, c, -b);
  return ordinary(a) ? -fmaf(to, c, -a) : (from - to) * c;
}

// Clusters: blocks that share a row.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// Address in block `rank` of the cluster of a variable of this block.
__device__ __forceinline__ uint32_t in_block(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}

// Few rows are shared by clusters, while the GPU has an SM for every block and a part 1,024 batches (one row of 5,000 fp32 batches by 1, 2, 4
// and 8 blocks: 6.0, 6.4, 5.8 and 6.0 us; 100 rows of 2,500: 5.9 us by single blocks, 7.1 by pairs).
constexpr int MAX_LOG_PARTS = 3;
inline int log_parts_of(int64_t N, int64_t batches) {
  int p = 0;
  while (p < MAX_LOG_PARTS && N << p <= 74 && batches >= 2048ll << p) ++p;
  return p;
}

// Checks of a [N, columns] tensor with rows `stride` elements apart, shared by the operators over rows.
inline int check_rows(const char* what, const char* name, const void* p, int32_t dtype, int64_t N, int64_t columns, int64_t stride) {
  if (stride < columns && N > 1) return set_error(MTS_ERR_INVALID_ARG, "%s: rows of %s are %lld apart, less than %lld", what, name, (long long)stride, (long long)columns);
  if (!p && N > 0) return set_error(MTS_ERR_INVALID_ARG, "%s: null %s", what, name);
  if ((uintptr_t)p % dtype_bytes(dtype)) return set_error(MTS_ERR_ALIGNMENT, "%s: %s is no multiple of its element size", what, name);
  return MTS_OK;
}

}  // namespace mts
