// Root-mean-square norm of the residual stream, forward (output in the tensors' type or in 8 bits) and backward.
//
//   r = round(x + residual),  c = 1 / sqrt(mean_j r_j^2 + eps),  y_j = r_j c w_j
//   dx_j = dr_j + c (dy_j w_j - r_j a),  a = c^2 mean_j(dy_j w_j r_j),   dw_j = sum over rows of dy_j r_j c
#include <cuda_fp8.h>

#include <type_traits>

#include "rows.cuh"

namespace mts {

constexpr float LEAST_MAX = 7.888609052210118e-31f;      // 2^-100: least maximum of a group of 8-bit codes
constexpr float TOP_CODE = 448.f;                        // largest number of e4m3
constexpr int NORM_CHUNK = 256;                          // columns of a warp: eight to a lane
constexpr int NORM_CHUNKS = 4;                           // chunks that a warp holds at most
constexpr int NORM_WARPS = MTS_RMS_NORM_MAX_D / (NORM_CHUNK * NORM_CHUNKS);

// A row's part that a warp holds: I chunks of 256 columns, `step` chunks apart.  VECTOR: a lane has eight neighbouring columns (rows on 16-byte
// boundaries); else every 32nd column, which any row can be read by in whole sectors.  Columns behind the row's end hold 0.
template <typename T, bool VECTOR, int I>
struct Tile {
  static constexpr int Q = VECTOR ? (int)sizeof(T) / 2 : 1;
  uint4 q[VECTOR ? I : 1][Q];
  T s[VECTOR ? 1 : I][8];

  static __device__ __forceinline__ int column(int chunk, int e) { return chunk * NORM_CHUNK + (VECTOR ? lane_id() * 8 + e : lane_id() + 32 * e); }
  __device__ __forceinline__ void load(const T* row, int D, int chunk, int step) {
#pragma unroll
    for (int i = 0; i < I; ++i, chunk += step) {
      if constexpr (VECTOR) {
        const int at = column(chunk, 0);
        if (at + 8 <= D) {
#pragma unroll
          for (int k = 0; k < Q; ++k) q[i][k] = reinterpret_cast<const uint4*>(row + at)[k];
        } else {
#pragma unroll
          for (int k = 0; k < Q; ++k) q[i][k] = make_uint4(0u, 0u, 0u, 0u);
          T* const e = reinterpret_cast<T*>(q[i]);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (at + k < D) e[k] = row[at + k];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = column(chunk, e) < D ? row[column(chunk, e)] : from_f32<T>(0.f);
      }
    }
  }
  __device__ __forceinline__ void get(int i, float (&v)[8]) const {
    if constexpr (VECTOR) {
#pragma unroll
      for (int k = 0; k < Q; ++k) {
        const uint32_t u[4] = {q[i][k].x, q[i][k].y, q[i][k].z, q[i][k].w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if constexpr (sizeof(T) == 4) {
            v[4 * k + w] = __uint_as_float(u[w]);
          } else {
            const float2 f = unpack2<T>(u[w]);
            v[2 * w] = f.x;
            v[2 * w + 1] = f.y;
          }
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_f32(s[i][e]);
    }
  }
};

// Eight values of a lane, written to their columns of a row.
template <typename T, bool VECTOR>
__device__ __forceinline__ void store8(T* row, int D, int chunk, const float (&v)[8]) {
  using Columns = Tile<T, VECTOR, 1>;
  if constexpr (VECTOR) {
    T* const to = row + Columns::column(chunk, 0);
    if (Columns::column(chunk, 8) <= D) {
      if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        *reinterpret_cast<uint4*>(to) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
      }
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (Columns::column(chunk, e) < D) row[Columns::column(chunk, e)] = from_f32<T>(v[e]);
}

struct Weight {
  const void* w;
  int32_t dtype, aligned;                                // aligned: on a 16-byte boundary
};

// A lane's eight weights, 0 behind the row's end.
template <bool VECTOR>
__device__ __forceinline__ void weights8(const Weight& w, int D, int chunk, float (&v)[8]) {
  const int at = Tile<float, VECTOR, 1>::column(chunk, 0);
  if (VECTOR && w.aligned && at + 8 <= D) {
    if (w.dtype == MTS_DTYPE_FP32) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w.w) + at)), b = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w.w) + at) + 1);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(static_cast<const __half*>(w.w) + at));
      const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 f = w.dtype == MTS_DTYPE_FP16 ? unpack2<__half>(u[k]) : unpack2<__nv_bfloat16>(u[k]);
        v[2 * k] = f.x;
        v[2 * k + 1] = f.y;
      }
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int j = Tile<float, VECTOR, 1>::column(chunk, e);
    v[e] = 0.f;
    if (j < D) v[e] = w.dtype == MTS_DTYPE_FP32 ? __ldg(static_cast<const float*>(w.w) + j)
                    : w.dtype == MTS_DTYPE_FP16 ? to_f32(__ldg(static_cast<const __half*>(w.w) + j)) : to_f32(__ldg(static_cast<const __nv_bfloat16*>(w.w) + j));
  }
}

// Sum and maximum over the warps of a row, in a fixed order; `room`: shared, of this use alone.
__device__ __forceinline__ float row_sum(float x, float* room, int warp, int warps) {
  x = warp_sum(x);
  if (warps == 1) return x;
  if (lane_id() == 0) room[warp] = x;
  __syncthreads();
  return warp_sum(lane_id() < warps ? room[lane_id()] : 0.f);
}
__device__ __forceinline__ float row_max(float x, float* room, int warp, int warps) {
  x = warp_max(x);
  if (warps == 1) return x;
  if (lane_id() == 0) room[warp] = x;
  __syncthreads();
  return warp_max(lane_id() < warps ? room[lane_id()] : 0.f);
}

template <typename T>
struct NormForward {
  const T* x;
  const T* residual;
  T* sum;
  T* out;
  uint8_t* codes;
  float* scales;
  float* inv_rms;
  int64_t x_stride, residual_stride, sum_stride, out_stride, N;
  Weight weight;
  int32_t D, group, groups;
  float eps;
};

// Eight codes of a lane.
template <bool VECTOR>
__device__ __forceinline__ void store_codes(uint8_t* row, int D, int chunk, const float (&y)[8]) {
  using Columns = Tile<float, VECTOR, 1>;
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    w[k] = __nv_cvt_float2_to_fp8x2(make_float2(y[4 * k], y[4 * k + 1]), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y[4 * k + 2], y[4 * k + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
  uint8_t* const to = row + Columns::column(chunk, 0);
  if (VECTOR && Columns::column(chunk, 8) <= D && (reinterpret_cast<uintptr_t>(to) & 7) == 0) {
    *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (Columns::column(chunk, e) < D) row[Columns::column(chunk, e)] = (uint8_t)(w[e / 4] >> 8 * (e % 4));
}

// A row by blockDim.x / 32 warps, up to 1,024 columns by each, and blockDim.y rows a block (of one warp each); everything of a row is in registers
// between its one reading and its one writing.
template <typename T, bool VECTOR, int I, int THREADS, bool CODES>
__global__ void __launch_bounds__(THREADS)
rms_norm_forward(const NormForward<T> a) {
  __shared__ float room[2][NORM_WARPS];
  const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= a.N) return;                                // a warp as a whole; blocks of several warps a row have one row
  float v[I][8];
  {
    Tile<T, VECTOR, I> x, r;
    x.load(a.x + row * a.x_stride, a.D, warp, warps);
    if (a.residual) r.load(a.residual + row * a.residual_stride, a.D, warp, warps);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      x.get(i, v[i]);
      if (a.residual) {
        float other[8];
        r.get(i, other);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = to_f32(from_f32<T>(v[i][e] + other[e]));       // the stream as it is stored
        store8<T, VECTOR>(a.sum + row * a.sum_stride, a.D, warp + i * warps, v[i]);
      }
    }
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(v[i][e], v[i][e], s);
  const float c = 1.f / sqrtf(row_sum(s, room[0], warp, warps) / a.D + a.eps);
  if (a.inv_rms && warp == 0 && lane_id() == 0) a.inv_rms[row] = c;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    float w[8];
    weights8<VECTOR>(a.weight, a.D, warp + i * warps, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * c * w[e];
    if (!CODES) store8<T, VECTOR>(a.out + row * a.out_stride, a.D, warp + i * warps, v[i]);
  }
  if constexpr (CODES) {
    const int log_part = __ffs(a.group) - 6;             // a group is 32 << log_part columns
    float all = 0.f;
    if (a.group == 0) {
#pragma unroll
      for (int i = 0; i < I; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) all = fmaxf(all, fabsf(v[i][e]));
      all = fmaxf(row_max(all, room[1], warp, warps), LEAST_MAX);
      if (warp == 0 && lane_id() == 0) a.scales[row] = all / TOP_CODE;
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int chunk = warp + i * warps;
      if (chunk * NORM_CHUNK >= a.D) continue;
      float m[8];                                        // of the group of element e
      if (a.group == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = all;
      } else if (VECTOR) {                               // a group is group / 8 neighbouring lanes
        float most = LEAST_MAX;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[i][e]));
        for (int o = 1; o < a.group / 8; o *= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = most;
        const int at = Tile<T, VECTOR, 1>::column(chunk, 0), g = at >> (log_part + 5);
        if ((at & (a.group - 1)) == 0 && g < a.groups) a.scales[row * a.groups + g] = most / TOP_CODE;
      } else {                                           // a group is all lanes of group / 32 elements
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = fmaxf(warp_max(fabsf(v[i][e])), LEAST_MAX);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          most = 0.f;
#pragma unroll
          for (int f = 0; f < 8; ++f)
            if (f >> log_part == e >> log_part) most = fmaxf(most, m[f]);
          const int g = (chunk * 8 + e) >> log_part;
          if (lane_id() == 0 && (e & ((1 << log_part) - 1)) == 0 && g < a.groups) a.scales[row * a.groups + g] = most / TOP_CODE;
          v[i][e] *= TOP_CODE / most;
        }
      }
      if (VECTOR || a.group == 0) {
        const float inverse = TOP_CODE / m[0];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] *= inverse;
      }
      store_codes<VECTOR>(a.codes + row * a.out_stride, a.D, chunk, v[i]);
    }
  }
}

// Eight codes a thread where rows and codes lie on boundaries of eight, else one.
template <typename T, bool VECTOR>
__global__ void __launch_bounds__(256)
rows_from_8bit(const uint8_t* __restrict__ codes, int64_t codes_stride, const float* __restrict__ scales, int group, int groups, int D, T* __restrict__ out,
               int64_t out_stride, int64_t N, int pieces) {
  constexpr int E = VECTOR ? 8 : 1;
  // threads lie along the columns, then along the rows
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = item <= UINT32_MAX ? (uint32_t)item / (uint32_t)pieces : item / pieces;
  const int j = (int)(item - row * pieces) * E;
  if (row >= N) return;
  const float scale = scales[group ? row * groups + j / group : row];
  const uint8_t* from = codes + row * codes_stride + j;
  T* to = out + row * out_stride + j;
  if (VECTOR && j + 8 <= D) {
    const uint2 w = __ldcs(reinterpret_cast<const uint2*>(from));
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((k < 2 ? w.x : w.y) >> 16 * (k % 2)), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      v[2 * k] = f.x * scale;
      v[2 * k + 1] = f.y * scale;
    }
    if constexpr (sizeof(T) == 4) {
      __stcs(reinterpret_cast<float4*>(to), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4*>(to) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
      __stcs(reinterpret_cast<uint4*>(to), make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])));
    }
    return;
  }
  for (int e = 0; e < E && j + e < D; ++e) to[e] = from_f32<T>(__half2float(__half(__nv_cvt_fp8_to_halfraw(from[e], __NV_E4M3))) * scale);
}

constexpr int NORM_BACK_ROWS = 8;                        // of a block whose rows are one warp's
constexpr int NORM_BACK_BLOCKS = 592;                    // at most: each leaves a row of partial sums of the weight's gradient

template <typename T>
struct NormBackward {
  const T* x;
  const float* inv_rms;
  const T* grad_out;
  const T* grad_sum;
  T* grad_x;
  float* partial;
  int64_t x_stride, out_stride, sum_stride, gx_stride, N;
  Weight weight;
  int32_t D;
};

// As many blocks as the GPU holds walk over the rows; each thread keeps the sums of its columns of the weight's gradient in registers.
template <typename T, bool VECTOR, int I, int THREADS>
__global__ void __launch_bounds__(THREADS)
rms_norm_backward(const NormBackward<T> a) {
  __shared__ float room[2][NORM_WARPS];
  __shared__ float columns[NORM_BACK_ROWS][NORM_CHUNK];
  const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
  float acc[I][8] = {};
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; row < a.N; row += (int64_t)gridDim.x * blockDim.y, turn ^= 1) {
    Tile<T, VECTOR, I> x, g, t;
    x.load(a.x + row * a.x_stride, a.D, warp, warps);
    g.load(a.grad_out + row * a.out_stride, a.D, warp, warps);
    if (a.grad_sum) t.load(a.grad_sum + row * a.sum_stride, a.D, warp, warps);
    const float c = a.inv_rms[row];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      float r[8], dy[8], w[8];
      x.get(i, r);
      g.get(i, dy);
      weights8<VECTOR>(a.weight, a.D, warp + i * warps, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(dy[e] * w[e], r[e], s);
    }
    const float m = row_sum(s, room[turn], warp, warps) / a.D * (c * c);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      float r[8], dy[8], w[8], d[8];
      x.get(i, r);
      g.get(i, dy);
      weights8<VECTOR>(a.weight, a.D, warp + i * warps, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        d[e] = c * (dy[e] * w[e] - r[e] * m);
        acc[i][e] = fmaf(dy[e], r[e] * c, acc[i][e]);
      }
      if (a.grad_sum) {
        float other[8];
        t.get(i, other);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] += other[e];
      }
      store8<T, VECTOR>(a.grad_x + row * a.gx_stride, a.D, warp + i * warps, d);
    }
  }
  if (!a.partial) return;
  float* const to = a.partial + (int64_t)blockIdx.x * a.D;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int chunk = warp + i * warps;
    if (blockDim.y == 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (Tile<T, VECTOR, 1>::column(chunk, e) < a.D) to[Tile<T, VECTOR, 1>::column(chunk, e)] = acc[i][e];
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) columns[threadIdx.y][Tile<T, VECTOR, 1>::column(0, e)] = acc[i][e];
    __syncthreads();
    const int j = threadIdx.y * 32 + lane_id();          // 256 threads, a column each
    float sum = 0.f;
#pragma unroll
    for (int y = 0; y < NORM_BACK_ROWS; ++y) sum += columns[y][j];
    if (chunk * NORM_CHUNK + j < a.D) to[chunk * NORM_CHUNK + j] = sum;
  }
}

// The blocks' sums, 32 columns a block, in 64 bits.
__global__ void __launch_bounds__(1024)
rms_norm_weight_gradient(const float* __restrict__ partial, int blocks, int D, float* __restrict__ grad_weight) {
  __shared__ double room[32][33];
  const int j = blockIdx.x * 32 + threadIdx.x;
  double s = 0.0;
  if (j < D)
    for (int b = threadIdx.y; b < blocks; b += 32) s += partial[(int64_t)b * D + j];
  room[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = room[threadIdx.x][threadIdx.y];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < D) grad_weight[blockIdx.x * 32 + threadIdx.y] = (float)s;
}

}  // namespace mts

using namespace mts;

namespace {

constexpr int64_t NORM_MAX_N = (1ll << 31) - 1;

int check_norm(const char* what, int32_t dtype, int32_t weight_dtype, const void* weight, int64_t N, int32_t D) {
  if (!known_dtype(dtype) || !known_dtype(weight_dtype)) return set_error(MTS_ERR_INVALID_ARG, "%s: dtype %d, weight dtype %d", what, dtype, weight_dtype);
  if (N < 0 || D < 1) return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, D %d", what, (long long)N, D);
  if (N > NORM_MAX_N || D > MTS_RMS_NORM_MAX_D) return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, D %d", what, (long long)N, D);
  if (!weight) return set_error(MTS_ERR_INVALID_ARG, "%s: null weight", what);
  if ((uintptr_t)weight % dtype_bytes(weight_dtype)) return set_error(MTS_ERR_ALIGNMENT, "%s: weight is no multiple of its element size", what);
  return MTS_OK;
}

int check_group(const char* what, int32_t group) {
  if (group != 0 && group != 32 && group != 64 && group != 128 && group != 256)
    return set_error(MTS_ERR_INVALID_ARG, "%s: groups of %d columns (0, 32, 64, 128 or 256)", what, group);
  return MTS_OK;
}

Weight weight_of(const void* w, int32_t dtype) { return {w, dtype, ((uintptr_t)w & 15) == 0}; }

// Bits of the places where rows start.
uintptr_t rows_bits(const void* p, int64_t stride, int32_t dtype) { return (uintptr_t)p | (uintptr_t)(stride * dtype_bytes(dtype)); }

// Warps of a row, chunks of each (1, 2 or 4), and rows of a block.
struct RowShape { int warps, chunks, rows; };
RowShape shape_of(int64_t N, int32_t D, int rows) {
  const int chunks = (D + NORM_CHUNK - 1) / NORM_CHUNK;
  if (chunks <= NORM_CHUNKS) return {1, chunks <= 2 ? chunks : 4, rows};
  return {(chunks + NORM_CHUNKS - 1) / NORM_CHUNKS, 4, 1};
}

// Calls fn(whether rows are on vector boundaries, chunks of a warp, threads of a block at most) with constants.
template <typename Fn>
void with_shape(bool vector, const RowShape& shape, Fn&& fn) {
  using std::integral_constant;
  const auto with_chunks = [&](auto v) {
    if (shape.chunks == 1) fn(v, integral_constant<int, 1>(), integral_constant<int, 256>());
    else if (shape.chunks == 2) fn(v, integral_constant<int, 2>(), integral_constant<int, 256>());
    else if (shape.warps <= 8) fn(v, integral_constant<int, 4>(), integral_constant<int, 256>());
    else if (shape.warps <= 16) fn(v, integral_constant<int, 4>(), integral_constant<int, 512>());
    else fn(v, integral_constant<int, 4>(), integral_constant<int, 1024>());
  };
  if (vector) with_chunks(std::true_type());
  else with_chunks(std::false_type());
}

int norm_forward(const char* what, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                 int32_t weight_dtype, int32_t dtype, int64_t N, int32_t D, float eps, void* sum_out, int64_t sum_stride, void* out, uint8_t* codes,
                 int64_t out_stride, float* scales, int32_t group, float* inv_rms, void* stream) {
  int rc = check_norm(what, dtype, weight_dtype, weight, N, D);
  if (rc == MTS_OK && !(eps >= 0.f && eps <= 3.4e38f)) rc = set_error(MTS_ERR_INVALID_ARG, "%s: eps %g", what, eps);
  if (rc == MTS_OK && !residual != !sum_out) rc = set_error(MTS_ERR_INVALID_ARG, "%s: a residual and the sum's place come together", what);
  if (rc == MTS_OK) rc = check_rows(what, "x", x, dtype, N, D, x_stride);
  if (rc == MTS_OK && residual) rc = check_rows(what, "residual", residual, dtype, N, D, residual_stride);
  if (rc == MTS_OK && sum_out) rc = check_rows(what, "sum_out", sum_out, dtype, N, D, sum_stride);
  if (rc == MTS_OK && !codes) rc = check_rows(what, "out", out, dtype, N, D, out_stride);
  if (rc == MTS_OK && (uintptr_t)inv_rms & 3) rc = set_error(MTS_ERR_ALIGNMENT, "%s: inv_rms is no multiple of its element size", what);
  if (rc != MTS_OK || N == 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    const int32_t groups = group ? (D + group - 1) / group : 1;
    const NormForward<T> a = {static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<T*>(sum_out), static_cast<T*>(out), codes, scales, inv_rms,
                              x_stride, residual_stride, sum_stride, out_stride, N, weight_of(weight, weight_dtype), D, group, groups, eps};
    const uintptr_t bits = rows_bits(x, x_stride, dtype) | (residual ? rows_bits(residual, residual_stride, dtype) | rows_bits(sum_out, sum_stride, dtype) : 0) |
                           (codes ? 0 : rows_bits(out, out_stride, dtype));
    const RowShape shape = shape_of(N, D, 8);
    const dim3 block(32 * shape.warps, shape.rows);
    const unsigned grid = (unsigned)ceil_div(N, shape.rows);
    LaunchScope scope(K_NORM_FWD, s);
    with_shape(bits % 16 == 0, shape, [&](auto vector, auto chunks, auto threads) {
      constexpr bool V = decltype(vector)::value;
      constexpr int I = decltype(chunks)::value, TH = decltype(threads)::value;
      if (codes) rms_norm_forward<T, V, I, TH, true><<<grid, block, 0, s>>>(a);
      else rms_norm_forward<T, V, I, TH, false><<<grid, block, 0, s>>>(a);
    });
    return check_launch(what);
  });
}

}  // namespace

extern "C" int mts_rms_norm_forward(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                                    int32_t weight_dtype, int32_t dtype, int64_t N, int32_t D, float eps, void* sum_out, int64_t sum_stride,
                                    void* out, int64_t out_stride, float* inv_rms, void* stream) {
  return norm_forward("rms_norm_forward", x, x_stride, residual, residual_stride, weight, weight_dtype, dtype, N, D, eps, sum_out, sum_stride, out,
                      nullptr, out_stride, nullptr, 0, inv_rms, stream);
}

extern "C" int mts_rms_norm_forward_8bit(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight,
                                         int32_t weight_dtype, int32_t dtype, int64_t N, int32_t D, float eps, void* sum_out, int64_t sum_stride,
                                         uint8_t* codes, int64_t codes_stride, float* scales, int32_t group, float* inv_rms, void* stream) {
  const char* what = "rms_norm_forward_8bit";
  int rc = check_group(what, group);
  if (rc == MTS_OK && N > 0 && (!codes || !scales)) rc = set_error(MTS_ERR_INVALID_ARG, "%s: null codes or scales", what);
  if (rc == MTS_OK && N > 1 && codes_stride < D) rc = set_error(MTS_ERR_INVALID_ARG, "%s: rows of codes are %lld apart, less than %d", what, (long long)codes_stride, D);
  if (rc == MTS_OK && (uintptr_t)scales & 3) rc = set_error(MTS_ERR_ALIGNMENT, "%s: scales is no multiple of its element size", what);
  if (rc != MTS_OK) return rc;
  uint8_t none;                                        // without rows the codes may be null; the checks of the other form are not for them
  return norm_forward(what, x, x_stride, residual, residual_stride, weight, weight_dtype, dtype, N, D, eps, sum_out, sum_stride, nullptr,
                      codes ? codes : &none, codes_stride, scales, group, inv_rms, stream);
}

extern "C" int mts_rows_from_8bit(const uint8_t* codes, int64_t codes_stride, const float* scales, int32_t group, int64_t N, int32_t D, void* out,
                                  int32_t out_dtype, int64_t out_stride, void* stream) {
  const char* what = "rows_from_8bit";
  int rc = check_group(what, group);
  if (rc != MTS_OK) return rc;
  if (!known_dtype(out_dtype) || N < 0 || D < 1) return set_error(MTS_ERR_INVALID_ARG, "%s: dtype %d, N %lld, D %d", what, out_dtype, (long long)N, D);
  if (N > NORM_MAX_N || D > MTS_RMS_NORM_MAX_D) return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, D %d", what, (long long)N, D);
  if (N > 0 && (!codes || !scales)) return set_error(MTS_ERR_INVALID_ARG, "%s: null codes or scales", what);
  if (N > 1 && codes_stride < D) return set_error(MTS_ERR_INVALID_ARG, "%s: rows of codes are %lld apart, less than %d", what, (long long)codes_stride, D);
  if ((uintptr_t)scales & 3) return set_error(MTS_ERR_ALIGNMENT, "%s: scales is no multiple of its element size", what);
  rc = check_rows(what, "out", out, out_dtype, N, D, out_stride);
  if (rc != MTS_OK || N == 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_dtype(out_dtype, [&](auto t) {
    using T = decltype(t);
    const bool vector = (rows_bits(out, out_stride, out_dtype) % 16 | (uintptr_t)codes % 8 | (uintptr_t)codes_stride % 8) == 0;
    const int groups = group ? (D + group - 1) / group : 1, pieces = vector ? (D + 7) / 8 : D;
    const int64_t blocks = ceil_div(N * pieces, 256);
    if (blocks > INT32_MAX) return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, D %d", what, (long long)N, D);
    LaunchScope scope(K_NORM_FWD, s);
    if (vector) rows_from_8bit<T, true><<<(unsigned)blocks, 256, 0, s>>>(codes, codes_stride, scales, group, groups, D, static_cast<T*>(out), out_stride, N, pieces);
    else rows_from_8bit<T, false><<<(unsigned)blocks, 256, 0, s>>>(codes, codes_stride, scales, group, groups, D, static_cast<T*>(out), out_stride, N, pieces);
    return check_launch(what);
  });
}

extern "C" size_t mts_rms_norm_workspace_bytes(int64_t N, int32_t D) {
  if (N < 0 || D < 1 || N > NORM_MAX_N || D > MTS_RMS_NORM_MAX_D) return 0;
  return align_up(sizeof(float) * (size_t)(N < NORM_BACK_BLOCKS ? (N > 0 ? N : 1) : NORM_BACK_BLOCKS) * D, 256);
}

extern "C" int mts_rms_norm_backward(const void* x, int64_t x_stride, const void* weight, int32_t weight_dtype, int32_t dtype, int64_t N, int32_t D,
                                     const float* inv_rms, const void* grad_out, int64_t grad_out_stride, const void* grad_sum,
                                     int64_t grad_sum_stride, void* grad_x, int64_t grad_x_stride, float* grad_weight, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  const char* what = "rms_norm_backward";
  int rc = check_norm(what, dtype, weight_dtype, weight, N, D);
  if (rc == MTS_OK) rc = check_rows(what, "x", x, dtype, N, D, x_stride);
  if (rc == MTS_OK) rc = check_rows(what, "grad_out", grad_out, dtype, N, D, grad_out_stride);
  if (rc == MTS_OK && grad_sum) rc = check_rows(what, "grad_sum", grad_sum, dtype, N, D, grad_sum_stride);
  if (rc == MTS_OK) rc = check_rows(what, "grad_x", grad_x, dtype, N, D, grad_x_stride);
  if (rc == MTS_OK && N > 0 && !inv_rms) rc = set_error(MTS_ERR_INVALID_ARG, "%s: null inv_rms", what);
  if (rc == MTS_OK && (((uintptr_t)inv_rms | (uintptr_t)grad_weight) & 3)) rc = set_error(MTS_ERR_ALIGNMENT, "%s: a pointer is no multiple of its element size", what);
  if (rc != MTS_OK) return rc;
  if (grad_weight) {
    const size_t need = mts_rms_norm_workspace_bytes(N, D);
    if (!workspace || workspace_bytes < need) return set_error(MTS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed", what, workspace_bytes, need);
    if ((uintptr_t)workspace & 255) return set_error(MTS_ERR_ALIGNMENT, "%s: the workspace must be 256-byte aligned", what);
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N == 0) return grad_weight ? check_cuda(cudaMemsetAsync(grad_weight, 0, sizeof(float) * (size_t)D, s), "cudaMemsetAsync(grad_weight)") : MTS_OK;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    float* partial = grad_weight ? static_cast<float*>(workspace) : nullptr;
    const NormBackward<T> a = {static_cast<const T*>(x), inv_rms, static_cast<const T*>(grad_out), static_cast<const T*>(grad_sum), static_cast<T*>(grad_x), partial,
                               x_stride, grad_out_stride, grad_sum_stride, grad_x_stride, N, weight_of(weight, weight_dtype), D};
    const uintptr_t bits = rows_bits(x, x_stride, dtype) | rows_bits(grad_out, grad_out_stride, dtype) | (grad_sum ? rows_bits(grad_sum, grad_sum_stride, dtype) : 0) |
                           rows_bits(grad_x, grad_x_stride, dtype);
    const RowShape shape = shape_of(N, D, NORM_BACK_ROWS);
    const int64_t wanted = ceil_div(N, shape.rows), most = shape.warps == 1 ? 296 : shape.warps <= 4 ? 592 : shape.warps <= 8 ? 296 : 148;
    const int blocks = (int)(wanted < most ? wanted : most);
    {
      LaunchScope scope(K_NORM_BWD, s);
      with_shape(bits % 16 == 0, shape, [&](auto vector, auto chunks, auto threads) {
        rms_norm_backward<T, decltype(vector)::value, decltype(chunks)::value, decltype(threads)::value><<<blocks, dim3(32 * shape.warps, shape.rows), 0, s>>>(a);
      });
    }
    int e = check_launch(what);
    if (e != MTS_OK || !grad_weight) return e;
    LaunchScope scope(K_NORM_BWD, s);
    rms_norm_weight_gradient<<<(unsigned)ceil_div(D, 32), dim3(32, 32), 0, s>>>(partial, blocks, D, grad_weight);
    return check_launch(what);
  });
}
