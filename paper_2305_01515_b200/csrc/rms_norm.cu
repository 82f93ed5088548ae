// Root-mean-square norm of the residual stream, forward (output in the tensors' type or in 8 bits) and backward.
//
//   r = round(x + residual),  c = 1 / sqrt(mean_j r_j^2 + eps),  y_j = r_j c w_j;  in 8 bits code_j = e4m3(r_j w_j 448 / max |r w|), scale = c max |r w| / 448
//   dx_j = dr_j + c (dy_j w_j - r_j a),  a = c^2 mean_j(dy_j w_j r_j),   dw_j = sum over rows of dy_j r_j c
//
// Memory bounds it: six operations an element forward, a dozen backward.  So a row is read once, held in registers until its sum is known, and written
// once; the sum of squares, of dw and everything between is fp32 (dw's parts of blocks are added in fp64), and each output is rounded to its type once.  r is rounded before it is
// normalised because that is the stream which the next layer and the backward see.
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
// boundaries); else every 32nd column, which any row can be read by in whole sectors.  Columns behind the row's end hold 0.  LANES: lanes of a row,
// fewer than 32 where rows are short and on boundaries.
template <typename T, bool VECTOR, int I, int LANES = 32>
struct Tile {
  static constexpr int Q = VECTOR ? (int)sizeof(T) / 2 : 1;
  uint4 q[VECTOR ? I : 1][Q];
  T s[VECTOR ? 1 : I][8];

  static __device__ __forceinline__ int column(int chunk, int e) { return chunk * NORM_CHUNK + (VECTOR ? lane_id() % LANES * 8 + e : lane_id() + 32 * e); }
  __device__ __forceinline__ void load(const T* row, int D, int chunk, int step) {
#pragma unroll
    for (int i = 0; i < I; ++i, chunk += step) {
      if constexpr (VECTOR) {
        constexpr int P = 8 / Q;                         // elements of 16 bytes
#pragma unroll
        for (int k = 0; k < Q; ++k) {
          const int at = column(chunk, k * P);
          if (at + P <= D) {
            q[i][k] = *reinterpret_cast<const uint4*>(row + at);
          } else {
            q[i][k] = make_uint4(0u, 0u, 0u, 0u);
            T* const e = reinterpret_cast<T*>(&q[i][k]);
#pragma unroll
            for (int p = 0; p < P; ++p)
              if (at + p < D) e[p] = row[at + p];
          }
        }
      } else {
        const T* const p = row + column(chunk, 0);
        const int left = D - column(chunk, 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = left > 32 * e ? p[32 * e] : from_f32<T>(0.f);
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
template <typename T, bool VECTOR, int LANES>
__device__ __forceinline__ void store8(T* row, int D, int chunk, const float (&v)[8]) {
  using Columns = Tile<T, VECTOR, 1, LANES>;
  if constexpr (VECTOR) {
    constexpr int Q = (int)sizeof(T) / 2, P = 8 / Q;
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const int at = Columns::column(chunk, k * P);
      if (at + P <= D) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(row + at) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        else *reinterpret_cast<uint4*>(row + at) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
          if (at + p < D) row[at + p] = from_f32<T>(v[k * P + p]);
      }
    }
    return;
  }
  T* const p = row + Columns::column(chunk, 0);
  const int left = D - Columns::column(chunk, 0);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (left > 32 * e) p[32 * e] = from_f32<T>(v[e]);
}

struct Weight {
  const void* w;
  int32_t dtype, aligned;                                // aligned: on a 16-byte boundary
};

// A lane's eight weights, 0 behind the row's end.
template <bool VECTOR, int LANES>
__device__ __forceinline__ void weights8(const Weight& w, int D, int chunk, float (&v)[8]) {
  const int at = Tile<float, VECTOR, 1, LANES>::column(chunk, 0);
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
  constexpr int STEP = VECTOR ? 1 : 32;
  const auto one_by_one = [&](auto* p) {
    p += at;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = D - at > STEP * e ? to_f32(__ldg(p + STEP * e)) : 0.f;
  };
  if (w.dtype == MTS_DTYPE_FP32) one_by_one(static_cast<const float*>(w.w));
  else if (w.dtype == MTS_DTYPE_FP16) one_by_one(static_cast<const __half*>(w.w));
  else one_by_one(static_cast<const __nv_bfloat16*>(w.w));
}

// Sum and maximum over the lanes, or the warps, of a row, in a fixed order; `room`: shared, of this row and use alone.
__device__ __forceinline__ void row_barrier(int warps) { __barrier_sync_count(threadIdx.y + 1, 32 * warps); }
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* room, int warp, int warps) {
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  if (LANES < 32 || warps == 1) return x;
  if (lane_id() == 0) room[warp] = x;
  row_barrier(warps);
  return warp_sum(lane_id() < warps ? room[lane_id()] : 0.f);
}
template <int LANES>
__device__ __forceinline__ float row_max(float x, float* room, int warp, int warps) {
  if constexpr (LANES == 32) {
    x = warp_max(x);
  } else {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  }
  if (LANES < 32 || warps == 1) return x;
  if (lane_id() == 0) room[warp] = x;
  row_barrier(warps);
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

// A group's scale, and what its values are multiplied with for their codes; `most`: the largest of them, without the factor c.
__device__ __forceinline__ float scale_of(float most, float c) { return fmaxf(most * c, LEAST_MAX) / TOP_CODE; }
__device__ __forceinline__ float inverse_of(float most, float c) {
  constexpr float MOST_C = 5.9e5f;                       // with more the product has no number (infinite and NaN as they are)
  return most * c >= LEAST_MAX ? TOP_CODE / most : TOP_CODE / LEAST_MAX * (c > MOST_C && c < INFINITY ? MOST_C : c);
}

// Eight codes of a lane.
template <bool VECTOR, int LANES>
__device__ __forceinline__ void store_codes(uint8_t* row, int D, int chunk, const float (&y)[8]) {
  using Columns = Tile<float, VECTOR, 1, LANES>;
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

// A row by blockDim.x / 32 warps, up to 1,024 columns by each, or R rows by a warp (times 32 / LANES), so that a warp has four chunks on their way
// whatever the width; blockDim.y such sets a block.  Everything of a row is in registers between its one reading and its one writing.
// us, with a residual: 131,072 x 1,024 bf16 162 (6.63 TB/s, the copy rate); 8,192 x 8,192 to 8 bits, groups of 128, 95 (4.8 TB/s: issue slots 72% busy with the
// codes and their maxima); 120,007 x 256 to 8 bits 45 (4.8 TB/s); 2,000 x 32,768 106 (one block of 1,024 threads an SM, 5.0 TB/s).  100,003 x 333 fp32 without, off
// boundaries, 52 (5.1 TB/s): single elements, and the last chunk's 179 places that hold none.
template <typename T, bool VECTOR, int R, int I, int LANES, int THREADS, bool CODES>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 1 : (VECTOR && sizeof(T) == 2) || R * I <= 2 ? 4 : 2)
rms_norm_forward(const NormForward<T> a) {
  using Columns = Tile<T, VECTOR, 1, LANES>;
  __shared__ float room[2][NORM_WARPS];
  const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
  const int64_t first = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * (R * (32 / LANES)) + lane_id() / LANES;
  if (first - lane_id() / LANES >= a.N) return;          // a warp as a whole; blocks of several warps a row have one row
  float v[R][I][8], c[R];
  int64_t row[R];
  int D[R];                                              // no columns where there is no row
#pragma unroll
  for (int r = 0; r < R; ++r) {
    row[r] = first + r * (32 / LANES);
    D[r] = row[r] < a.N ? a.D : 0;
    if (row[r] >= a.N) row[r] = a.N - 1;
  }
  {
    Tile<T, VECTOR, I, LANES> x[R], other[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      x[r].load(a.x + row[r] * a.x_stride, D[r], warp, warps);
      if (a.residual) other[r].load(a.residual + row[r] * a.residual_stride, D[r], warp, warps);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < I; ++i) {
        x[r].get(i, v[r][i]);
        if (a.residual) {
          float o[8];
          other[r].get(i, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[r][i][e] = to_f32(from_f32<T>(v[r][i][e] + o[e]));     // the stream as it is stored
          store8<T, VECTOR, LANES>(a.sum + row[r] * a.sum_stride, D[r], warp + i * warps, v[r][i]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(v[r][i][e], v[r][i][e], s);
    c[r] = 1.f / sqrtf(row_sum<LANES>(s, room[0], warp, R == 1 ? warps : 1) / a.D + a.eps);
    if (a.inv_rms && warp == 0 && lane_id() % LANES == 0 && D[r]) a.inv_rms[row[r]] = c[r];
  }
  // In 8 bits c cancels out of the codes and goes to the scales alone: which code a value between two has depends on x and weight, not on the last bit of a sum over the row.
#pragma unroll
  for (int i = 0; i < I; ++i) {
    float w[8];
    weights8<VECTOR, LANES>(a.weight, a.D, warp + i * warps, w);
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int e = 0; e < 8; ++e) if (CODES) v[r][i][e] *= w[e]; else v[r][i][e] = v[r][i][e] * c[r] * w[e];
      if (!CODES) store8<T, VECTOR, LANES>(a.out + row[r] * a.out_stride, D[r], warp + i * warps, v[r][i]);
    }
  }
  if constexpr (CODES) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float inverse = 0.f;
      if (a.group == 0) {
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) all = fmaxf(all, fabsf(v[r][i][e]));
        all = row_max<LANES>(all, room[1], warp, R == 1 ? warps : 1);
        if (warp == 0 && lane_id() % LANES == 0 && D[r]) a.scales[row[r]] = scale_of(all, c[r]);
        inverse = inverse_of(all, c[r]);
      }
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int chunk = warp + i * warps;
        if (chunk * NORM_CHUNK >= a.D) continue;
        float(&y)[8] = v[r][i];
        if (a.group == 0 || VECTOR) {
          if (a.group) {                                 // a group is group / 8 neighbouring lanes
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(y[e]));
            for (int o = 1; o < min(a.group / 8, LANES); o *= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
            inverse = inverse_of(most, c[r]);
            const int at = Columns::column(chunk, 0), g = at >> (__ffs(a.group) - 1);
            if ((at & (a.group - 1)) == 0 && at < D[r]) a.scales[row[r] * a.groups + g] = scale_of(most, c[r]);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] *= inverse;
        } else {                                         // a group is all lanes of group / 32 elements
          const auto groups_of = [&](auto part) {
            constexpr int PART = decltype(part)::value;
#pragma unroll
            for (int p = 0; p < 8; p += PART) {
              float most = 0.f;
#pragma unroll
              for (int e = 0; e < PART; ++e) most = fmaxf(most, fabsf(y[p + e]));
              most = warp_max(most);
              const float inverse_of_group = inverse_of(most, c[r]);
#pragma unroll
              for (int e = 0; e < PART; ++e) y[p + e] *= inverse_of_group;
              const int g = (chunk * 8 + p) / PART;
              if (lane_id() == 0 && g < a.groups && D[r]) a.scales[row[r] * a.groups + g] = scale_of(most, c[r]);
            }
          };
          if (a.group == 32) groups_of(std::integral_constant<int, 1>());
          else if (a.group == 64) groups_of(std::integral_constant<int, 2>());
          else if (a.group == 128) groups_of(std::integral_constant<int, 4>());
          else groups_of(std::integral_constant<int, 8>());
        }
        store_codes<VECTOR, LANES>(a.codes + row[r] * a.out_stride, D[r], chunk, y);
      }
    }
  }
}

// Pieces of eight codes where rows and codes lie on boundaries of eight, else single ones: 1 << log_threads threads a row, U pieces on their way for each.
// 120,007 x 256 codes to bf16: 21 us (4.4 TB/s); 20,011 x 5,000: 58 (5.2).
template <typename T, bool VECTOR, int U>
__global__ void __launch_bounds__(256)
rows_from_8bit(const uint8_t* __restrict__ codes, int64_t codes_stride, const float* __restrict__ scales, int group, int groups, int D, T* __restrict__ out,
               int64_t out_stride, int64_t N, int log_threads) {
  constexpr int E = VECTOR ? 8 : 1;
  const int64_t row = ((int64_t)blockIdx.x << (8 - log_threads)) + (threadIdx.x >> log_threads);
  if (row >= N) return;
  const uint8_t* from = codes + row * codes_stride;
  T* to = out + row * out_stride;
  const int shift = group ? __ffs(group) - 1 : 31;       // 0: all columns are of group 0
  const float* scale = scales + row * groups;
  for (int j0 = (threadIdx.x & ((1 << log_threads) - 1)) * E; j0 < D; j0 += (U * E) << log_threads) {
    uint2 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + (u << log_threads) * E;
      if (VECTOR && j + 8 <= D) w[u] = __ldcs(reinterpret_cast<const uint2*>(from + j));
      else if (j < D) w[u].x = from[j];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + (u << log_threads) * E;
      if (j >= D) break;
      const float s = __ldg(scale + (j >> shift));
      if (VECTOR && j + 8 <= D) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((k < 2 ? w[u].x : w[u].y) >> 16 * (k % 2)), __NV_E4M3);
          const float2 f = __half22float2(__half2(h));
          v[2 * k] = f.x * s;
          v[2 * k + 1] = f.y * s;
        }
        if constexpr (sizeof(T) == 4) {
          __stcs(reinterpret_cast<float4*>(to + j), make_float4(v[0], v[1], v[2], v[3]));
          __stcs(reinterpret_cast<float4*>(to + j) + 1, make_float4(v[4], v[5], v[6], v[7]));
        } else {
          __stcs(reinterpret_cast<uint4*>(to + j), make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])));
        }
      } else {
        for (int e = 0; e < E && j + e < D; ++e)
          to[j + e] = from_f32<T>(__half2float(__half(__nv_cvt_fp8_to_halfraw(e ? from[j + e] : (uint8_t)w[u].x, __NV_E4M3))) * s);
      }
    }
  }
}

constexpr int NORM_BACK_WARPS = 16;                      // of a row at most
static_assert(NORM_BACK_WARPS * NORM_CHUNK * 8 >= MTS_RMS_NORM_MAX_D, "eight chunks a warp hold the widest row");
constexpr int NORM_BACK_BLOCKS = 444;                    // at most: each leaves a row of partial sums of the weight's gradient

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

// As many blocks as the GPU holds walk over the rows (shaped as in the forward, with two chunks a warp while there are warps enough: three arrays are in
// registers); each thread keeps the sums of its columns of the weight's gradient, and the blocks' sums are added by the kernel below: no atomics, so that
// results are the same in every run.  131,072 x 1,024 bf16 with the stream's gradient: 197-207 us (5.2-5.5 TB/s of what moves); 100,003 x 333 fp32 86-92 (4.3-4.6).
// Four chunks a warp and a third fewer warps took 272 us there, one chunk a warp 200 for 332 fp32 columns (93-98 with two).
// A thread has 80 registers where rows come in vectors of 16-bit elements and a warp has two chunks, 128 else, and spills none: no instance has a stack.  A row has 16 warps at
// most; where two chunks for each do not hold it they have four or eight.  Where the arrays of these do not fit (HELD false) they are read again for the second part,
// from L1 or L2 where the row has just passed.  us: 10,000 x 5,000 bf16 117 (3 arrays, 2.6 TB/s), 6,000 x 16,384 242 (with the stream's gradient, 3.3), 3,000 x 32,768 264 and 332
// (2.2 and 2.4); fp32 8,000 x 4,099 135 (2.9), 6,000 x 8,192 141 (4.2), 5,000 x 10,001 195 (3.1); 5,000 x 10,001 fp16 188 (1.6).
template <typename T>
__host__ __device__ constexpr int back_blocks(bool vector) { return vector && sizeof(T) == 2 ? 3 : 2; }       // of 256 threads on an SM, two chunks a warp
// Warps of a row at most while they have two chunks each.
template <typename T>
__host__ __device__ constexpr int back_warps(bool vector) { return vector && sizeof(T) == 2 ? 12 : NORM_BACK_WARPS; }
template <typename T, bool VECTOR, int R, int I, int LANES, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? back_blocks<T>(VECTOR) : THREADS == 384 ? 2 : 1)
rms_norm_backward(const NormBackward<T> a) {
  using Columns = Tile<T, VECTOR, 1, LANES>;
  __shared__ float room[2][NORM_WARPS];
  __shared__ float columns[8][NORM_CHUNK];               // of 8 warps
  const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
  float acc[I][8] = {};
  int turn = 0;
  // A warp's i-th chunk; eight of them would have their addresses kept from row to row, for which there are no registers.
  const auto chunk_of = [&](int i) {
    int chunk = warp + i * warps;
    if (I == 8) asm volatile("" : "+r"(chunk));
    return chunk;
  };
  constexpr int SET = R * (32 / LANES);                  // rows of a warp
  constexpr bool HELD = I <= (VECTOR && sizeof(T) == 2 ? 4 : 2);      // in registers between the two parts
  constexpr bool LATE = HELD && I == 4;                  // but for the stream's gradient, which the second part reads
  const int64_t step = (int64_t)gridDim.x * blockDim.y * SET;
  for (int64_t set = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * SET; set < a.N; set += step, turn ^= 1) {
    Tile<T, VECTOR, HELD ? I : 1, LANES> x[R], g[R];
    Tile<T, VECTOR, HELD && !LATE ? I : 1, LANES> t[R];
    float c[R], m[R];
    int64_t row[R];
    int D[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      row[r] = set + r * (32 / LANES) + lane_id() / LANES;
      D[r] = row[r] < a.N ? a.D : 0;
      if (row[r] >= a.N) row[r] = a.N - 1;
      if (HELD) {
        x[r].load(a.x + row[r] * a.x_stride, D[r], warp, warps);
        g[r].load(a.grad_out + row[r] * a.out_stride, D[r], warp, warps);
        if (a.grad_sum && !LATE) t[r].load(a.grad_sum + row[r] * a.sum_stride, D[r], warp, warps);
      }
      c[r] = a.inv_rms[row[r]];
      m[r] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int chunk = chunk_of(i);
      float w[8];
      weights8<VECTOR, LANES>(a.weight, a.D, chunk, w);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float y[8], dy[8];
        if (!HELD) {
          x[r].load(a.x + row[r] * a.x_stride, D[r], chunk, warps);
          g[r].load(a.grad_out + row[r] * a.out_stride, D[r], chunk, warps);
        }
        x[r].get(HELD ? i : 0, y);
        g[r].get(HELD ? i : 0, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[r] = fmaf(dy[e] * w[e], y[e], m[r]);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) m[r] = row_sum<LANES>(m[r], room[turn] + threadIdx.y * warps, warp, R == 1 ? warps : 1) / a.D * (c[r] * c[r]);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int chunk = chunk_of(i);
      float w[8];
      weights8<VECTOR, LANES>(a.weight, a.D, chunk, w);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float y[8], dy[8], d[8];
        if (!HELD) {
          x[r].load(a.x + row[r] * a.x_stride, D[r], chunk, warps);
          g[r].load(a.grad_out + row[r] * a.out_stride, D[r], chunk, warps);
        }
        x[r].get(HELD ? i : 0, y);
        g[r].get(HELD ? i : 0, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          d[e] = c[r] * (dy[e] * w[e] - y[e] * m[r]);
          acc[i][e] = fmaf(dy[e], y[e] * c[r], acc[i][e]);
        }
        if (a.grad_sum) {
          if (I == 8 && !VECTOR) asm volatile("" ::: "memory");      // not before x and dy have been used
          float o[8];
          if (!HELD || LATE) t[r].load(a.grad_sum + row[r] * a.sum_stride, D[r], chunk, warps);
          t[r].get(HELD && !LATE ? i : 0, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] += o[e];
        }
        store8<T, VECTOR, LANES>(a.grad_x + row[r] * a.gx_stride, D[r], chunk, d);
      }
    }
  }
  if (!a.partial) return;
  float* const to = a.partial + (int64_t)blockIdx.x * a.D;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    if (LANES < 32) {
#pragma unroll
      for (int o = LANES; o < 32; o *= 2)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[i][e] += __shfl_xor_sync(0xFFFFFFFFu, acc[i][e], o);
    }
    if (blockDim.y == 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (Columns::column(warp + i * warps, e) < a.D) to[Columns::column(warp + i * warps, e)] = acc[i][e];
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) columns[threadIdx.y * warps + warp][Columns::column(0, e)] = acc[i][e];
    __syncthreads();
    for (int j = threadIdx.y * blockDim.x + threadIdx.x; j < warps * NORM_CHUNK; j += blockDim.x * blockDim.y) {
      const int chunk = j / NORM_CHUNK, at = (chunk + i * warps) * NORM_CHUNK + j % NORM_CHUNK;
      float sum = 0.f;
      for (int y = 0; y < (int)blockDim.y; ++y) sum += columns[y * warps + chunk][j % NORM_CHUNK];
      if (j % NORM_CHUNK < LANES * 8 && at < a.D) to[at] = sum;
    }
  }
}

// The blocks' sums, 32 columns a block, in 64 bits (6 us).
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

// Warps of a row, chunks of each, lanes of a row, and sets (rows, or what a warp has of them) of a block.  Chunks of a warp: most_chunks, or twice and four times as
// many where that takes more than most_warps (in the backward alone, and then NORM_BACK_WARPS).
struct RowShape { int warps, chunks, lanes, sets; };
RowShape shape_of(int32_t D, bool vector, int most_chunks, int most_warps) {
  const int chunks = (D + NORM_CHUNK - 1) / NORM_CHUNK;
  if (chunks <= most_chunks) return {1, chunks <= 2 ? chunks : 4, vector && D <= 32 ? 4 : vector && D <= 64 ? 8 : vector && D <= 128 ? 16 : 32, 8};
  for (; (chunks + most_chunks - 1) / most_chunks > most_warps; most_warps = NORM_BACK_WARPS) most_chunks *= 2;
  const int warps = (chunks + most_chunks - 1) / most_chunks;
  return {warps, most_chunks, 32, most_chunks == 2 && warps <= 4 ? 8 / warps : 1};
}

// Calls fn(whether rows are on vector boundaries, rows of a warp, chunks of a row, lanes of a row, threads of a block at most) with constants.  MOST: chunks
// that a warp has on their way; `several`: several short rows for them, where T is kept in 16 bits and by vectors (else they take too many registers: 54 and 68 us
// for 100,003 x 332 in fp32 with one row and two) and there are rows for all warps (192 rows of 128 take 2 us less with one).
template <int MOST, typename T, typename Fn>
void with_shape(bool vector, bool several, const RowShape& shape, Fn&& fn) {
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  using Full = integral_constant<int, 32>;
  using Small = integral_constant<int, 256>;
  using Middle = integral_constant<int, 512>;
  using Large = integral_constant<int, 1024>;
  const bool small = shape.warps * shape.sets <= 8;
  const auto with_rows = [&](auto v, auto chunks, auto lanes) {
    if constexpr (decltype(v)::value && sizeof(T) == 2 && decltype(chunks)::value < MOST) {
      if (several) return fn(v, integral_constant<int, MOST / decltype(chunks)::value>(), chunks, lanes, Small());
    }
    return fn(v, One(), chunks, lanes, Small());
  };
  const auto with_chunks = [&](auto v) {
    if (shape.chunks == 1) return with_rows(v, One(), Full());
    if (shape.chunks == 2 && small) return with_rows(v, integral_constant<int, 2>(), Full());
    if constexpr (MOST == 4) {
      if (small) return fn(v, One(), integral_constant<int, 4>(), Full(), Small());
      return fn(v, One(), integral_constant<int, 4>(), Full(), Large());
    } else {
      if (shape.chunks == 2) return fn(v, One(), integral_constant<int, 2>(), Full(), integral_constant<int, back_warps<T>(decltype(v)::value) * 32>());
      if (shape.chunks == 4) return fn(v, One(), integral_constant<int, 4>(), Full(), Middle());
      return fn(v, One(), integral_constant<int, 8>(), Full(), Middle());
    }
  };
  if (shape.lanes == 4) with_rows(std::true_type(), One(), integral_constant<int, 4>());
  else if (shape.lanes == 8) with_rows(std::true_type(), One(), integral_constant<int, 8>());
  else if (shape.lanes == 16) with_rows(std::true_type(), One(), integral_constant<int, 16>());
  else if (vector) with_chunks(std::true_type());
  else with_chunks(std::false_type());
}

// Whether a warp has several rows, and the rows of a block.
bool several_rows(const RowShape& shape, bool vector, int32_t dtype, int64_t N, int most) {
  return vector && dtype_bytes(dtype) == 2 && shape.warps == 1 && shape.chunks < most && N >= 148ll * 32 * most * (32 / shape.lanes);
}
int rows_of(const RowShape& shape, bool several, int most) { return shape.sets * (several ? most / shape.chunks : 1) * (32 / shape.lanes); }

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
    const bool vector = bits % 16 == 0;
    const RowShape shape = shape_of(D, vector, NORM_CHUNKS, NORM_WARPS);
    const dim3 block(32 * shape.warps, shape.sets);
    const bool several = several_rows(shape, vector, dtype, N, NORM_CHUNKS);
    const unsigned grid = (unsigned)ceil_div(N, rows_of(shape, several, NORM_CHUNKS));
    LaunchScope scope(K_NORM_FWD, s);
    with_shape<NORM_CHUNKS, T>(vector, several, shape, [&](auto v, auto rows, auto chunks, auto lanes, auto threads) {
      constexpr bool V = decltype(v)::value;
      constexpr int R = decltype(rows)::value, I = decltype(chunks)::value, L = decltype(lanes)::value, TH = decltype(threads)::value;
      if (codes) rms_norm_forward<T, V, R, I, L, TH, true><<<grid, block, 0, s>>>(a);
      else rms_norm_forward<T, V, R, I, L, TH, false><<<grid, block, 0, s>>>(a);
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
    int log_threads = 0;
    while (log_threads < 8 && 1 << log_threads < pieces) ++log_threads;
    const int64_t blocks = ceil_div(N, 256 >> log_threads);
    LaunchScope scope(K_ROWS_FROM_8BIT, s);
    if (vector && pieces <= 256) rows_from_8bit<T, true, 1><<<(unsigned)blocks, 256, 0, s>>>(codes, codes_stride, scales, group, groups, D, static_cast<T*>(out), out_stride, N, log_threads);
    else if (vector) rows_from_8bit<T, true, 4><<<(unsigned)blocks, 256, 0, s>>>(codes, codes_stride, scales, group, groups, D, static_cast<T*>(out), out_stride, N, log_threads);
    else rows_from_8bit<T, false, 4><<<(unsigned)blocks, 256, 0, s>>>(codes, codes_stride, scales, group, groups, D, static_cast<T*>(out), out_stride, N, log_threads);
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
    const bool vector = bits % 16 == 0;
    const RowShape shape = shape_of(D, vector, 2, back_warps<T>(vector));
    // blocks that the GPU holds at once
    const bool several = several_rows(shape, vector, dtype, N, 2);
    const int64_t wanted = ceil_div(N, rows_of(shape, several, 2)), threads = shape.warps * shape.sets * 32;
    const int64_t most = 148 * (threads <= 256 ? (shape.chunks <= 2 ? back_blocks<T>(vector) : 2) : threads <= 384 && shape.chunks == 2 && back_warps<T>(vector) == 12 ? 2 : 1);
    const int blocks = (int)(wanted < most ? wanted : most);
    {
      LaunchScope scope(K_NORM_BWD, s);
      with_shape<2, T>(vector, several, shape, [&](auto v, auto rows, auto chunks, auto lanes, auto th) {
        rms_norm_backward<T, decltype(v)::value, decltype(rows)::value, decltype(chunks)::value, decltype(lanes)::value, decltype(th)::value>
            <<<blocks, dim3(32 * shape.warps, shape.sets), 0, s>>>(a);
      });
    }
    int e = check_launch(what);
    if (e != MTS_OK || !grad_weight) return e;
    LaunchScope scope(K_NORM_BWD, s);
    rms_norm_weight_gradient<<<(unsigned)ceil_div(D, 32), dim3(32, 32), 0, s>>>(partial, blocks, D, grad_weight);
    return check_launch(what);
  });
}
