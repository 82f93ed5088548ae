// Learned relative position bias by buckets, forward and gradient of its table.
//
//   out[h, i, j] = table[bucket(j - i - q_offset), h]
//   grad_table[k, h] = sum over b and the (i, j) of bucket k of grad_out[b, h, i, j]
//
// The bucket depends on the diagonal j - i alone.  Forward: a head's matrix is one vector of Lq + Lk - 1 values of which every row
// shows a window; what bounds it is writing the rows.  Gradient: the sum of each diagonal first, then of the diagonals of a
// bucket; what bounds it is reading the gradient.
#include <limits.h>
#include <math.h>

#include "dense.cuh"

namespace mts {

// Starts of the buckets, passed to kernels by value.
struct Buckets {
  int32_t n, two_sided, causal;
  int32_t starts[MTS_RELPOS_MAX_BUCKETS];
};

// Row of the table for distance r = key - query: the last bucket that starts at or before it.
__device__ __forceinline__ int bucket_row(const Buckets& b, int r) {
  const int d = b.two_sided ? abs(r) : max(-r, 0);
  int lo = 0, hi = b.n;                     // starts[lo] <= d < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.starts[mid] <= d) lo = mid; else hi = mid;
  }
  return b.two_sided && r > 0 ? b.n + lo : lo;
}

__device__ __forceinline__ float table_value(const void* table, int dtype, int64_t i) {
  if (dtype == MTS_DTYPE_FP32) return static_cast<const float*>(table)[i];
  if (dtype == MTS_DTYPE_FP16) return to_f32(static_cast<const __half*>(table)[i]);
  return to_f32(static_cast<const __nv_bfloat16*>(table)[i]);
}

struct BiasGeometry {
  int32_t heads, Lq, Lk, q_offset;
};

__device__ __forceinline__ float bias_value(const Buckets& b, const BiasGeometry& g, const void* table, int table_dtype, int h, int r) {
  return b.causal && r > 0 ? -INFINITY : table_value(table, table_dtype, (int64_t)bucket_row(b, r) * g.heads + h);
}

// Few rows: one element per thread and step.
template <typename T>
__global__ void __launch_bounds__(256)
relpos_forward_direct(const __grid_constant__ Buckets b, BiasGeometry g, const void* __restrict__ table, int table_dtype, T* __restrict__ out,
                      int64_t head_stride, int64_t row_stride) {
  const int h = blockIdx.z;
  for (int i = blockIdx.y; i < g.Lq; i += gridDim.y)
    for (int64_t j = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; j < g.Lk; j += (int64_t)gridDim.x * blockDim.x)
      out[h * head_stride + i * row_stride + j] = from_f32<T>(bias_value(b, g, table, table_dtype, h, (int)j - i - g.q_offset));
}

// A block writes `rows` queries x up to FWD_COLS keys of one head: bound by the bytes it writes.  It holds their part of the vector in shared memory once for each of the
// 16 / sizeof(T) positions that a 16-byte boundary can have in it, so that every row is one bulk copy to global memory from an
// aligned place of one of the copies, whatever its window and the alignment of the row; up to 15 bytes at either end of a row are
// stored by threads.  16 x 4,096 x 4,096 in bf16: 88.6 to 89.7 us, 6.0 TB/s, 92% of the copy rate (a thread per element: 1,320 us, a search of
// the buckets each); 12 x 1,023 x 1,023: 10.2 us.
//
// Blocks a call is cut into, where it has the rows.  148, 296, 592 and 1,184 take 12.4 / 12.4 / 16.4 / 16.4 us for 4 x 2,048 x 2,048 in bf16 (each
// block makes its vector) and 10.4 / 10.4 / 10.4 / 12.7 us for 12 x 1,023 x 1,023.
constexpr int FWD_WANTED = 148 * 2;
constexpr int FWD_COLS = 2048;
// Rows of up to FWD_COLS keys below which a call's elements are written one by one.  Direct / by rows in bf16: 16 heads x 2,048 keys with 1, 8,
// 12, 16 and 32 queries 2.0 / 4.7, 3.5 / 5.7, 4.1 / 5.7, 4.9 / 5.7 and 8.2 / 5.9 us; 8 x 300 with 16 and 32 queries 2.3 / 2.9 and 2.5 / 2.9 us;
// 32 x 8,192 with 1, 2 and 4 queries 3.5 / 5.1, 4.8 / 5.5 and 8.0 / 5.6 us.
constexpr int FWD_DIRECT = 256;
constexpr int FWD_THREADS = 256;

template <typename T>
__global__ void __launch_bounds__(FWD_THREADS)
relpos_forward_rows(const __grid_constant__ Buckets b, BiasGeometry g, const void* __restrict__ table, int table_dtype, T* __restrict__ out,
                    int64_t head_stride, int64_t row_stride, int rows, int pitch) {
  constexpr int COPIES = 16 / (int)sizeof(T);
  extern __shared__ __align__(16) unsigned char smem[];
  T* line = reinterpret_cast<T*>(smem);                                 // [COPIES][pitch]: copy s holds element e at e - s
  const int h = blockIdx.z, i0 = blockIdx.y * rows, j0 = blockIdx.x * FWD_COLS;
  const int nr = min(rows, g.Lq - i0), nc = min(FWD_COLS, g.Lk - j0), n = nr + nc - 1;
  // element e: distance of the last query of the block to key j0, plus e
  const int r0 = j0 - (i0 + nr - 1) - g.q_offset;
  for (int e = threadIdx.x; e < n; e += FWD_THREADS) {
    const T v = from_f32<T>(bias_value(b, g, table, table_dtype, h, r0 + e));
#pragma unroll
    for (int s = 0; s < COPIES; ++s)
      if (e >= s) line[s * pitch + e - s] = v;
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // the copies below read what these stores wrote
  __syncthreads();
  T* to = out + h * head_stride + (int64_t)i0 * row_stride + j0;
  for (int i = threadIdx.x; i < nr; i += FWD_THREADS) {
    T* row = to + i * row_stride;
    const int w = nr - 1 - i;                                           // the row's window: elements [w, w + nc)
    const int head = min(nc, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T)), body = (nc - head) / COPIES * COPIES;
    const int s = (w + head) % COPIES;
    if (body > 0) {
      const uint32_t from = (uint32_t)__cvta_generic_to_shared(line + s * pitch + (w + head - s));
      asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" :: "l"(row + head), "r"(from), "r"(body * (int)sizeof(T)) : "memory");
    }
  }
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  for (int k = threadIdx.x; k < nr * 2 * COPIES; k += FWD_THREADS) {      // the ends of the rows
    const int i = k / (2 * COPIES), e = k % (2 * COPIES);
    T* row = to + i * row_stride;
    const int head = min(nc, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T)), body = (nc - head) / COPIES * COPIES;
    const int j = e < COPIES ? e : head + body + e - COPIES;
    if (e < COPIES ? j < head : j < nc) row[j] = line[nr - 1 - i + j];
  }
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");        // shared memory stays until it has been read
}

constexpr int GRAD_CTAS = 592;            // blocks over all heads; also bounds the partial sums kept in the workspace
constexpr int GRAD_WARPS = 8;
constexpr int GRAD_ROWS = 8;              // rows of a patch
constexpr int GRAD_PATCHES = 96;          // patches of a warp after which the diagonals' fp32 sums are handed on (768 terms)
inline int grad_ctas_per_head(int heads) { return heads < GRAD_CTAS ? GRAD_CTAS / heads : 1; }

// A diagonal per lane, at distance r, to the warp's bucket sums, in a fixed order.
__device__ __forceinline__ void add_to_buckets(const Buckets& b, float sum, int r, bool counts, double* acc) {
  const int row = counts ? bucket_row(b, r) : -1;
  unsigned left = __ballot_sync(0xFFFFFFFFu, counts);
  while (left) {
    const int k = __shfl_sync(0xFFFFFFFFu, row, __ffs(left) - 1);
    const bool mine = row == k;
    float s = mine ? sum : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane_id() == 0) acc[k] += (double)s;
    left &= ~__ballot_sync(0xFFFFFFFFu, mine);
  }
}

// Bands of neighbouring diagonals, BAND wide, and the patches of 8 rows down each of them that hold anything.
struct Bands {
  int32_t band, count, steps, below, Lk, first_masked;
  __device__ __forceinline__ Bands(const Buckets& b, const BiasGeometry& g, int band_)
      : band(band_), steps((g.Lq + GRAD_ROWS - 1) / GRAD_ROWS), below(steps * GRAD_ROWS), Lk(g.Lk) {
    count = (below + g.Lk + band - 1) / band;                           // the first begins at column -below of row 0
    // causal: diagonals from q_offset + 1 on are masked, a band's lowest is 7 below its first column
    first_masked = b.causal ? g.q_offset + GRAD_ROWS : INT_MAX;
  }
  __device__ __forceinline__ int column(int k) const { return k * band - below; }       // of row 0
  __device__ __forceinline__ int first(int k) const { return max(0, (-band - column(k)) / GRAD_ROWS + 1); }
  __device__ __forceinline__ int patches(int k) const {
    const int c = column(k);
    if (k >= count || c >= first_masked) return 0;
    return max(0, min(steps, (Lk - c + GRAD_ROWS - 1) / GRAD_ROWS) - first(k));
  }
};

// A warp walks down a band in patches of 8 rows; the columns move with the rows, so each accumulator stays on its diagonal.  The patches
// of all bands and batch entries of a head, band by band, are dealt out evenly in runs to the blocks, whose warps take them in turn;
// where the band changes the block adds up its warps' diagonals and hands them on to the buckets.
//   VECTOR: a lane holds 16 bytes of each row (E neighbouring columns): an 8 x E patch has E + 7 diagonals.  Rows on 16-byte
//           boundaries, Lk a multiple of E.
//   else:   a lane holds every 32nd column (E = 4 of them): one diagonal for each of its 8 E elements.  Any alignment.
// Vectors / single elements for the same input: 64 / 121 us for 16 x 8 x 1,024 x 1,024 in bf16 (4.2 TB/s, 64% of the copy rate by vectors), 33 / 41 us
// for 5 x 12 x 776 x 1,000 in fp32 causal, 44 / 56 us without the mask; 777 x 1,001, which has no vectors, 39 to 41 and 57 us.  The width of the loads is
// a quarter of the odd call.  What bounds both forms is the reads in flight: 64 registers a thread (four blocks per SM) hold eight 16-byte
// rows, and a warp waits for its patch before it asks for the next: 17 of them in a row in the first call, 7 of two waits each in the odd one.  One
// call of 8 heads x 256 x 256 takes 14 us, mostly the emptying of the bands and the second kernel.
template <typename T, bool VECTOR>
__global__ void __launch_bounds__(GRAD_WARPS * 32, 4)
relpos_backward_partial(const __grid_constant__ Buckets b, BiasGeometry g, int64_t B, const T* __restrict__ grad, int64_t batch_stride,
                        int64_t head_stride, int64_t row_stride, double* __restrict__ partial) {
  constexpr int E = VECTOR ? 16 / (int)sizeof(T) : 4, BAND = 32 * E, ROWS = GRAD_ROWS, SHIFT = ROWS - 1;
  __shared__ double sums[GRAD_WARPS][2 * MTS_RELPOS_MAX_BUCKETS];
  __shared__ float lines[GRAD_WARPS][BAND + ROWS];
  const int rows = b.two_sided ? 2 * b.n : b.n, w = threadIdx.x / 32, lane = lane_id(), h = blockIdx.y;
  double* acc = sums[w];
  float* line = lines[w];
  for (int k = lane; k < rows; k += 32) acc[k] = 0.0;
  __syncwarp();
  const Bands bands(b, g, BAND);
  int64_t total = 0;
  for (int k0 = 0; k0 < bands.count; k0 += 32) total += __reduce_add_sync(0xFFFFFFFFu, bands.patches(k0 + lane));
  total *= B;
  // this block's run of patches, counted from the first band's first
  int64_t at = blockIdx.x * total / gridDim.x;
  const int64_t stop = (blockIdx.x + 1) * total / gridDim.x;
  int band = 0;
  int64_t skip = at;                                                    // patches of band `band` before the run

  while (at < stop) {
    const int n = bands.patches(band);
    if (skip >= B * n) { skip -= B * n; ++band; continue; }
    const int c0 = bands.column(band);
    const int run = (int)min(min(stop - at, B * n - skip), (int64_t)GRAD_PATCHES * GRAD_WARPS);
    const int end = bands.first(band) + n;
    int64_t batch = (skip + w) / n;
    int step = bands.first(band) + (int)(skip + w - batch * n);
    float sum[VECTOR ? E + SHIFT : E * ROWS];
#pragma unroll
    for (int k = 0; k < (int)(sizeof(sum) / 4); ++k) sum[k] = 0.f;
#pragma unroll 1
    for (int p = w; p < run; p += GRAD_WARPS) {
      const int i = step * ROWS, j = i + c0, here = min(ROWS, g.Lq - i);     // the patch: rows i..., columns j... of all lanes
      const T* from = grad + batch * batch_stride + h * head_stride + (int64_t)i * row_stride + j;
      // nothing of the patch outside the matrix, no lane behind the mask: no tests
      const bool whole = here == ROWS && j >= 0 && j + BAND <= g.Lk && c0 + BAND - 1 < bands.first_masked;
      if constexpr (VECTOR) {
        const int col = j + lane * E;
        const bool in = col >= 0 && col < g.Lk && c0 + lane * E < bands.first_masked;
        const T* mine = from + lane * E;
        uint4 v[ROWS];
        if (whole) {
#pragma unroll
          for (int k = 0; k < ROWS; ++k, mine += row_stride) v[k] = __ldcs(reinterpret_cast<const uint4*>(mine));
        } else {
#pragma unroll
          for (int k = 0; k < ROWS; ++k, mine += row_stride)
            v[k] = in && k < here ? __ldcs(reinterpret_cast<const uint4*>(mine)) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
          const uint32_t u[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if constexpr (sizeof(T) == 4) {
              sum[q - k + SHIFT] += __uint_as_float(u[q]);
            } else {
              const float2 f = unpack2<T>(u[q]);
              sum[2 * q - k + SHIFT] += f.x;
              sum[2 * q + 1 - k + SHIFT] += f.y;
            }
          }
        }
      } else {
        bool in[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int col = j + lane + 32 * e;
          in[e] = col >= 0 && col < g.Lk && c0 + lane + 32 * e < bands.first_masked;
        }
        const T* mine = from + lane;
#pragma unroll
        for (int k0 = 0; k0 < ROWS; k0 += ROWS / 2) {                     // half the rows at a time: 64 registers, 32 warps per SM
          T v[ROWS / 2][E];
#pragma unroll
          for (int k = 0; k < ROWS / 2; ++k, mine += row_stride)
#pragma unroll
            for (int e = 0; e < E; ++e) v[k][e] = whole || (in[e] && k0 + k < here) ? __ldcs(mine + 32 * e) : from_f32<T>(0.f);
#pragma unroll
          for (int k = 0; k < ROWS / 2; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e * ROWS + k0 + k] += to_f32(v[k][e]);
        }
      }
      for (step += GRAD_WARPS; step >= end; step -= n) ++batch;
    }
    at += run;
    skip += run;
    // line[d]: the sum of diagonal c0 - 7 + d; lanes add to it one after the other where their diagonals overlap
    for (int d = lane; d < BAND + ROWS; d += 32) line[d] = 0.f;
    __syncwarp();
    if constexpr (VECTOR) {
#pragma unroll
      for (int k = 0; k < E + SHIFT; k += E) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (k + e < E + SHIFT) line[lane * E + k + e] += sum[k + e];
        __syncwarp();
      }
    } else {
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
#pragma unroll
        for (int e = 0; e < E; ++e) line[lane + 32 * e - k + SHIFT] += sum[e * ROWS + k];
        __syncwarp();
      }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < (BAND + SHIFT + 31) / 32 * 32; d += GRAD_WARPS * 32) {
      const int r = c0 - SHIFT + d - g.q_offset;
      const bool counts = d < BAND + SHIFT && r > -g.Lq - g.q_offset && r < g.Lk - g.q_offset && !(b.causal && r > 0);
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < GRAD_WARPS; ++v) s += counts ? lines[v][d] : 0.f;
      add_to_buckets(b, s, r, counts, acc);
    }
    __syncthreads();
  }
  __syncthreads();
  for (int k = threadIdx.x; k < rows; k += blockDim.x) {
    double s = 0.0;
    for (int v = 0; v < GRAD_WARPS; ++v) s += sums[v][k];
    partial[((int64_t)h * gridDim.x + blockIdx.x) * rows + k] = s;
  }
}

// grad_table[k, h] = the sum of the blocks' partial sums, a warp each, in a fixed order.
__global__ void __launch_bounds__(128)
relpos_backward_combine(const double* __restrict__ partial, int ctas, int rows, int heads, float* __restrict__ grad_table) {
  const int i = blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
  if (i >= rows * heads) return;
  const int h = i / rows, k = i % rows;
  double s = 0.0;
#pragma unroll 4
  for (int c = lane_id(); c < ctas; c += 32) s += partial[((int64_t)h * ctas + c) * rows + k];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (lane_id() == 0) grad_table[k * heads + h] = (float)s;
}

}  // namespace mts

using namespace mts;

namespace {

int fill_buckets(const char* what, const mts_relpos_buckets* in, Buckets* out) {
  if (!in || !in->host_starts || in->n < 1) return set_error(MTS_ERR_INVALID_ARG, "%s: null or empty buckets", what);
  if (in->n > MTS_RELPOS_MAX_BUCKETS) return set_error(MTS_ERR_UNSUPPORTED, "%s: %d buckets per side", what, in->n);
  if (in->host_starts[0] != 0) return set_error(MTS_ERR_INVALID_ARG, "%s: the first bucket starts at %d, not 0", what, in->host_starts[0]);
  out->n = in->n;
  out->two_sided = in->two_sided != 0;
  out->causal = in->causal != 0;
  for (int k = 0; k < in->n; ++k) {
    if (k && in->host_starts[k] < in->host_starts[k - 1])
      return set_error(MTS_ERR_INVALID_ARG, "%s: bucket %d starts before bucket %d", what, k, k - 1);
    out->starts[k] = in->host_starts[k];
  }
  return MTS_OK;
}

int check_geometry(const char* what, int32_t heads, int64_t Lq, int64_t Lk, int64_t q_offset, int64_t head_stride, int64_t row_stride) {
  if (heads < 1 || Lq < 0 || Lk < 0) return set_error(MTS_ERR_INVALID_ARG, "%s: heads %d, Lq %lld, Lk %lld", what, heads, (long long)Lq, (long long)Lk);
  if (heads > 65535 || Lq >= (1 << 29) || Lk >= (1 << 29) || q_offset >= (1 << 29) || q_offset <= -(1 << 29))
    return set_error(MTS_ERR_UNSUPPORTED, "%s: heads %d, Lq %lld, Lk %lld, q_offset %lld", what, heads, (long long)Lq, (long long)Lk, (long long)q_offset);
  if (head_stride < 0 || row_stride < 0)
    return set_error(MTS_ERR_INVALID_ARG, "%s: negative stride", what);
  return MTS_OK;
}

}  // namespace

extern "C" int mts_relpos_bias_forward(const mts_relpos_buckets* buckets, const void* table, int32_t table_dtype, int32_t heads,
                                       int64_t Lq, int64_t Lk, int64_t q_offset, void* out, int32_t out_dtype,
                                       int64_t out_head_stride, int64_t out_row_stride, void* stream) {
  const char* what = "relpos_bias_forward";
  Buckets b;
  int rc = fill_buckets(what, buckets, &b);
  if (rc == MTS_OK) rc = check_geometry(what, heads, Lq, Lk, q_offset, out_head_stride, out_row_stride);
  if (rc != MTS_OK) return rc;
  if (!known_dtype(table_dtype) || !known_dtype(out_dtype))
    return set_error(MTS_ERR_INVALID_ARG, "%s: table dtype %d, out dtype %d", what, table_dtype, out_dtype);
  if (Lq == 0 || Lk == 0) return MTS_OK;
  if (!table || !out) return set_error(MTS_ERR_INVALID_ARG, "%s: null table or output", what);
  if (((uintptr_t)table % dtype_bytes(table_dtype)) || ((uintptr_t)out % dtype_bytes(out_dtype)))
    return set_error(MTS_ERR_ALIGNMENT, "%s: a pointer is no multiple of its element size", what);
  if ((Lq > 1 && out_row_stride < Lk) || (heads > 1 && out_head_stride < (Lq - 1) * out_row_stride + Lk))
    return set_error(MTS_ERR_INVALID_ARG, "%s: rows or heads of the output overlap", what);
  const BiasGeometry g = {heads, (int32_t)Lq, (int32_t)Lk, (int32_t)q_offset};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_dtype(out_dtype, [&](auto t) {
    using T = decltype(t);
    LaunchScope scope(K_RELPOS_FWD, s);
    const int64_t strips = ceil_div(Lk, FWD_COLS);
    if (heads * Lq * strips < FWD_DIRECT) {
      const dim3 grid((unsigned)ceil_div(Lk, 256), (unsigned)Lq, (unsigned)heads);
      relpos_forward_direct<T><<<grid, 256, 0, s>>>(b, g, table, table_dtype, static_cast<T*>(out), out_head_stride, out_row_stride);
      return check_launch(what);
    }
    // rows of a block: as many as leave the GPU two blocks per SM, 128 at most (the vector is made once for all of them), and not
    // more blocks down than a grid has room for
    int rows = 128;
    while (rows > 8 && ceil_div(Lq, rows) * strips * heads < FWD_WANTED) rows /= 2;
    if (ceil_div(Lq, rows) > 65535) rows = (int)ceil_div(Lq, 65535);      // 8,193 at most: 164 KB of shared memory
    const int pitch = (int)align_up((size_t)(Lk < FWD_COLS ? Lk : FWD_COLS) + (size_t)rows, 16);
    const size_t smem = (size_t)pitch * 16;
    if (smem > 48 * 1024) {
      const int e = check_cuda(cudaFuncSetAttribute(relpos_forward_rows<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem), "shared memory size");
      if (e != MTS_OK) return e;
    }
    const dim3 grid((unsigned)strips, (unsigned)ceil_div(Lq, rows), (unsigned)heads);
    relpos_forward_rows<T><<<grid, FWD_THREADS, smem, s>>>(b, g, table, table_dtype, static_cast<T*>(out), out_head_stride, out_row_stride, rows, pitch);
    return check_launch(what);
  });
}

extern "C" size_t mts_relpos_bias_workspace_bytes(const mts_relpos_buckets* buckets, int32_t heads) {
  if (!buckets || buckets->n < 1 || buckets->n > MTS_RELPOS_MAX_BUCKETS || heads < 1 || heads > 65535) return 0;
  const size_t rows = (size_t)buckets->n * (buckets->two_sided ? 2 : 1);
  return align_up((size_t)grad_ctas_per_head(heads) * heads * rows * sizeof(double), 256);
}

extern "C" int mts_relpos_bias_backward(const mts_relpos_buckets* buckets, const void* grad_out, int32_t grad_dtype, int64_t B,
                                        int32_t heads, int64_t Lq, int64_t Lk, int64_t q_offset, int64_t batch_stride,
                                        int64_t head_stride, int64_t row_stride, float* grad_table, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  const char* what = "relpos_bias_backward";
  Buckets b;
  int rc = fill_buckets(what, buckets, &b);
  if (rc == MTS_OK) rc = check_geometry(what, heads, Lq, Lk, q_offset, head_stride, row_stride);
  if (rc != MTS_OK) return rc;
  if (!known_dtype(grad_dtype) || B < 0 || batch_stride < 0) return set_error(MTS_ERR_INVALID_ARG, "%s: dtype %d, B %lld", what, grad_dtype, (long long)B);
  const bool empty = B == 0 || Lq == 0 || Lk == 0;
  if (!grad_table || (!empty && !grad_out)) return set_error(MTS_ERR_INVALID_ARG, "%s: null gradient", what);
  if (((uintptr_t)grad_out % dtype_bytes(grad_dtype)) || ((uintptr_t)grad_table & 3))
    return set_error(MTS_ERR_ALIGNMENT, "%s: a pointer is no multiple of its element size", what);
  const size_t need = mts_relpos_bias_workspace_bytes(buckets, heads);
  if (!workspace || workspace_bytes < need) return set_error(MTS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed", what, workspace_bytes, need);
  if ((uintptr_t)workspace & 255) return set_error(MTS_ERR_ALIGNMENT, "%s: the workspace must be 256-byte aligned", what);
  const int rows = b.two_sided ? 2 * b.n : b.n, ctas = grad_ctas_per_head(heads);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (empty) return check_cuda(cudaMemsetAsync(grad_table, 0, sizeof(float) * (size_t)rows * heads, s), "cudaMemsetAsync(grad_table)");
  const BiasGeometry g = {heads, (int32_t)Lq, (int32_t)Lk, (int32_t)q_offset};
  return with_dtype(grad_dtype, [&](auto t) {
    using T = decltype(t);
    {
      LaunchScope scope(K_RELPOS_BWD, s);
      const uintptr_t bits = (uintptr_t)grad_out | (uintptr_t)((batch_stride | head_stride | row_stride | Lk) * (int64_t)sizeof(T));
      if (bits % 16 == 0)
        relpos_backward_partial<T, true><<<dim3(ctas, heads), GRAD_WARPS * 32, 0, s>>>(b, g, B, static_cast<const T*>(grad_out), batch_stride, head_stride,
                                                                                     row_stride, static_cast<double*>(workspace));
      else
        relpos_backward_partial<T, false><<<dim3(ctas, heads), GRAD_WARPS * 32, 0, s>>>(b, g, B, static_cast<const T*>(grad_out), batch_stride, head_stride,
                                                                                      row_stride, static_cast<double*>(workspace));
    }
    int e = check_launch(what);
    if (e != MTS_OK) return e;
    LaunchScope scope(K_RELPOS_BWD, s);
    relpos_backward_combine<<<(unsigned)ceil_div((int64_t)rows * heads, 4), 128, 0, s>>>(static_cast<const double*>(workspace), ctas, rows, heads, grad_table);
    return check_launch(what);
  });
}
