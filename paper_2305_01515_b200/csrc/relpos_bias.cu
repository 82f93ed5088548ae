// Learned relative position bias by buckets, forward and gradient of its table.
//
//   out[h, i, j] = table[bucket(j - i - q_offset), h]
//   grad_table[k, h] = sum over b and the (i, j) of bucket k of grad_out[b, h, i, j]
//
// The bucket depends on the diagonal alone.
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

// One element per thread and step.
template <typename T>
__global__ void __launch_bounds__(256)
relpos_forward_direct(Buckets b, BiasGeometry g, const void* __restrict__ table, int table_dtype, T* __restrict__ out,
                      int64_t head_stride, int64_t row_stride) {
  const int h = blockIdx.z;
  for (int i = blockIdx.y; i < g.Lq; i += gridDim.y) {
    for (int64_t j = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; j < g.Lk; j += (int64_t)gridDim.x * blockDim.x) {
      const int r = (int)j - i - g.q_offset;
      const float v = b.causal && r > 0 ? -INFINITY : table_value(table, table_dtype, (int64_t)bucket_row(b, r) * g.heads + h);
      out[h * head_stride + i * row_stride + j] = from_f32<T>(v);
    }
  }
}

constexpr int GRAD_CTAS = 592;            // blocks over all heads; also bounds the partial sums kept in the workspace
constexpr int GRAD_WARPS = 8;
constexpr int GRAD_ROWS = 256;            // queries of one piece of work
inline int grad_ctas_per_head(int heads) { return (int)ceil_div(GRAD_CTAS, heads); }

// A warp takes 32 neighbouring diagonals, one per lane, and walks down GRAD_ROWS queries of one batch entry.  The sums of a piece of
// work are added per bucket, in a fixed order, to the warp's own row of accumulators.
template <typename T>
__global__ void __launch_bounds__(GRAD_WARPS * 32)
relpos_backward_partial(Buckets b, BiasGeometry g, int64_t B, const T* __restrict__ grad, int64_t batch_stride, int64_t head_stride,
                        int64_t row_stride, double* __restrict__ partial) {
  __shared__ double acc[GRAD_WARPS][2 * MTS_RELPOS_MAX_BUCKETS];
  const int rows = b.two_sided ? 2 * b.n : b.n, w = threadIdx.x / 32, lane = lane_id(), h = blockIdx.y;
  for (int k = lane; k < rows; k += 32) acc[w][k] = 0.0;
  __syncwarp();
  // diagonal c: distance r = c - (Lq - 1) - q_offset, key j = i + c - (Lq - 1)
  const int64_t bands = ((int64_t)g.Lq + g.Lk - 1 + 31) / 32, pieces = (g.Lq + GRAD_ROWS - 1) / GRAD_ROWS;
  for (int64_t item = (int64_t)blockIdx.x * GRAD_WARPS + w; item < bands * pieces * B; item += (int64_t)gridDim.x * GRAD_WARPS) {
    const int c = (int)(item % bands) * 32 + lane;
    const int piece = (int)(item / bands % pieces);
    const int64_t batch = item / (bands * pieces);
    const int shift = c - (g.Lq - 1), r = shift - g.q_offset;
    const bool counts = !(b.causal && r > 0) && c < g.Lq + g.Lk - 1;
    const int i0 = max(piece * GRAD_ROWS, -shift), i1 = min(min(piece * GRAD_ROWS + GRAD_ROWS, g.Lq), g.Lk - shift);
    float sum = 0.f;
    if (counts)
      for (int i = i0; i < i1; ++i) sum += to_f32(grad[batch * batch_stride + h * head_stride + i * row_stride + (i + shift)]);
    const int row = counts ? bucket_row(b, r) : -1;
    unsigned left = __ballot_sync(0xFFFFFFFFu, counts);
    while (left) {
      const int k = __shfl_sync(0xFFFFFFFFu, row, __ffs(left) - 1);
      const bool mine = row == k;
      float s = mine ? sum : 0.f;
      for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      if (lane == 0) acc[w][k] += (double)s;
      left &= ~__ballot_sync(0xFFFFFFFFu, mine);
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < rows; k += blockDim.x) {
    double s = 0.0;
    for (int v = 0; v < GRAD_WARPS; ++v) s += acc[v][k];
    partial[((int64_t)h * gridDim.x + blockIdx.x) * rows + k] = s;
  }
}

// grad_table[k, h] = the sum of the blocks' partial sums, in the order of the blocks.
__global__ void relpos_backward_combine(const double* __restrict__ partial, int ctas, int rows, int heads, float* __restrict__ grad_table) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= rows * heads) return;
  const int h = i / rows, k = i % rows;
  double s = 0.0;
  for (int c = 0; c < ctas; ++c) s += partial[((int64_t)h * ctas + c) * rows + k];
  grad_table[k * heads + h] = (float)s;
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
    const dim3 grid((unsigned)ceil_div(Lk, 256), (unsigned)(Lq < 65535 ? Lq : 65535), (unsigned)heads);
    relpos_forward_direct<T><<<grid, 256, 0, s>>>(b, g, table, table_dtype, static_cast<T*>(out), out_head_stride, out_row_stride);
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
      relpos_backward_partial<T><<<dim3(ctas, heads), GRAD_WARPS * 32, 0, s>>>(b, g, B, static_cast<const T*>(grad_out), batch_stride, head_stride,
                                                                              row_stride, static_cast<double*>(workspace));
    }
    int e = check_launch(what);
    if (e != MTS_OK) return e;
    LaunchScope scope(K_RELPOS_BWD, s);
    relpos_backward_combine<<<(unsigned)ceil_div((int64_t)rows * heads, 128), 128, 0, s>>>(static_cast<const double*>(workspace), ctas, rows, heads, grad_table);
    return check_launch(what);
  });
}
