// Root-mean-square norm of the residual stream, forward (output in the tensors' type or in 8 bits) and backward.
//
//   r = round(x + residual),  c = 1 / sqrt(mean_j r_j^2 + eps),  y_j = r_j c w_j
//   dx_j = dr_j + c (dy_j w_j - r_j a),  a = c^2 mean_j(dy_j w_j r_j),   dw_j = sum over rows of dy_j r_j c
#include <cuda_fp8.h>

#include "rows.cuh"

namespace mts {

constexpr int NORM_THREADS = 256;
constexpr float LEAST_MAX = 7.888609052210118e-31f;      // 2^-100: least maximum of a group of 8-bit codes
constexpr float TOP_CODE = 448.f;                        // largest number of e4m3

__device__ __forceinline__ float weight_value(const void* w, int dtype, int64_t i) {
  if (dtype == MTS_DTYPE_FP32) return static_cast<const float*>(w)[i];
  if (dtype == MTS_DTYPE_FP16) return to_f32(static_cast<const __half*>(w)[i]);
  return to_f32(static_cast<const __nv_bfloat16*>(w)[i]);
}

template <typename T>
struct NormForward {
  const T* x;
  const T* residual;
  const void* weight;
  T* sum;
  T* out;
  uint8_t* codes;
  float* scales;
  float* inv_rms;
  int64_t x_stride, residual_stride, sum_stride, out_stride;
  int32_t weight_dtype, D, group;
  float eps;
};

template <typename T>
__device__ __forceinline__ float stream_value(const NormForward<T>& a, int64_t row, int j) {
  const float x = to_f32(a.x[row * a.x_stride + j]);
  return a.residual ? to_f32(from_f32<T>(x + to_f32(a.residual[row * a.residual_stride + j]))) : x;
}

template <typename T>
__global__ void __launch_bounds__(NORM_THREADS)
rms_norm_forward(const NormForward<T> a) {
  __shared__ float room[NORM_THREADS / 32];
  const int64_t row = blockIdx.x;
  float s = 0.f;
  for (int j = threadIdx.x; j < a.D; j += NORM_THREADS) {
    const float r = stream_value(a, row, j);
    s += r * r;
  }
  const float c = 1.f / sqrtf(block_sum<NORM_THREADS>(s, room) / a.D + a.eps);
  if (a.inv_rms && threadIdx.x == 0) a.inv_rms[row] = c;
  const int step = a.group ? a.group : a.D, groups = (a.D + step - 1) / step;
  for (int g = 0; g < groups; ++g) {
    const int end = min(a.D, (g + 1) * step);
    float scale = 0.f, inverse = 0.f;
    if (a.codes) {
      float m = 0.f;
      for (int j = g * step + threadIdx.x; j < end; j += NORM_THREADS)
        m = fmaxf(m, fabsf(stream_value(a, row, j) * c * weight_value(a.weight, a.weight_dtype, j)));
      m = fmaxf(block_max<NORM_THREADS>(m, room), LEAST_MAX);
      scale = m / TOP_CODE;
      inverse = TOP_CODE / m;
      if (threadIdx.x == 0) a.scales[row * groups + g] = scale;
    }
    for (int j = g * step + threadIdx.x; j < end; j += NORM_THREADS) {
      const float r = stream_value(a, row, j);
      const float y = r * c * weight_value(a.weight, a.weight_dtype, j);
      if (a.codes) a.codes[row * a.out_stride + j] = __nv_cvt_float_to_fp8(y * inverse, __NV_SATFINITE, __NV_E4M3);
      else a.out[row * a.out_stride + j] = from_f32<T>(y);
    }
  }
  __syncthreads();
  if (a.residual)
    for (int j = threadIdx.x; j < a.D; j += NORM_THREADS) a.sum[row * a.sum_stride + j] = from_f32<T>(stream_value(a, row, j));
}

template <typename T>
__global__ void __launch_bounds__(NORM_THREADS)
rows_from_8bit(const uint8_t* __restrict__ codes, int64_t codes_stride, const float* __restrict__ scales, int group, int D, T* __restrict__ out,
               int64_t out_stride) {
  const int64_t row = blockIdx.x;
  const int step = group ? group : D, groups = (D + step - 1) / step;
  for (int j = threadIdx.x; j < D; j += NORM_THREADS) {
    const __half h = __half(__nv_cvt_fp8_to_halfraw(codes[row * codes_stride + j], __NV_E4M3));
    out[row * out_stride + j] = from_f32<T>(__half2float(h) * scales[row * groups + j / step]);
  }
}

constexpr int NORM_BACK_BLOCKS = 592;

template <typename T>
struct NormBackward {
  const T* x;
  const void* weight;
  const float* inv_rms;
  const T* grad_out;
  const T* grad_sum;
  T* grad_x;
  float* partial;
  int64_t x_stride, out_stride, sum_stride, gx_stride, N;
  int32_t weight_dtype, D;
};

template <typename T>
__global__ void __launch_bounds__(NORM_THREADS)
rms_norm_backward(const NormBackward<T> a) {
  __shared__ float room[NORM_THREADS / 32];
  float* mine = a.partial ? a.partial + (int64_t)blockIdx.x * a.D : nullptr;
  if (mine)
    for (int j = threadIdx.x; j < a.D; j += NORM_THREADS) mine[j] = 0.f;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const float c = a.inv_rms[row];
    float s = 0.f;
    for (int j = threadIdx.x; j < a.D; j += NORM_THREADS)
      s += to_f32(a.grad_out[row * a.out_stride + j]) * weight_value(a.weight, a.weight_dtype, j) * to_f32(a.x[row * a.x_stride + j]);
    const float m = block_sum<NORM_THREADS>(s, room) / a.D * (c * c);
    for (int j = threadIdx.x; j < a.D; j += NORM_THREADS) {
      const float r = to_f32(a.x[row * a.x_stride + j]), dy = to_f32(a.grad_out[row * a.out_stride + j]);
      float d = c * (dy * weight_value(a.weight, a.weight_dtype, j) - r * m);
      if (a.grad_sum) d += to_f32(a.grad_sum[row * a.sum_stride + j]);
      if (mine) mine[j] += dy * (r * c);
      a.grad_x[row * a.gx_stride + j] = from_f32<T>(d);
    }
  }
}

__global__ void __launch_bounds__(256)
rms_norm_weight_gradient(const float* __restrict__ partial, int blocks, int D, float* __restrict__ grad_weight) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= D) return;
  double s = 0.0;
  for (int b = 0; b < blocks; ++b) s += partial[(int64_t)b * D + j];
  grad_weight[j] = (float)s;
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
    const NormForward<T> a = {static_cast<const T*>(x), static_cast<const T*>(residual), weight, static_cast<T*>(sum_out), static_cast<T*>(out), codes,
                              scales, inv_rms, x_stride, residual_stride, sum_stride, out_stride, weight_dtype, D, group, eps};
    LaunchScope scope(K_NORM_FWD, s);
    rms_norm_forward<T><<<(unsigned)N, NORM_THREADS, 0, s>>>(a);
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
    LaunchScope scope(K_NORM_FWD, s);
    rows_from_8bit<T><<<(unsigned)N, NORM_THREADS, 0, s>>>(codes, codes_stride, scales, group, D, static_cast<T*>(out), out_stride);
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
    const int blocks = (int)(N < NORM_BACK_BLOCKS ? N : NORM_BACK_BLOCKS);
    float* partial = grad_weight ? static_cast<float*>(workspace) : nullptr;
    const NormBackward<T> a = {static_cast<const T*>(x), weight, inv_rms, static_cast<const T*>(grad_out), static_cast<const T*>(grad_sum),
                               static_cast<T*>(grad_x), partial, x_stride, grad_out_stride, grad_sum_stride, grad_x_stride, N, weight_dtype, D};
    {
      LaunchScope scope(K_NORM_BWD, s);
      rms_norm_backward<T><<<blocks, NORM_THREADS, 0, s>>>(a);
    }
    int e = check_launch(what);
    if (e != MTS_OK || !grad_weight) return e;
    LaunchScope scope(K_NORM_BWD, s);
    rms_norm_weight_gradient<<<(unsigned)ceil_div(D, 256), 256, 0, s>>>(partial, blocks, D, grad_weight);
    return check_launch(what);
  });
}
