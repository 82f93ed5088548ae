// Log probabilities of given items under a softmax over V scores, with its entropy and the best alternatives, and their gradient.
//
//   z = scale x,  m = max x,  S = sum_v exp(scale (x_v - m)),  log p_v = scale (x_v - m) - log S
//   entropy = -sum_v p_v log p_v = log S - (sum_v exp(scale (x_v - m)) scale (x_v - m)) / S
//   dx_v = scale (g_logp ([v = target] - p_v) - g_entropy p_v (log p_v + entropy))
#include "rows.cuh"

namespace mts {

constexpr int LOGP_THREADS = 256;

struct LogprobsOut {
  float* logp;
  float* entropy;
  float* stats;
  int64_t* top_index;
  float* top_logp;
};

template <int THREADS>
__device__ __forceinline__ uint64_t block_max64(uint64_t x, uint64_t* room) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  __syncthreads();
  if (lane_id() == 0) room[threadIdx.x / 32] = x;
  __syncthreads();
  x = room[0];
  for (int w = 1; w < THREADS / 32; ++w) x = max(x, room[w]);
  return x;
}

template <typename T>
__global__ void __launch_bounds__(LOGP_THREADS)
logprobs_forward(const T* __restrict__ logits, int64_t row_stride, int32_t V, float scale, const int64_t* __restrict__ targets, int top_k, LogprobsOut out) {
  __shared__ float room[LOGP_THREADS / 32];
  __shared__ uint64_t room64[LOGP_THREADS / 32];
  const int64_t n = blockIdx.x;
  const RowBatches<T> r(logits + n * row_stride, V);
  constexpr int E = RowBatches<T>::E;
  const float c = scale * LOG2E;
  float m = -INFINITY, v[E];
  for (int b = threadIdx.x; b < r.count; b += LOGP_THREADS) {
    r.load(b, v);
#pragma unroll
    for (int e = 0; e < E; ++e) m = fmaxf(m, v[e]);
  }
  m = block_max<LOGP_THREADS>(m, room);
  const float base = m == -INFINITY ? 0.f : m;
  float S = 0.f, P = 0.f;
  for (int b = threadIdx.x; b < r.count; b += LOGP_THREADS) {
    r.load(b, v);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = exponent((v[e] - base) * c), p = exp2_fast(d);
      S += p;
      P += p * d;
    }
  }
  S = block_sum<LOGP_THREADS>(S, room);
  __syncthreads();
  P = block_sum<LOGP_THREADS>(P, room);
  const float log_s = S > 0.f ? logf(S) : S == 0.f ? 0.f : NAN;
  const float nothing = S == 0.f ? -INFINITY : 0.f;
  if (threadIdx.x == 0) {
    if (out.logp) {
      const int64_t t = targets[n];
      out.logp[n] = t < 0 ? 0.f : t >= V ? NAN : (to_f32(r.row[t]) - base) * scale - log_s + nothing;
    }
    if (out.entropy) out.entropy[n] = S == 0.f ? 0.f : log_s - P / S * LN2;
    if (out.stats) {
      out.stats[2 * n] = base;
      out.stats[2 * n + 1] = log_s;
    }
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < top_k; ++k) {
    uint64_t best = 0;
    for (int b = threadIdx.x; b < r.count; b += LOGP_THREADS) {
      r.load(b, v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = r.first(b) + e;
        const uint64_t o = score_order(v[e], i);
        if (i >= 0 && i < V && o < last && o > best) best = o;
      }
    }
    last = block_max64<LOGP_THREADS>(best, room64);
    if (threadIdx.x == 0) {
      const int i = order_index(last);
      if (out.top_index) out.top_index[n * top_k + k] = i;
      if (out.top_logp) out.top_logp[n * top_k + k] = (to_f32(r.row[i]) - base) * scale - log_s + nothing;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(LOGP_THREADS)
logprobs_backward(const T* logits, int64_t row_stride, int32_t V, float scale, const int64_t* __restrict__ targets, const float* __restrict__ stats,
                  const float* __restrict__ entropy, const float* __restrict__ grad_logp, const float* __restrict__ grad_entropy, T* grad_logits,
                  int64_t grad_stride) {
  const int64_t n = blockIdx.x;
  const float c = scale * LOG2E, m = stats[2 * n], log_s = stats[2 * n + 1];
  const int64_t t = targets ? targets[n] : -1;
  const float gl = !grad_logp || t < 0 ? 0.f : t >= V ? NAN : grad_logp[n], gh = grad_entropy ? grad_entropy[n] : 0.f;
  // dx = p (alpha + beta d) + [v = target] scale gl, with d = log2 of exp(scale (x - m))
  const float alpha = -scale * (gl + (gh != 0.f ? gh * (entropy[n] - log_s) : 0.f)), beta = -scale * gh * LN2, bias = log_s * LOG2E;
  for (int j = threadIdx.x; j < V; j += LOGP_THREADS) {
    float g = 0.f;
    if (gl != 0.f || gh != 0.f) {
      const float x = to_f32(logits[n * row_stride + j]);
      const float d = exponent((x - m) * c), p = exp2_fast(d - bias);
      g = p * (alpha + beta * d) + (j == t ? scale * gl : 0.f);
    }
    grad_logits[n * grad_stride + j] = from_f32<T>(g);
  }
}

}  // namespace mts

using namespace mts;

namespace {

int check_logits(const char* what, const void* logits, int64_t row_stride, int32_t dtype, int64_t N, int64_t V, float scale) {
  if (!known_dtype(dtype)) return set_error(MTS_ERR_INVALID_ARG, "%s: dtype %d", what, dtype);
  if (N < 0 || V < 1) return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, V %lld", what, (long long)N, (long long)V);
  if (N > MTS_SCORES_MAX_N || V > MTS_SCORES_MAX_V) return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, V %lld", what, (long long)N, (long long)V);
  if (!(scale > 0.f && scale <= 3.4e38f)) return set_error(MTS_ERR_INVALID_ARG, "%s: scale %g", what, scale);
  return check_rows(what, "logits", logits, dtype, N, V, row_stride);
}

}  // namespace

extern "C" int mts_logprobs_forward(const void* logits, int64_t row_stride, int32_t dtype, int64_t N, int64_t V, float scale, const int64_t* targets,
                                    int32_t top_k, float* logp, float* entropy, float* stats, int64_t* top_index, float* top_logp, void* stream) {
  const char* what = "logprobs_forward";
  const int rc = check_logits(what, logits, row_stride, dtype, N, V, scale);
  if (rc != MTS_OK) return rc;
  if (top_k < 0 || top_k > V) return set_error(MTS_ERR_INVALID_ARG, "%s: the best %d of %lld", what, top_k, (long long)V);
  if (top_k > MTS_LOGPROBS_MAX_TOP) return set_error(MTS_ERR_UNSUPPORTED, "%s: the best %d", what, top_k);
  if (logp && !targets) return set_error(MTS_ERR_INVALID_ARG, "%s: log probabilities of no targets", what);
  if (top_k && !top_index && !top_logp) top_k = 0;
  if ((((uintptr_t)targets | (uintptr_t)top_index) & 7) || (((uintptr_t)logp | (uintptr_t)entropy | (uintptr_t)stats | (uintptr_t)top_logp) & 3))
    return set_error(MTS_ERR_ALIGNMENT, "%s: a pointer is no multiple of its element size", what);
  if (N == 0) return MTS_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const LogprobsOut out = {logp, entropy, stats, top_index, top_logp};
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    LaunchScope scope(K_LOGPROBS_FWD, s);
    logprobs_forward<T><<<(unsigned)N, LOGP_THREADS, 0, s>>>(static_cast<const T*>(logits), row_stride, (int32_t)V, scale, targets, top_k, out);
    return check_launch(what);
  });
}

extern "C" int mts_logprobs_backward(const void* logits, int64_t row_stride, int32_t dtype, int64_t N, int64_t V, float scale, const int64_t* targets,
                                     const float* stats, const float* entropy, const float* grad_logp, const float* grad_entropy, void* grad_logits,
                                     int64_t grad_stride, void* stream) {
  const char* what = "logprobs_backward";
  int rc = check_logits(what, logits, row_stride, dtype, N, V, scale);
  if (rc == MTS_OK) rc = check_rows(what, "grad_logits", grad_logits, dtype, N, V, grad_stride);
  if (rc != MTS_OK) return rc;
  if (N > 0 && !stats) return set_error(MTS_ERR_INVALID_ARG, "%s: null stats", what);
  if ((grad_logp && !targets) || (grad_entropy && !entropy))
    return set_error(MTS_ERR_INVALID_ARG, "%s: a gradient without what the forward pass had or left for it", what);
  if (((uintptr_t)targets & 7) || (((uintptr_t)stats | (uintptr_t)entropy | (uintptr_t)grad_logp | (uintptr_t)grad_entropy) & 3))
    return set_error(MTS_ERR_ALIGNMENT, "%s: a pointer is no multiple of its element size", what);
  if (N == 0) return MTS_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    LaunchScope scope(K_LOGPROBS_BWD, s);
    logprobs_backward<T><<<(unsigned)N, LOGP_THREADS, 0, s>>>(static_cast<const T*>(logits), row_stride, (int32_t)V, scale, targets, stats, entropy,
                                                              grad_logp, grad_entropy, static_cast<T*>(grad_logits), grad_stride);
    return check_launch(what);
  });
}
