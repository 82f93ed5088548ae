// Loss of a student's scores over V items against a teacher's best K of them, and its gradient.
//
//   q = softmax of scale teacher_k over the listed items (and exp(rest) for all others together),  p = softmax(scale x)
//   loss = sum_k q_k (log q_k - log p_{i_k}) + q_rest (log q_rest - log p_rest),   p_rest = what p gives to the items not listed
//   dx_v = weight scale (p_v - q_v) for a listed item, weight scale p_v (1 - q_rest / p_rest) for another
#include "rows.cuh"

namespace mts {

constexpr int DISTILL_THREADS = 256;
constexpr int DISTILL_MAX_K = MTS_DISTILL_MAX_K;

template <typename T, typename Q>
__global__ void __launch_bounds__(DISTILL_THREADS)
distill_loss(const T* logits, int64_t row_stride, int32_t V, float scale, const int64_t* __restrict__ index, const Q* __restrict__ teacher, int K,
             const float* __restrict__ rest, const float* __restrict__ weights, float* __restrict__ loss, T* grad, int64_t grad_stride) {
  __shared__ float room[DISTILL_THREADS / 32];
  __shared__ float q_of[DISTILL_MAX_K];
  __shared__ int32_t at[DISTILL_MAX_K];
  const int64_t n = blockIdx.x;
  const T* row = logits + n * row_stride;
  const float c = scale * LOG2E;
  // the teacher's distribution
  const int k = threadIdx.x;
  const int64_t i = k < K ? index[n * K + k] : -1;
  const bool listed = i >= 0, wrong = i >= V;
  const float t = listed ? to_f32(teacher[n * K + k]) * scale : -INFINITY, t_rest = rest ? rest[n] : -INFINITY;
  const float tm = block_max<DISTILL_THREADS>(fmaxf(t, t_rest), room), t_base = tm == -INFINITY ? 0.f : tm;
  const float e = wrong ? NAN : expf(t - t_base), e_rest = expf(t_rest - t_base);
  __syncthreads();
  const float total = block_sum<DISTILL_THREADS>(e, room) + e_rest;
  const bool any = total != 0.f;
  const float q = any ? e / total : 0.f, q_rest = any ? e_rest / total : 0.f, log_total = any ? logf(total) : 0.f;
  if (k < K) {
    q_of[k] = q;
    at[k] = listed && !wrong ? (int32_t)i : -1;
  }
  __syncthreads();
  // the student's sums
  float m = -INFINITY;
  for (int j = threadIdx.x; j < V; j += DISTILL_THREADS) m = fmaxf(m, to_f32(row[j]));
  m = block_max<DISTILL_THREADS>(m, room);
  const float base = m == -INFINITY ? 0.f : m;
  float all = 0.f, others = 0.f;
  for (int j = threadIdx.x; j < V; j += DISTILL_THREADS) {
    const float x = to_f32(row[j]), p = exp2_fast(exponent((x - base) * c));
    all += p;
    if (rest) {
      bool in = false;
      for (int u = 0; u < K; ++u) in |= at[u] == j;
      if (!in) others += p;
    }
  }
  __syncthreads();
  all = block_sum<DISTILL_THREADS>(all, room);
  __syncthreads();
  others = block_sum<DISTILL_THREADS>(others, room);
  const float log_all = all == 0.f ? 0.f : logf(all);
  float part = 0.f;
  if (q != 0.f) part = q * (t - t_base - log_total - ((to_f32(row[listed && !wrong ? i : 0]) - base) * scale - log_all));
  if (k == 0 && q_rest != 0.f) part += q_rest * (t_rest - t_base - log_total - (logf(others) - log_all));
  __syncthreads();
  part = block_sum<DISTILL_THREADS>(part, room);
  if (loss && threadIdx.x == 0) loss[n] = part;
  if (!grad) return;
  T* to = grad + n * grad_stride;
  const float w = weights ? weights[n] * scale : scale;
  const float inv_all = all == 0.f ? 0.f : 1.f / all;
  const float f = !any ? 0.f : w * (q_rest != 0.f && others != 0.f ? inv_all - q_rest / others : inv_all);
  const bool off = w == 0.f || !any;
  __syncthreads();
  for (int j = threadIdx.x; j < V; j += DISTILL_THREADS) {
    float g = 0.f;
    if (!off) {
      const float x = to_f32(row[j]), p = exp2_fast(exponent((x - base) * c));
      float want = 0.f;
      bool in = false;
      for (int u = 0; u < K; ++u)
        if (at[u] == j) { want += q_of[u]; in = true; }
      g = in ? w * (p * inv_all - want) : p * f;
      g += total * 0.f;
    }
    to[j] = from_f32<T>(g);
  }
}

}  // namespace mts

using namespace mts;

extern "C" int mts_distill_loss(const void* logits, int64_t row_stride, int32_t dtype, int64_t N, int64_t V, float scale, const int64_t* teacher_index,
                                const void* teacher_logits, int32_t teacher_dtype, int32_t K, const float* teacher_rest, const float* weights,
                                float* loss, void* grad_logits, int64_t grad_stride, void* stream) {
  const char* what = "distill_loss";
  if (!known_dtype(dtype) || !known_dtype(teacher_dtype)) return set_error(MTS_ERR_INVALID_ARG, "%s: dtype %d, teacher dtype %d", what, dtype, teacher_dtype);
  if (N < 0 || V < 1 || K < 1) return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, V %lld, K %d", what, (long long)N, (long long)V, K);
  if (N > MTS_SCORES_MAX_N || V > MTS_SCORES_MAX_V || K > MTS_DISTILL_MAX_K)
    return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, V %lld, K %d", what, (long long)N, (long long)V, K);
  if (!(scale > 0.f && scale <= 3.4e38f)) return set_error(MTS_ERR_INVALID_ARG, "%s: scale %g", what, scale);
  int rc = check_rows(what, "logits", logits, dtype, N, V, row_stride);
  if (rc == MTS_OK && grad_logits) rc = check_rows(what, "grad_logits", grad_logits, dtype, N, V, grad_stride);
  if (rc != MTS_OK) return rc;
  if (N > 0 && !loss && !grad_logits) return set_error(MTS_ERR_INVALID_ARG, "%s: neither a loss nor a gradient", what);
  if (N > 0 && (!teacher_index || !teacher_logits)) return set_error(MTS_ERR_INVALID_ARG, "%s: null teacher", what);
  if (((uintptr_t)teacher_index & 7) || ((uintptr_t)teacher_logits % dtype_bytes(teacher_dtype)) ||
      (((uintptr_t)teacher_rest | (uintptr_t)weights | (uintptr_t)loss) & 3))
    return set_error(MTS_ERR_ALIGNMENT, "%s: a pointer is no multiple of its element size", what);
  if (N == 0) return MTS_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    return with_dtype(teacher_dtype, [&](auto u) {
      using Q = decltype(u);
      LaunchScope scope(K_DISTILL, s);
      distill_loss<T, Q><<<(unsigned)N, DISTILL_THREADS, 0, s>>>(static_cast<const T*>(logits), row_stride, (int32_t)V, scale, teacher_index,
                                                                 static_cast<const Q*>(teacher_logits), K, teacher_rest, weights, loss,
                                                                 static_cast<T*>(grad_logits), grad_stride);
      return check_launch(what);
    });
  });
}
