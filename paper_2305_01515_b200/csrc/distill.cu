// Loss of a student's scores over V items against a teacher's best K of them, and its gradient.
//
//   q = softmax of scale teacher_k over the listed items (and exp(rest) for all others together),  p = softmax(scale x)
//   loss = sum_k q_k (log q_k - log p_{i_k}) + q_rest (log q_rest - log p_rest),   p_rest = what p gives to the items not listed
//   dx_v = weight scale (p_v - q_v) for a listed item, weight scale p_v (1 - q_rest / p_rest) for another
#include "rows.cuh"

namespace mts {

constexpr int DISTILL_WARPS = 16;
constexpr int DISTILL_MAX_K = MTS_DISTILL_MAX_K;
constexpr int DISTILL_UNROLL = 8, DISTILL_GRAD_UNROLL = 4;     // batches on their way for a thread
constexpr int LISTED_BYTES = 32768;                            // of the bits that say which batches of a part hold a listed item

// Sums of 2^(c x - base) over a set of scores, relative to their largest: over the listed items where these are told apart, and over the others.
struct DistillSums { float m, listed, others; };

__device__ __forceinline__ DistillSums scaled_to(const DistillSums& s, float m, float c) {
  if (s.m == -INFINITY) return {m, s.listed, s.others};
  const float base = base_of(m, c), f = exp2_fast(ordinary(base) ? base_of(s.m, c) - base : (s.m - m) * c);
  return {m, f * s.listed, f * s.others};
}
__device__ __forceinline__ DistillSums join_lanes(DistillSums s, float c) {
  const float m = warp_max(s.m);
  s = scaled_to(s, m, c);
  return {m, warp_sum(s.listed), warp_sum(s.others)};
}

__device__ __forceinline__ float teacher_value(const void* t, int dtype, int64_t i) {
  if (dtype == MTS_DTYPE_FP32) return static_cast<const float*>(t)[i];
  if (dtype == MTS_DTYPE_FP16) return to_f32(static_cast<const __half*>(t)[i]);
  return to_f32(static_cast<const __nv_bfloat16*>(t)[i]);
}

struct DistillCall {
  int64_t row_stride, grad_stride;
  const int64_t* index;
  const void* teacher;
  const float* rest;
  const float* weights;
  float* loss;
  int32_t V, K, teacher_dtype, log_parts, share;
  float scale;
};

struct DistillRoom {
  float q[DISTILL_MAX_K], score[DISTILL_MAX_K], log_q[DISTILL_MAX_K];
  int32_t at[DISTILL_MAX_K];                                   // -1: not used
  DistillSums of_warp[DISTILL_WARPS], of_part[1 << MAX_LOG_PARTS];
  float total, q_rest, log_q_rest;
};

// Exponentials of a batch.
template <typename T, bool ORDINARY>
__device__ __forceinline__ void exponentials(const uint4& w, float m, float base, float c, float (&v)[RowBatches<T>::E]) {
  constexpr int E = RowBatches<T>::E;
  RowBatches<T>::unpack(w, v);
  const Pair minus(-base, -base), c2(c, c);
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const float2 d = ORDINARY ? fma2(Pair(v[e], v[e + 1]), c2, minus).get() : make_float2((v[e] - m) * c, (v[e + 1] - m) * c);
    v[e] = exp2_fast(d.x);
    v[e + 1] = exp2_fast(d.y);
  }
}
template <typename T>
__device__ __forceinline__ Pair sum_of(const float (&v)[RowBatches<T>::E]) {
  Pair s = Pair(v[0], v[1]) + Pair(v[2], v[3]);
  if constexpr (RowBatches<T>::E == 8) s = s + (Pair(v[4], v[5]) + Pair(v[6], v[7]));
  return s;
}

// A row (or a part of it, by a cluster of blocks) by a block.  The sums of the exponentials take one pass over the scores as in the log probabilities; the
// gradient reads them once more, from L2, where the row has just passed.
// With the rest's weight given (REST) the sum over the items that are not listed is made without the listed ones: what is left of a difference would lose its
// digits where the listed ones have almost everything.  Bits in shared memory, eight to a thread's group, say which batches hold a listed item; the pass
// leaves these out, and they are added afterwards item by item.
// The gradient is written as if nothing were listed, and the listed places once more.
template <typename T, bool REST>
__global__ void __launch_bounds__(DISTILL_WARPS * 32, 2)
distill_loss(const T* logits, T* grad, const DistillCall a) {
  constexpr int E = RowBatches<T>::E, U = DISTILL_UNROLL;
  __shared__ DistillRoom room;
  extern __shared__ __align__(16) uint8_t left_out[];
  const int tid = threadIdx.x, lane = lane_id(), warp = tid / 32, threads = blockDim.x, warps = threads / 32;
  const int parts = 1 << a.log_parts, part = blockIdx.x & (parts - 1);
  const int64_t n = blockIdx.x >> a.log_parts;
  if (parts > 1) cluster_arrive();                             // all blocks have begun before others write to them
  const RowBatches<T, false> r(logits + n * a.row_stride, a.V);
  const int32_t b0 = min(r.count, part * a.share), b1 = min(r.count, b0 + a.share);
  const float c = a.scale * LOG2E;

  // the bits of the batches that are left out: byte of a thread's group, bit of the batch in it
  if (REST) {
    const int bytes = min(LISTED_BYTES, (b1 - b0 + threads * U - 1) / (threads * U) * threads);
    for (int i = tid; i < bytes / 4; i += threads) reinterpret_cast<uint32_t*>(left_out)[i] = 0;
    __syncthreads();
    for (int k = tid; k < a.K; k += threads) {
      const int64_t i = a.index[n * a.K + k];
      if (i < 0 || i >= a.V) continue;
      const int32_t b = (int32_t)(i + r.shift) / E - b0, group = b / (threads * U), in = b - group * threads * U;
      const int64_t byte = (int64_t)group * threads + in % threads;
      if (b >= 0 && b < b1 - b0 && byte < LISTED_BYTES) atomicOr(reinterpret_cast<uint32_t*>(left_out) + byte / 4, 1u << (in / threads + byte % 4 * 8));
    }
  }
  // the teacher's distribution, by the first warp
  if (warp == 0) {
    float most = -INFINITY;
    bool wrong = false;
    for (int k = lane; k < a.K; k += 32) {
      const int64_t i = a.index[n * a.K + k];
      const float t = i >= 0 ? teacher_value(a.teacher, a.teacher_dtype, n * a.K + k) * a.scale : -INFINITY;
      wrong |= i >= a.V || isnan(t);
      room.log_q[k] = t;
      room.at[k] = i >= 0 && i < a.V ? (int32_t)i : -1;
      most = fmaxf(most, t);
    }
    const float t_rest = REST ? a.rest[n] : -INFINITY;
    most = fmaxf(warp_max(most), t_rest);
    const float base = most == -INFINITY ? 0.f : most;
    const float e_rest = expf(t_rest - base);
    float total = 0.f;
    for (int k = lane; k < a.K; k += 32) total += expf(room.log_q[k] - base);
    total = warp_sum(total) + e_rest;
    if (__any_sync(0xFFFFFFFFu, wrong)) total = NAN;
    const bool any = total != 0.f;                             // else nothing is left of the teacher's row
    const float log_total = any ? logf(total) : 0.f;
    for (int k = lane; k < a.K; k += 32) {
      const float t = room.log_q[k] - base;
      room.q[k] = any ? expf(t) / total : 0.f;
      room.log_q[k] = t - log_total;
      const int32_t i = room.at[k];
      room.score[k] = i >= 0 ? to_f32(r.row[i]) : 0.f;
    }
    if (lane == 0) {
      room.total = total;
      room.q_rest = any ? e_rest / total : 0.f;
      room.log_q_rest = t_rest - base - log_total;
    }
  }
  if (REST) __syncthreads();

  // the student's sums
  float m = -INFINITY, base = 0.f, listed = 0.f;
  Pair others(0.f, 0.f);
  const uint4 nothing_there = make_uint4(RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW);
  // whether batch b holds a listed item, where the bits do not reach
  const auto holds_listed = [&](int32_t b) {
    for (int k = 0; k < a.K; ++k)
      if (room.at[k] >= 0 && (room.at[k] + r.shift) / E == b) return true;
    return false;
  };
  const auto rescale = [&](float most) {
    const DistillSums s = scaled_to({m, listed, others.sum()}, most, c);
    listed = s.listed;
    others = Pair(s.others, 0.f);
    m = most;
    base = base_of(m, c);
  };
  int32_t byte = tid;
  for (int32_t g = b0; g < b1; g += threads * U) {
    const int32_t b = g + tid;
    const bool all = r.template all_whole<U>(g, b1, tid, threads);
    uint4 w[U];
    r.load_held(g, min(b1, g + threads * U), tid, threads, all, w);
    if (!all) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (b + u * threads >= b1) w[u] = nothing_there;
    }
    uint32_t most_bits = max_bits<T>(w[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) most_bits = max_bits<T>(most_bits, w[u]);
    const float most = max_value<T>(most_bits);
    if (most > m) rescale(most);
    unsigned out = 0;
    if (REST) {
      if (byte < LISTED_BYTES) {
        out = left_out[byte];
      } else {
        for (int u = 0; u < U; ++u) out |= holds_listed(b + u * threads) << u;
      }
      byte += threads;
    }
    if (!ordinary(base)) {
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        if (b + u * threads >= b1 || out >> u & 1) continue;
        float v[E];
        exponentials<T, false>(r.raw(b + u * threads), m, base, c, v);
        others = others + sum_of<T>(v);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!all && b + u * threads >= b1) continue;
        float v[E];
        exponentials<T, true>(w[u], m, base, c, v);
        const Pair s = sum_of<T>(v);
        if (!REST || !(out >> u & 1)) others = others + s;
      }
    }
  }
  if (REST) {
    // the batches left out, each by the thread of the first place in it
    for (int k = tid; k < a.K; k += threads) {
      const int32_t b = (room.at[k] + r.shift) / E;
      if (room.at[k] < 0 || b < b0 || b >= b1) continue;
      unsigned places = 0;
      bool first = true;
      for (int j = 0; j < a.K; ++j) {
        const int32_t i = room.at[j] + r.shift;
        if (room.at[j] >= 0 && i / E == b) {
          places |= 1u << i % E;
          first &= j >= k;
        }
      }
      if (!first) continue;
      const uint4 batch = r.raw(b);
      const float most = max_value<T>(max_bits<T>(batch));
      if (most > m) rescale(most);
      float v[E];
      if (ordinary(base)) exponentials<T, true>(batch, m, base, c, v);
      else exponentials<T, false>(batch, m, base, c, v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (places >> e & 1) listed += v[e];
        else others = others + Pair(v[e], 0.f);
      }
    }
  }
  const DistillSums nobody = {-INFINITY, 0.f, 0.f};
  DistillSums s = join_lanes({m, listed, others.sum()}, c);
  if (lane == 0) room.of_warp[warp] = s;
  __syncthreads();
  s = join_lanes(lane < warps ? room.of_warp[lane] : nobody, c);
  if (parts > 1) {
    cluster_wait();
    if (tid < parts) {
      const uint32_t to = in_block(&room.of_part[part], tid);
      asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\tst.shared::cluster.f32 [%0 + 8], %3;" :: "r"(to), "f"(s.m), "f"(s.listed), "f"(s.others) : "memory");
    }
    cluster_arrive();
    cluster_wait();                                            // (and no block writes over scores that another still reads)
    s = join_lanes(lane < parts ? room.of_part[lane] : nobody, c);
  }
  const float all = s.listed + s.others, m0 = s.m == -INFINITY ? 0.f : s.m;
  base = base_of(s.m, c);
  if (warp == 0 && part == 0 && a.loss) {
    const float off = log_excess(s.m, base, c), log_all = all == 0.f ? 0.f : logf(all) - off;
    float sum = 0.f;
    for (int k = lane; k < a.K; k += 32) {
      const float q = room.q[k];
      if (q != 0.f) sum += q * (room.log_q[k] - ((room.score[k] - m0) * a.scale - log_all));
    }
    if (REST && lane == 0 && room.q_rest != 0.f) sum += room.q_rest * (room.log_q_rest - (logf(s.others) - off - log_all));
    sum = warp_sum(sum);
    if (lane == 0) a.loss[n] = sum;
  }
  if (!grad) return;

  const RowBatches<T> to(grad + n * a.grad_stride, a.V);
  const RowUnder<T> under(r.row, to);
  const int32_t g0 = min(to.count, part * a.share), g1 = min(to.count, g0 + a.share);
  const float w = (a.weights ? a.weights[n] : 1.f) * a.scale, inv_all = all == 0.f ? 0.f : 1.f / all, total = room.total;
  if (w == 0.f || total == 0.f) {
    const float zero[E] = {};
    for (int32_t b = g0 + tid; b < g1; b += threads) to.store(b, zero);
    return;
  }
  const float f = w * (REST && room.q_rest != 0.f && s.others != 0.f ? inv_all - room.q_rest / s.others : inv_all) + total * 0.f;
  const bool usual = ordinary(base);
  const auto gradient = [&](const uint4& x, float (&v)[E]) {
    RowBatches<T>::unpack(x, v);
    const Pair minus(-base, -base), c2(c, c), f2(f, f);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 d = usual ? fma2(Pair(v[e], v[e + 1]), c2, minus).get() : make_float2((v[e] - m0) * c, (v[e + 1] - m0) * c);
      const float2 g = (Pair(exp2_fast(d.x), exp2_fast(d.y)) * f2).get();
      v[e] = g.x;
      v[e + 1] = g.y;
    }
  };
  constexpr int GU = DISTILL_GRAD_UNROLL;
  int32_t in0, in1;
  under.inner(&in0, &in1);
  in1 = min(in1, g1);
  for (int32_t g = g0; g < g1; g += threads * GU) {
    const int32_t b = g + tid;
    float v[E];
    if (usual && g >= in0 && g + threads * GU <= in1) {        // nothing to test
      const T* from = r.row + (to.first(b) - under.ahead);
      T* at = grad + n * a.grad_stride + to.first(b);
      uint4 x[GU];
#pragma unroll
      for (int u = 0; u < GU; ++u, from += threads * E) x[u] = under.inside(from);
#pragma unroll
      for (int u = 0; u < GU; ++u, at += threads * E) {
        RowBatches<T>::unpack(x[u], v);
        const Pair minus(-base, -base), c2(c, c), f2(f, f);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 d = fma2(Pair(v[e], v[e + 1]), c2, minus).get();
          const float2 y = (Pair(exp2_fast(d.x), exp2_fast(d.y)) * f2).get();
          v[e] = y.x;
          v[e + 1] = y.y;
        }
        RowBatches<T>::store16(at, v);
      }
    } else {
#pragma unroll 1
      for (int32_t q = b; q < min(g1, g + threads * GU); q += threads) {
        gradient(under.raw(q), v);
        to.store(q, v);
      }
    }
  }
  __syncthreads();
  // the listed items' places once more, by the block that wrote them
  for (int k = tid; k < a.K; k += threads) {
    const int32_t i = room.at[k];
    if (i < 0) continue;
    const int32_t b = (i + to.shift) / E;
    if (b < g0 || b >= g1) continue;
    float want = 0.f;
    for (int j = 0; j < a.K; ++j) want += room.at[j] == i ? room.q[j] : 0.f;
    const float p = exp2_fast(usual ? fmaf(room.score[k], c, -base) : (room.score[k] - m0) * c) * inv_all;
    grad[n * a.grad_stride + i] = from_f32<T>(w * (p - want) + total * 0.f);
  }
}

template <typename T, bool REST>
int launch_distill(const char* what, const T* logits, T* grad, const DistillCall& a, int64_t N, int warps, cudaStream_t s) {
  cudaLaunchAttribute cluster;
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = 1u << a.log_parts;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3((unsigned)(N << a.log_parts));
  config.blockDim = dim3(32 * warps);
  const int64_t groups = ceil_div(a.share, 32 * warps * DISTILL_UNROLL);
  config.dynamicSmemBytes = !REST ? 0 : (size_t)(groups * 32 * warps < LISTED_BYTES ? groups * 32 * warps : LISTED_BYTES);
  config.stream = s;
  config.attrs = &cluster;
  config.numAttrs = a.log_parts ? 1 : 0;
  LaunchScope scope(K_DISTILL, s);
  return check_cuda(cudaLaunchKernelEx(&config, distill_loss<T, REST>, logits, grad, a), what);
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
  if (!(scale > 0.f && scale <= 1e30f)) return set_error(MTS_ERR_INVALID_ARG, "%s: scale %g", what, scale);
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
    const int64_t batches = ceil_div(V, RowBatches<T>::E) + 1;          // wherever rows start
    const int log_parts = log_parts_of(N, batches);
    const int32_t share = (int32_t)ceil_div(batches, 1 << log_parts);
    int warps = share <= 700 ? 1 : share <= 3000 ? 2 : share <= 8000 ? 4 : 8;
    while (warps < DISTILL_WARPS && (N << log_parts) * warps < 148 * 16 && share >= (warps < 8 ? 64 : 256) * warps) warps *= 2;
    const DistillCall a = {row_stride, grad_stride, teacher_index, teacher_logits, teacher_rest, weights, loss, (int32_t)V, K, teacher_dtype, log_parts, share, scale};
    const T* x = static_cast<const T*>(logits);
    T* d = static_cast<T*>(grad_logits);
    return teacher_rest ? launch_distill<T, true>(what, x, d, a, N, warps, s) : launch_distill<T, false>(what, x, d, a, N, warps, s);
  });
}
