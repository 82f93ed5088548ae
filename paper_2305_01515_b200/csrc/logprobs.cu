// Log probabilities of given items under a softmax over V scores, with its entropy and the best alternatives, and their gradient.
//
//   z = scale x,  m = max x,  S = sum_v exp(scale (x_v - m)),  log p_v = scale (x_v - m) - log S
//   entropy = -sum_v p_v log p_v = log S - (sum_v exp(scale (x_v - m)) scale (x_v - m)) / S
//   dx_v = scale (g_logp ([v = target] - p_v) - g_entropy p_v (log p_v + entropy))
#include "rows.cuh"

namespace mts {

constexpr int LOGP_THREADS = 256;
constexpr int LOGP_MAX_PARTS = 8;              // blocks of a cluster that share a row
constexpr int LOGP_UNROLL = 4;                 // batches on their way for a thread

struct LogprobsOut {
  float* logp;
  float* entropy;
  float* stats;
  int64_t* top_index;
  float* top_logp;
};

// Statistics of a set of scores: the largest, and relative to it the sums of p = 2^(c (x - m)) and of p log2 p.
struct RowStats {
  float m, S, P;
  // those of two sets together
  __device__ __forceinline__ void join(const RowStats& o, float c) {
    const float top = fmaxf(m, o.m), base = top == -INFINITY ? 0.f : top;
    const float a = exponent((m - base) * c), b = exponent((o.m - base) * c), fa = exp2_fast(a), fb = exp2_fast(b);
    P = fa * (P + S * a) + fb * (o.P + o.S * b);
    S = fa * S + fb * o.S;
    m = top;
  }
};

// Those of the first LANES lanes (a power of two) together, in all lanes.
template <int LANES>
__device__ __forceinline__ RowStats join_lanes(RowStats st, float c) {
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    const RowStats other = {__shfl_xor_sync(0xFFFFFFFFu, st.m, o), __shfl_xor_sync(0xFFFFFFFFu, st.S, o), __shfl_xor_sync(0xFFFFFFFFu, st.P, o)};
    st.join(other, c);
  }
  if constexpr (LANES < 32) st = {__shfl_sync(0xFFFFFFFFu, st.m, 0), __shfl_sync(0xFFFFFFFFu, st.S, 0), __shfl_sync(0xFFFFFFFFu, st.P, 0)};
  return st;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// Address in the first block of the cluster of a variable of this block.
__device__ __forceinline__ uint32_t in_first_block(const void* p) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)));
  return a;
}

// A row by a cluster of blocks, each a run of batches, each thread every THREADS-th of them.  One pass over the scores:
//   Sums: a thread keeps the running maximum of its scores and the sums relative to it; where a group of batches has a larger score the sums are
//   scaled (rare after the first few).  They are joined over warp, block and cluster.
//   Best k: nothing is kept but the batch in which each thread's maximum came first.  With (score, index) ordered so that the lowest index comes first
//   among equals, a thread's order is at least that of all its scores, and the k-th largest of the 32 largest orders of groups of threads is a
//   bound that k scores reach.  Only the few threads whose order reaches it can hold more of them: a warp reads each such thread's batches again
//   (k / THREADS of the row about), collects the scores that reach the bound, and a score's place is the number of those before it.  Where the bound
//   lets too many pass (a row made for it) or too few (NaN), the block finds its best one after the other.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS)
logprobs_forward(const T* __restrict__ logits, int64_t row_stride, int32_t V, float scale, const int64_t* __restrict__ targets, int top_k, int parts,
                 LogprobsOut out) {
  constexpr int E = RowBatches<T>::E, WARPS = THREADS / 32, CAP = THREADS < 64 ? 256 : 512;
  __shared__ RowStats warp_stats[WARPS], part_stats[LOGP_MAX_PARTS];
  __shared__ uint64_t room64[32], found[CAP], part_best[LOGP_MAX_PARTS * MTS_LOGPROBS_MAX_TOP], best[MTS_LOGPROBS_MAX_TOP];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  const int64_t n = blockIdx.x / parts;
  const int part = blockIdx.x % parts;
  if (parts > 1) cluster_arrive();                                      // the first block has begun before others write to it
  const RowBatches<T> r(logits + n * row_stride, V);
  const int32_t b0 = (int32_t)((int64_t)r.count * part / parts), b1 = (int32_t)((int64_t)r.count * (part + 1) / parts);
  const float c = scale * LOG2E;
  int64_t target = -1;
  float target_score = 0.f;
  if (part == 0 && tid == 0 && out.logp) {
    target = targets[n];
    if (target >= 0 && target < V) target_score = to_f32(r.row[target]);
  }
  if (tid == 0) count = 0;

  float m = -INFINITY, base = 0.f;
  Pair S(0.f, 0.f), P(0.f, 0.f);
  const Pair c2(c, c);
  int32_t best_batch = b0 + tid;
  for (int32_t g = b0; g < b1; g += THREADS * LOGP_UNROLL) {
    uint4 w[LOGP_UNROLL];
    const int32_t b = g + tid;
    if (g > 0 && g + THREADS * LOGP_UNROLL < r.count && g + THREADS * LOGP_UNROLL <= b1) {
#pragma unroll
      for (int u = 0; u < LOGP_UNROLL; ++u) w[u] = __ldg(reinterpret_cast<const uint4*>(r.row + r.first(b + u * THREADS)));
    } else {
#pragma unroll
      for (int u = 0; u < LOGP_UNROLL; ++u) w[u] = r.raw(b + u * THREADS < b1 ? b + u * THREADS : r.count);
    }
    float top[LOGP_UNROLL];
#pragma unroll
    for (int u = 0; u < LOGP_UNROLL; ++u) top[u] = max_of<T>(w[u]);
    float most = top[0];
#pragma unroll
    for (int u = 1; u < LOGP_UNROLL; ++u) most = fmaxf(most, top[u]);
    if (most > m) {
      const float a = exponent((m - most) * c), f = exp2_fast(a);
      P = (P + S * Pair(a, a)) * Pair(f, f);
      S = S * Pair(f, f);
#pragma unroll
      for (int u = LOGP_UNROLL - 1; u >= 0; --u)
        if (top[u] == most) best_batch = b + u * THREADS;
      m = base = most;
    }
    const Pair minus(-base, -base);
#pragma unroll
    for (int u = 0; u < LOGP_UNROLL; ++u) {
      float v[E];
      RowBatches<T>::unpack(w[u], v);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 d = ((Pair(v[e], v[e + 1]) + minus) * c2).get();
        const float d0 = exponent(d.x), d1 = exponent(d.y);
        const Pair p(exp2_fast(d0), exp2_fast(d1));
        S = S + p;
        P = fma2(p, Pair(d0, d1), P);
      }
    }
  }
  RowStats st = {m, S.get().x + S.get().y, P.get().x + P.get().y};
  st = join_lanes<32>(st, c);
  // the thread's order, and the largest of its group of THREADS / 32 threads
  uint64_t order = 0;
  if (b0 + tid < b1) order = score_order(m, max(r.first(best_batch), 0));
  uint64_t group = order;
#pragma unroll
  for (int o = THREADS / 64; o; o >>= 1) group = max(group, __shfl_xor_sync(0xFFFFFFFFu, group, o));
  if (lane % (THREADS / 32) == 0) room64[tid / (THREADS / 32)] = group;
  if (lane == 0) warp_stats[warp] = st;
  __syncthreads();

  const int k = min((int64_t)top_k, (int64_t)V);
  if (k > 0) {
    // the k-th largest of the 32
    const uint64_t mine = room64[lane];
    int before = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const uint64_t o = room64[i];
      before += o > mine || (o == mine && i < lane);
    }
    const unsigned kth = __ballot_sync(0xFFFFFFFFu, before == k - 1);
    uint64_t bound = __shfl_sync(0xFFFFFFFFu, mine, __ffs(kth) - 1);
    bound = bound > E ? bound - (E - 1) : 0;                            // the score itself lies up to E - 1 places behind its batch's first
    unsigned winners = __ballot_sync(0xFFFFFFFFu, order >= bound && b0 + tid < b1);
    while (winners) {
      const int w = __ffs(winners) - 1;
      winners &= winners - 1;
      for (int32_t b = b0 + warp * 32 + w + lane * THREADS; b < b1; b += 32 * THREADS) {
        float v[E];
        RowBatches<T>::unpack(r.raw(b), v);
        const int32_t i = r.first(b);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint64_t o = score_order(v[e], i + e);
          if (o >= bound && i + e >= 0 && i + e < V) {
            const int at = atomicAdd(&count, 1);
            if (at < CAP) found[at] = o;
          }
        }
      }
    }
    __syncthreads();
    const int have = count;
    if (have <= CAP && (have >= k || bound == 0)) {
      if (tid < k) best[tid] = 0;
      __syncthreads();
      for (int i = tid; i < have; i += THREADS) {
        const uint64_t o = found[i];
        int place = 0;
        for (int j = 0; j < have; ++j) place += found[j] > o;
        if (place < k) best[place] = o;
      }
    } else {
      uint64_t last = ~0ull;
      for (int q = 0; q < k; ++q) {
        uint64_t top = 0;
        for (int32_t b = b0 + tid; b < b1; b += THREADS) {
          float v[E];
          RowBatches<T>::unpack(r.raw(b), v);
          const int32_t i = r.first(b);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint64_t o = score_order(v[e], i + e);
            if (i + e >= 0 && i + e < V && o < last && o > top) top = o;
          }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        __syncthreads();
        if (lane == 0) room64[warp] = top;
        __syncthreads();
        for (int w = 0; w < WARPS; ++w) top = max(top, room64[w]);
        last = top;
        if (tid == 0) best[q] = top;
      }
    }
    __syncthreads();
  }
  const RowStats nobody = {-INFINITY, 0.f, 0.f};
  st = join_lanes<WARPS>(lane < WARPS ? warp_stats[lane] : nobody, c);

  if (parts > 1) {
    // to the first block, which joins them
    cluster_wait();
    const uint32_t to = in_first_block(&part_stats[part]);
    if (tid == 0)
      asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\tst.shared::cluster.f32 [%0 + 8], %3;" :: "r"(to), "f"(st.m), "f"(st.S), "f"(st.P) : "memory");
    if (tid < k) asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(in_first_block(&part_best[part * k + tid])), "l"(best[tid]) : "memory");
    cluster_arrive();
    cluster_wait();
    if (part != 0) return;
    st = join_lanes<LOGP_MAX_PARTS>(lane < parts ? part_stats[lane] : nobody, c);
    for (int i = tid; i < parts * k; i += THREADS) {
      const uint64_t o = part_best[i];
      int place = 0;
      for (int j = 0; j < parts * k; ++j) place += part_best[j] > o;
      if (place < k && o != 0) best[place] = o;
    }
    __syncthreads();
  }
  base = st.m == -INFINITY ? 0.f : st.m;
  const float log_s = st.S > 0.f ? logf(st.S) : st.S == 0.f ? 0.f : NAN;
  const float nothing = st.S == 0.f ? -INFINITY : 0.f;
  if (tid == 0) {
    if (out.logp) out.logp[n] = target < 0 ? 0.f : target >= V ? NAN : (target_score - base) * scale - log_s + nothing;
    if (out.entropy) out.entropy[n] = st.S == 0.f ? 0.f : log_s - st.P / st.S * LN2;
    if (out.stats) {
      out.stats[2 * n] = base;
      out.stats[2 * n + 1] = log_s;
    }
  }
  if (tid < k) {
    const uint64_t o = best[tid];
    if (out.top_index) out.top_index[n * top_k + tid] = order_index(o);
    if (out.top_logp) out.top_logp[n * top_k + tid] = (order_score(o) - base) * scale - log_s + nothing;
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

template <typename T, int THREADS>
int launch_forward(const char* what, const T* logits, int64_t row_stride, int64_t N, int64_t V, float scale, const int64_t* targets, int top_k, int parts,
                   const LogprobsOut& out, cudaStream_t s) {
  cudaLaunchAttribute cluster;
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = (unsigned)parts;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3((unsigned)(N * parts));
  config.blockDim = dim3(THREADS);
  config.stream = s;
  config.attrs = &cluster;
  config.numAttrs = parts > 1 ? 1 : 0;
  LaunchScope scope(K_LOGPROBS_FWD, s);
  return check_cuda(cudaLaunchKernelEx(&config, logprobs_forward<T, THREADS>, logits, row_stride, (int32_t)V, scale, targets, top_k, parts, out), what);
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
    const int64_t batches = ceil_div(V, RowBatches<T>::E);
    int threads = 32, parts = 1;
    while (threads < 512 && batches >= 8 * threads) threads *= 2;
    while (parts < LOGP_MAX_PARTS && N * parts < 296 && batches >= 1024 * parts) parts *= 2;
    const T* x = static_cast<const T*>(logits);
    switch (threads) {
      case 32: return launch_forward<T, 32>(what, x, row_stride, N, V, scale, targets, top_k, parts, out, s);
      case 64: return launch_forward<T, 64>(what, x, row_stride, N, V, scale, targets, top_k, parts, out, s);
      case 128: return launch_forward<T, 128>(what, x, row_stride, N, V, scale, targets, top_k, parts, out, s);
      case 256: return launch_forward<T, 256>(what, x, row_stride, N, V, scale, targets, top_k, parts, out, s);
      default: return launch_forward<T, 512>(what, x, row_stride, N, V, scale, targets, top_k, parts, out, s);
    }
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
