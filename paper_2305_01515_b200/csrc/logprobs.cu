// Log probabilities of given items under a softmax over V scores, with its entropy and the best alternatives, and their gradient.
//
//   z = scale x,  m = max x,  S = sum_v exp(scale (x_v - m)),  log p_v = scale (x_v - m) - log S
//   entropy = -sum_v p_v log p_v = log S - (sum_v exp(scale (x_v - m)) scale (x_v - m)) / S
//   dx_v = scale (g_logp ([v = target] - p_v) - g_entropy p_v (log p_v + entropy))
//
// Scores are read once forward; backward they are read and the gradient written once.  Statistics are fp32; outputs are rounded to their type once.  Reading bounds both passes
// until the instructions do (about six a score forward): the exponential is one instruction on a rounded base whose error is put right in the logarithm,
// sums go by pairs, maxima by pairs (16 bits) or threes (fp32).
#include "rows.cuh"

namespace mts {

constexpr int LOGP_WARPS = 16;                 // of a block that works on a row
constexpr int LOGP_ROWS = 4;                   // rows of a block whose warps have one each
constexpr int LOGP_MAX_PARTS = 1 << MAX_LOG_PARTS;      // blocks of a cluster that share a row
constexpr int LOGP_UNROLL = 8;                 // batches on their way for a thread: a group
constexpr int LOGP_UNITS = 8;                  // runs of a thread's groups whose maxima are kept
constexpr int LOGP_HITS = 128;                 // of them that can hold a score which reaches the bound
constexpr int LOGP_FOUND = 512;                // scores that can reach it

struct LogprobsOut {
  float* logp;
  float* entropy;
  float* stats;
  int64_t* top_index;
  float* top_logp;
};

// Statistics of a set of scores: the largest, and the sums of p = 2^exponent and of p log2 p.
struct RowStats { float m, S, P; };

__device__ __forceinline__ RowStats scaled_to(const RowStats& s, float m, float c) {
  const float a = exponent(change_of_base(s.m, m, c)), f = exp2_fast(a);
  return s.m == -INFINITY ? RowStats{m, s.S, s.P} : RowStats{m, f * s.S, f * (s.P + s.S * a)};
}
// Those of a warp's lanes together.
__device__ __forceinline__ RowStats join_lanes(RowStats s, float c) {
  const float m = warp_max(s.m);
  s = scaled_to(s, m, c);
  return {m, warp_sum(s.S), warp_sum(s.P)};
}

// A batch added to the sums.
template <typename T, bool ORDINARY>
__device__ __forceinline__ void add_batch(const uint4& w, float m, float base, float c, Pair& S, Pair& P) {
  constexpr int E = RowBatches<T>::E;
  float v[E];
  RowBatches<T>::unpack(w, v);
  const Pair minus(-base, -base), c2(c, c);
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const float2 f = ORDINARY ? fma2(Pair(v[e], v[e + 1]), c2, minus).get() : make_float2((v[e] - m) * c, (v[e + 1] - m) * c);
    const float d0 = exponent(f.x), d1 = exponent(f.y);
    const Pair p(exp2_fast(d0), exp2_fast(d1));
    S = S + p;
    P = fma2(p, Pair(d0, d1), P);
  }
}

// Working memory of a row, behind which lie, for W warps: float top[2 W][32], each thread's maxima of its even and of its odd units, and float
// unit[LOGP_UNITS][32 W].
struct RowRoom {
  uint64_t found[LOGP_FOUND], best[MTS_LOGPROBS_MAX_TOP], bound;
  int32_t hits[LOGP_HITS];
  RowStats stats[LOGP_WARPS];
  float bound_score, m, log_s, nothing;
  int hit_count, found_count;
};
constexpr int LOGP_ROOM = (sizeof(RowRoom) + 15) / 16 * 16;
__host__ __device__ constexpr int room_bytes(int warps) { return LOGP_ROOM + (2 + LOGP_UNITS) * 32 * 4 * warps; }

// The k-th largest of the maxima of 32 R groups of threads (X: float or uint64_t), by one warp; `of_thread` is used up.  Equal ones count one by one.
template <int R, typename X>
__device__ __forceinline__ X kth_largest(X (*of_thread)[32], int rows, int k, X least, X most) {
  constexpr int PER = 16 / (int)sizeof(X);
  const int lane = lane_id();
  X mine[R];
#pragma unroll
  for (int q = 0; q < R; ++q) {
    mine[q] = least;
    for (int w = q; w < rows; w += R) mine[q] = max(mine[q], of_thread[w][lane]);
  }
  __syncwarp();
  X* flat = &of_thread[0][0];
#pragma unroll
  for (int q = 0; q < R; ++q) flat[q * 32 + lane] = mine[q];
  __syncwarp();
  int before[R] = {};
#pragma unroll 4
  for (int i = 0; i < 32 * R; i += PER) {
    X o[PER];
    *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(flat + i);
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
      for (int e = 0; e < PER; ++e) before[q] += o[e] > mine[q];
  }
  // the smallest of those with fewer than k before them
  X bound = before[0] < k ? mine[0] : most;
#pragma unroll
  for (int q = 1; q < R; ++q)
    if (before[q] < k && mine[q] < bound) bound = mine[q];
  if constexpr (sizeof(X) == 4) return warp_min(bound);
#pragma unroll
  for (int o = 16; o; o >>= 1) bound = min(bound, __shfl_xor_sync(0xFFFFFFFFu, bound, o));
  return bound;
}
template <typename X>
__device__ __forceinline__ X kth_of_groups(X (*of_thread)[32], int rows, int k, X least, X most) {
  return k <= 16 || rows < 2 ? kth_largest<1>(of_thread, rows, k, least, most) : kth_largest<2>(of_thread, rows, k, least, most);
}

// The best k of batches [b0, b1) into room.best where the bound by score alone lets too many pass or too few: rows with many equal scores (ruled out
// altogether, say), and rows with NaN.  The threads find where their maximum came first and the bound is made of (score, index); where that does not
// settle it either, the best are found one after the other.
template <typename T, bool ONE_WARP>
__device__ __noinline__ void best_of_equals(const RowBatches<T> r, int32_t b0, int32_t b1, int k, RowRoom& room) {
  constexpr int E = RowBatches<T>::E;
  const int lane = lane_id(), warp = ONE_WARP ? 0 : threadIdx.x / 32, tid = ONE_WARP ? lane : threadIdx.x;
  const int threads = ONE_WARP ? 32 : blockDim.x, warps = threads / 32;
  const auto sync = [] { if (ONE_WARP) __syncwarp(); else __syncthreads(); };
  const int32_t b = b0 + tid;
  uint64_t order = 0;
  float m = -INFINITY;
  for (int32_t at = b; at < b1; at += threads) {
    const float most = max_value<T>(max_bits<T>(r.raw(at)));
    if (most > m || !order) order = score_order(most, max(r.first(at), 0));
    m = fmaxf(m, most);
  }
  sync();                                                               // what was found before has been looked at
  uint64_t(*orders)[32] = reinterpret_cast<uint64_t(*)[32]>(room.found);
  orders[warp][lane] = order;
  sync();
  if (warp == 0) {
    // the score itself lies up to E - 1 places behind its batch's first
    const uint64_t kth = kth_of_groups<uint64_t>(orders, warps, k, 0, ~0ull);
    if (lane == 0) {
      room.bound = kth > E ? kth - (E - 1) : 0;
      room.found_count = 0;
    }
  }
  sync();
  const uint64_t bound = room.bound;
  if (order >= bound) {
    for (int32_t at = b; at < b1 && *const_cast<volatile int*>(&room.found_count) <= LOGP_FOUND; at += threads) {
      float v[E];
      RowBatches<T>::unpack(r.raw(at), v);
      const int32_t i = r.first(at);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint64_t o = score_order(v[e], i + e);
        if (o >= bound && i + e >= 0 && i + e < r.V) {
          const int place = atomicAdd(&room.found_count, 1);
          if (place < LOGP_FOUND) room.found[place] = o;
        }
      }
    }
  }
  if (tid < k) room.best[tid] = 0;
  sync();
  const int have = room.found_count;
  if (have <= LOGP_FOUND && (have >= k || bound == 0)) {
    for (int i = tid; i < have; i += threads) {
      const uint64_t o = room.found[i];
      int place = 0;
      for (int j = 0; j < have; ++j) place += room.found[j] > o;
      if (place < k) room.best[place] = o;
    }
  } else {
    uint64_t last = ~0ull;
    for (int q = 0; q < k; ++q) {
      uint64_t most = 0;
      for (int32_t at = b; at < b1; at += threads) {
        float v[E];
        RowBatches<T>::unpack(r.raw(at), v);
        const int32_t i = r.first(at);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint64_t o = score_order(v[e], i + e);
          if (i + e >= 0 && i + e < r.V && o < last && o > most) most = o;
        }
      }
      for (int o = 16; o; o >>= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
      sync();
      if (lane == 0) room.found[warp] = most;
      sync();
      for (int x = 0; x < warps; ++x) most = max(most, room.found[x]);
      last = most;
      if (tid == 0) room.best[q] = most;
    }
  }
  sync();
}

// A row (or a part of it, by a cluster of blocks) by the warps of a block, each thread every T-th whole batch of it, and a few lanes the elements before
// and behind these; where there are rows enough a warp has one for itself.  A thread keeps the running maximum of its scores and sums relative to it, which are scaled where a group of its batches has a
// larger one (rare after the first few).
// The best k cost the pass nothing but the maxima of each thread's groups, or of up to LOGP_UNITS runs of them: the k-th largest of the
// maxima of 32 or 64 groups of threads is a bound that at least k scores reach, and few others.  The units whose maxima reach it are read again, and a
// score's place is the number of those found before it, where (score, index) are ordered so that the lowest index comes first among equals.
// SHORT: rows of one group of a warp, which list the batches themselves instead of units.
// us without and with the best: 30,011 x 5,001 fp32, 10 of them, 99 and 141-148 (6.1 and 4.1-4.3 TB/s); 2,048 x 131,072 bf16, 16, 93-95 and 104-115 (5.7 and 4.7-5.2);
// 20,000 x 4,000 fp16, 20, - and 73; one row of 100,000, 20, 8.5-10.6: a chain of the cluster's exchange and three barriers.  Groups of four batches and 48 registers a thread (40 warps an SM instead of 32) took 167
// for the first: eight loads on their way hide more than the warps.  Ends as masked batches of the main loop took 160.
template <typename T, bool ONE_WARP, bool SHORT>
__global__ void __launch_bounds__(ONE_WARP ? LOGP_ROWS * 32 : LOGP_WARPS * 32, ONE_WARP ? 8 : 2)
logprobs_forward(const T* __restrict__ logits, int64_t row_stride, int64_t N, int32_t V, float scale, const int64_t* __restrict__ targets, int top_k, int log_parts,
                 int32_t share, int log_unit, LogprobsOut out) {
  constexpr int E = RowBatches<T>::E, U = LOGP_UNROLL;
  extern __shared__ __align__(16) unsigned char rooms[];
  __shared__ RowStats part_stats[ONE_WARP ? 1 : LOGP_MAX_PARTS];
  __shared__ uint64_t part_best[ONE_WARP ? 1 : LOGP_MAX_PARTS * MTS_LOGPROBS_MAX_TOP];
  const int lane = lane_id(), warp = ONE_WARP ? 0 : threadIdx.x / 32, tid = ONE_WARP ? lane : threadIdx.x;
  const int threads = ONE_WARP ? 32 : blockDim.x, warps = threads / 32;
  unsigned char* const mine = rooms + (ONE_WARP ? threadIdx.x / 32 * room_bytes(1) : 0);
  RowRoom& room = *reinterpret_cast<RowRoom*>(mine);
  float(*const top)[32] = reinterpret_cast<float(*)[32]>(mine + LOGP_ROOM);
  float* const unit_top = &top[2 * warps][0];
  const int parts = ONE_WARP ? 1 : 1 << log_parts, part = ONE_WARP ? 0 : blockIdx.x & (parts - 1);
  const int64_t n = ONE_WARP ? (int64_t)blockIdx.x * LOGP_ROWS + threadIdx.x / 32 : blockIdx.x >> log_parts;
  if (ONE_WARP && n >= N) return;
  const auto sync = [] { if (ONE_WARP) __syncwarp(); else __syncthreads(); };
  if (!ONE_WARP && parts > 1) cluster_arrive();                         // the first block has begun before others write to it
  const RowBatches<T> r(logits + n * row_stride, V);
  const int32_t b0 = min(r.whole_end, r.whole_begin + part * share), b1 = min(r.whole_end, b0 + share);
  const float c = scale * LOG2E;
  const int k = top_k;
  // an element of the row's ends, for some lanes of the first warp
  float edge = -INFINITY;
  if (warp == 0 && lane < 2 * E) {
    const int32_t i = r.edge(lane);
    if (i >= 0 && (lane < E ? part == 0 : part == parts - 1)) edge = to_f32(r.row[i]);
  }
  int64_t target = -1;
  float target_score = 0.f;
  if (part == 0 && tid == 0 && out.logp) {
    target = targets[n];
    if (target >= 0 && target < V) target_score = to_f32(r.row[target]);
  }
  if (tid == 0) room.hit_count = room.found_count = 0;

  const uint4 nothing_there = make_uint4(RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW);
  float m = -INFINITY, base = 0.f, of_unit = -INFINITY, of_units[2] = {-INFINITY, -INFINITY};
  Pair S(0.f, 0.f), P(0.f, 0.f);
  const auto rescale = [&](float most) {
    const RowStats s = scaled_to({m, S.sum(), P.sum()}, most, c);
    S = Pair(s.S, 0.f);
    P = Pair(s.P, 0.f);
    m = most;
    base = base_of(m, c);
  };
  int group = 0;
  uint4 w[U];
  for (int32_t g = b0; g < b1; g += threads * U, ++group) {
    const int32_t b = g + tid, left = b1 - (b - lane);                  // of the warp's first batch
    const T* p = r.row + r.first(b);
    if (left > (U - 1) * threads + 31) {
#pragma unroll
      for (int u = 0; u < U; ++u, p += threads * E) w[u] = r.load16(p);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u, p += threads * E) {
        w[u] = nothing_there;
        if (b + u * threads < b1) w[u] = r.load16(p);
      }
    }
    uint32_t most_bits = max_bits<T>(w[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) most_bits = max_bits<T>(most_bits, w[u]);
    const float most = max_value<T>(most_bits);
    if (k > 0 && !SHORT) {
      const int unit = group >> log_unit;
      of_unit = unit << log_unit == group ? most : fmaxf(of_unit, most);
      unit_top[unit * threads + tid] = of_unit;
      of_units[unit & 1] = fmaxf(of_units[unit & 1], most);
    }
    if (most > m) rescale(most);
    if (ordinary(base)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (u * threads >= left) break;
        add_batch<T, true>(w[u], m, base, c, S, P);
      }
    } else {
#pragma unroll 1
      for (int32_t at = b; at < min(b1, g + threads * U); at += threads) add_batch<T, false>(r.raw(at), m, base, c, S, P);
    }
    if (SHORT) break;
  }
  if (edge != -INFINITY) {
    if (edge > m) rescale(edge);
    const float d = exponent(ordinary(base) ? fmaf(edge, c, -base) : (edge - m) * c), p = exp2_fast(d);
    S = S + Pair(p, 0.f);
    P = P + Pair(p * d, 0.f);
    of_units[0] = fmaxf(of_units[0], edge);
  }
  if (SHORT) of_units[0] = m;
  RowStats st = join_lanes({m, S.sum(), P.sum()}, c);
  if (k > 0) {
    top[2 * warp][lane] = of_units[0];
    top[2 * warp + 1][lane] = of_units[1];
  }
  if (!ONE_WARP && lane == 0) room.stats[warp] = st;
  if (!ONE_WARP || k > 0) sync();
  const RowStats nobody = {-INFINITY, 0.f, 0.f};
  if (warp == 0) {
    if (k > 0) {
      const float kth = kth_of_groups<float>(top, 2 * warps, k, -INFINITY, INFINITY);
      if (lane == 0) room.bound_score = kth;
    }
    if (!ONE_WARP) st = join_lanes(lane < warps ? room.stats[lane] : nobody, c);     // which this warp alone has
  }
  if (k > 0) {
    sync();
    const float bound = room.bound_score;
    // (-infinity: fewer than k of the groups have a score, those of a short row, or ruled out)
    if (m >= bound && bound != -INFINITY) {
      if (edge >= bound) {
        const int at = atomicAdd(&room.found_count, 1);
        if (at < LOGP_FOUND) room.found[at] = score_order(edge, r.edge(lane));
      }
      const auto hit = [&](int unit) {
        const int at = atomicAdd(&room.hit_count, 1);
        if (at < LOGP_HITS) room.hits[at] = unit << 16 | tid;
      };
      if constexpr (SHORT) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (max_value<T>(max_bits<T>(w[u])) >= bound) hit(u);
      } else {
        for (int unit = 0; unit << log_unit < group; ++unit)
          if (unit_top[unit * threads + tid] >= bound) hit(unit);
      }
    }
  }
  if (warp == 0 && (ONE_WARP || parts == 1)) {
    const float m0 = st.m == -INFINITY ? 0.f : st.m, off = log_excess(st.m, base_of(st.m, c), c);
    const float log_sum = logf(st.S), log_s = st.S > 0.f ? log_sum - off : st.S == 0.f ? 0.f : NAN;
    const float nothing = st.S == 0.f ? -INFINITY : 0.f;
    if (lane == 0) {
      room.m = m0;
      room.log_s = log_s;
      room.nothing = nothing;
      if (out.logp) out.logp[n] = target < 0 ? 0.f : target >= V ? NAN : scaled_difference(target_score, m0, scale) - log_s + nothing;
      if (out.entropy) out.entropy[n] = st.S == 0.f ? 0.f : log_sum - st.P / st.S * LN2;
      if (out.stats) {
        out.stats[2 * n] = m0;
        out.stats[2 * n + 1] = log_s;
      }
    }
  }
  if (k == 0 && (ONE_WARP || parts == 1)) return;

  const auto write = [&](int place, uint64_t o) {
    if (out.top_index) out.top_index[n * k + place] = order_index(o);
    if (out.top_logp) out.top_logp[n * k + place] = scaled_difference(order_score(o), room.m, scale) - room.log_s + room.nothing;
  };
  if (k > 0) {
    sync();
    const int hits = room.hit_count;
    const float bound = room.bound_score;
    bool settled = bound != -INFINITY && hits <= LOGP_HITS;
    if (settled) {
      const int log_per = SHORT ? 0 : 3 + log_unit;                                 // a unit's batches
      static_assert(U == 8, "a group of 2^3 batches");
      for (int i = tid; i < hits << log_per; i += threads) {
        const int which = room.hits[i >> log_per];
        const int64_t at = b0 + (which & 0xFFFF) + (((int64_t)(which >> 16) << log_per) + (i & ((1 << log_per) - 1))) * threads;
        if (at >= b1) continue;
        const uint4 batch = r.load16(r.row + r.first((int32_t)at));
        float v[E];
        RowBatches<T>::unpack(batch, v);
        unsigned reach = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) reach |= (v[e] >= bound) << e;
#pragma unroll 1
        for (; reach; reach &= reach - 1) {
          const int32_t j = r.first((int32_t)at) + __ffs(reach) - 1;
          const int place = atomicAdd(&room.found_count, 1);
          if (place < LOGP_FOUND) room.found[place] = score_order(to_f32(r.row[j]), j);
        }
      }
      if (!ONE_WARP && parts > 1 && tid < k) room.best[tid] = 0;
      sync();
      const int have = room.found_count;
      settled = have <= LOGP_FOUND;
      if (settled) {
        for (int i = tid; i < have; i += threads) {
          const uint64_t o = room.found[i];
          int place = 0;
#pragma unroll 8
          for (int j = 0; j < have; ++j) place += room.found[j] > o;
          if (place < k) {
            if (ONE_WARP || parts == 1) write(place, o);
            else room.best[place] = o;
          }
        }
        if (ONE_WARP || parts == 1) return;
        sync();
      }
    }
    if (!settled) {
      best_of_equals<T, ONE_WARP>(r, part == 0 ? 0 : b0, part == parts - 1 ? r.count : b1, k, room);
      if (ONE_WARP || parts == 1) {
        if (tid < k) write(tid, room.best[tid]);
        return;
      }
    }
  }

  if constexpr (!ONE_WARP) {
    // to the first block of the cluster, which joins the parts
    cluster_wait();
    const uint32_t to = in_block(&part_stats[part], 0);
    if (tid == 0)
      asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\tst.shared::cluster.f32 [%0 + 8], %3;" :: "r"(to), "f"(st.m), "f"(st.S), "f"(st.P) : "memory");
    if (tid < k) asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(in_block(&part_best[part * k + tid], 0)), "l"(room.best[tid]) : "memory");
    cluster_arrive();
    cluster_wait();
    if (part != 0) return;
    st = join_lanes(lane < parts ? part_stats[lane] : nobody, c);
    const float m0 = st.m == -INFINITY ? 0.f : st.m, off = log_excess(st.m, base_of(st.m, c), c);
    const float log_sum = logf(st.S), log_s = st.S > 0.f ? log_sum - off : st.S == 0.f ? 0.f : NAN;
    const float nothing = st.S == 0.f ? -INFINITY : 0.f;
    if (tid == 0) {
      if (out.logp) out.logp[n] = target < 0 ? 0.f : target >= V ? NAN : scaled_difference(target_score, m0, scale) - log_s + nothing;
      if (out.entropy) out.entropy[n] = st.S == 0.f ? 0.f : log_sum - st.P / st.S * LN2;
      if (out.stats) {
        out.stats[2 * n] = m0;
        out.stats[2 * n + 1] = log_s;
      }
    }
    for (int i = tid; i < parts * k; i += threads) {
      const uint64_t o = part_best[i];
      int place = 0;
#pragma unroll 8
      for (int j = 0; j < parts * k; ++j) place += part_best[j] > o;
      if (place < k && o != 0) {
        if (out.top_index) out.top_index[n * k + place] = order_index(o);
        if (out.top_logp) out.top_logp[n * k + place] = scaled_difference(order_score(o), m0, scale) - log_s + nothing;
      }
    }
  }
}

// Gradient, dx = p (alpha + beta d) + [v = target] scale g_logp: 4,099 x 50,001 bf16, rows of gradients and of scores at different places, 130-149 us (5.5-6.3 TB/s, 84-96% of
// the copy rate); issue slots 87% busy with the shifts.  A thread takes BACK_UNROLL batches of the gradient's row (16 bytes that start on a 16-byte boundary of it) and reads the scores that lie under them.
constexpr int BACK_THREADS = 256, BACK_UNROLL = 4;

template <typename T>
__global__ void __launch_bounds__(BACK_THREADS, 8)
logprobs_backward(const T* logits, int64_t row_stride, int32_t V, float scale, const int64_t* __restrict__ targets, const float* __restrict__ stats,
                  const float* __restrict__ entropy, const float* __restrict__ grad_logp, const float* __restrict__ grad_entropy, T* grad_logits,
                  int64_t grad_stride, int32_t pieces) {
  constexpr int E = RowBatches<T>::E, U = BACK_UNROLL;
  const int64_t n = blockIdx.x / pieces;
  const int32_t piece = blockIdx.x - (int32_t)(n * pieces);
  const RowBatches<T> r(grad_logits + n * grad_stride, V);
  const RowUnder<T> under(logits + n * row_stride, r);
  const float c = scale * LOG2E, m = stats[2 * n], log_s = stats[2 * n + 1];
  const int64_t t = targets ? targets[n] : -1;
  const float g = grad_logp ? grad_logp[n] : 0.f, gl = t < 0 || g == 0.f ? 0.f : t >= V ? NAN : g, gh = grad_entropy ? grad_entropy[n] : 0.f;
  // dx = p (alpha + beta d) + [v = target] scale gl, with d = log2 of exp(scale (x - m)) and p = 2^(d - bias)
  const float alpha = -scale * (gl + (gh != 0.f ? gh * (entropy[n] - log_s) : 0.f)), beta = -scale * gh * LN2, bias = log_s * LOG2E;
  const bool any = gl != 0.f || gh != 0.f;
  const Pair minus(-0.5f * m, -0.5f * m), c2(2.f * c, 2.f * c);
  const int32_t b = piece * (int)(blockDim.x * U) + threadIdx.x;
  uint4 w[U];
  if (any) {
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = under.raw(b + u * (int)blockDim.x);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int32_t at = b + u * (int)blockDim.x, i = r.first(at);
    if (at >= r.count) break;
    float v[E];
    if (any) {
      RowBatches<T>::unpack(w[u], v);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 x = (fma2(Pair(v[e], v[e + 1]), Pair(0.5f, 0.5f), minus) * c2).get();      // as in scaled_difference
        const Pair d(exponent(x.x), exponent(x.y));
        const float2 f = (d + Pair(-bias, -bias)).get(), y = (Pair(exp2_fast(f.x), exp2_fast(f.y)) * fma2(Pair(beta, beta), d, Pair(alpha, alpha))).get();
        v[e] = y.x;
        v[e + 1] = y.y;
      }
      if (t >= i && t < i + E) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (t == i + e) v[e] += scale * gl;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = 0.f;
    }
    r.store(at, v);
  }
}

}  // namespace mts

using namespace mts;

namespace {

int check_logits(const char* what, const void* logits, int64_t row_stride, int32_t dtype, int64_t N, int64_t V, float scale) {
  if (!known_dtype(dtype)) return set_error(MTS_ERR_INVALID_ARG, "%s: dtype %d", what, dtype);
  if (N < 0 || V < 1) return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, V %lld", what, (long long)N, (long long)V);
  if (N > MTS_SCORES_MAX_N || V > MTS_SCORES_MAX_V) return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, V %lld", what, (long long)N, (long long)V);
  if (!(scale > 0.f && scale <= 1e30f)) return set_error(MTS_ERR_INVALID_ARG, "%s: scale %g", what, scale);
  return check_rows(what, "logits", logits, dtype, N, V, row_stride);
}

struct ForwardCall {
  int64_t row_stride, N;
  int32_t V;
  float scale;
  const int64_t* targets;
  int top_k;
  LogprobsOut out;
  cudaStream_t stream;
};

template <typename T, bool ONE_WARP, bool SHORT>
int launch_forward(const char* what, const T* logits, const ForwardCall& a, int warps, int log_parts, int32_t share) {
  int log_unit = 0;
  while (ceil_div(share, (int64_t)warps * 32 * LOGP_UNROLL << log_unit) > LOGP_UNITS) ++log_unit;
  const int parts = 1 << log_parts;
  cudaLaunchAttribute cluster;
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = (unsigned)parts;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3((unsigned)(ONE_WARP ? ceil_div(a.N, LOGP_ROWS) : a.N * parts));
  config.blockDim = dim3(32 * (ONE_WARP ? LOGP_ROWS : warps));
  config.stream = a.stream;
  config.attrs = &cluster;
  config.numAttrs = parts > 1 ? 1 : 0;
  config.dynamicSmemBytes = ONE_WARP ? LOGP_ROWS * room_bytes(1) : room_bytes(warps);
  LaunchScope scope(K_LOGPROBS_FWD, a.stream);
  return check_cuda(cudaLaunchKernelEx(&config, logprobs_forward<T, ONE_WARP, SHORT>, logits, a.row_stride, a.N, a.V, a.scale, a.targets, a.top_k, log_parts, share, log_unit, a.out), what);
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
    const T* x = static_cast<const T*>(logits);
    const ForwardCall a = {row_stride, N, (int32_t)V, scale, targets, top_k, out, s};
    const int64_t batches = ceil_div(V, RowBatches<T>::E) + 1;          // wherever rows start
    const int log_parts = log_parts_of(N, batches);
    const int32_t share = (int32_t)ceil_div(V / RowBatches<T>::E, 1 << log_parts);
    // Warps of a row: what a warp does for a row apart from its scores costs as much as a dozen batches a lane, so as few as keep the row short: us
    // with 1, 2, 4, 8 for 50,000 rows of 500 batches 172, 183, 265, 462; 25,000 of 1,000 148, 131, 144, 249; 6,250 of 4,000 153, 98, 95, 102; 2,048 of
    // 16,384 243, 125, 111, 101 (16: 111).  Where that leaves SMs idle more, while a thread has a few batches (300 rows of 1,250: 19.0, 11.8, 9.4, 8.6).
    int warps = share <= 700 ? 1 : share <= 3000 ? 2 : share <= 8000 ? 4 : 8;
    while (warps < LOGP_WARPS && (N << log_parts) * warps < 148 * 16 && share >= (warps < 8 ? 64 : 256) * warps) warps *= 2;
    if (warps == 1 && log_parts == 0)
      return share <= 32 * LOGP_UNROLL ? launch_forward<T, true, true>(what, x, a, 1, 0, share) : launch_forward<T, true, false>(what, x, a, 1, 0, share);
    return launch_forward<T, false, false>(what, x, a, warps, log_parts, share);
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
    const int64_t batches = ceil_div(V, RowBatches<T>::E) + 1;          // wherever rows start
    int threads = 32;
    while (threads < BACK_THREADS && batches > threads * BACK_UNROLL) threads *= 2;
    const int64_t pieces = ceil_div(batches, threads * BACK_UNROLL);
    if (N * pieces > INT32_MAX) return set_error(MTS_ERR_UNSUPPORTED, "%s: %lld rows of %lld", what, (long long)N, (long long)V);
    LaunchScope scope(K_LOGPROBS_BWD, s);
    logprobs_backward<T><<<(unsigned)(N * pieces), threads, 0, s>>>(static_cast<const T*>(logits), row_stride, (int32_t)V, scale, targets, stats, entropy,
                                                                    grad_logp, grad_entropy, static_cast<T*>(grad_logits), grad_stride, (int32_t)pieces);
    return check_launch(what);
  });
}
