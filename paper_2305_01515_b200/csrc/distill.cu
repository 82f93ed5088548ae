// Loss of a student's scores over V items against a teacher's best K of them, and its gradient.
//
//   q = softmax of scale teacher_k over the listed items (and exp(rest) for all others together),  p = softmax(scale x)
//   loss = sum_k q_k (log q_k - log p_{i_k}) + q_rest (log q_rest - log p_rest),   p_rest = what p gives to the items not listed
//   dx_v = weight scale (p_v - q_v) for a listed item, weight scale p_v (1 - q_rest / p_rest) for another
//
// The loss reads the scores once; with the gradient they are read again and it is written, all in one launch, so that the second reading comes from L2.  Sums and the
// teacher's distribution are fp32, the gradient is rounded to its type once.
#include "rows.cuh"

namespace mts {

constexpr int DISTILL_WARPS = 16;
constexpr int DISTILL_UNROLL = 8, DISTILL_GRAD_UNROLL = 4;     // batches on their way for a thread
constexpr int LISTED_BYTES = 24576;                            // of the bits that say which batches of a part hold a listed item

// Sums of 2^(c x - base) over a set of scores, each relative to the largest of its own: of all items (the listed ones empty), or of the items that are not listed and
// of those that are.  What one set has can be hundreds of powers of two below the other.
struct DistillSums { float m, sum, m_listed, listed; };

__device__ __forceinline__ float scaled_to(float sum, float from, float to, float c) { return from == -INFINITY ? sum : exp2_fast(change_of_base(from, to, c)) * sum; }
template <bool REST>
__device__ __forceinline__ DistillSums join_lanes(const DistillSums& s, float c) {
  DistillSums j = {warp_max(s.m), 0.f, -INFINITY, 0.f};
  j.sum = warp_sum(scaled_to(s.sum, s.m, j.m, c));
  if (REST) {
    j.m_listed = warp_max(s.m_listed);
    j.listed = warp_sum(scaled_to(s.listed, s.m_listed, j.m_listed, c));
  }
  return j;
}
// 2^(c x - base) of one score.
__device__ __forceinline__ float power(float x, float m, float base, float c) { return exp2_fast(ordinary(base) ? fmaf(x, c, -base) : (x - m) * c); }

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
  int32_t V, K, teacher_dtype, log_parts, share, warps, log_slots;      // warps: those that take part in the sums
  float scale;
};

struct DistillRoom {
  DistillSums of_warp[DISTILL_WARPS + 1], of_part[1 << MAX_LOG_PARTS];
  float total, q_rest, log_q_rest;
  uint32_t edges_listed;                                       // of the elements before and behind the whole batches, a bit for the lane that has it
};
// Behind it: float q[K], score[K], log_q[K], int32_t place[K], and with the rest's weight the table of the batches that hold a listed item (int32_t batch[],
// uint32_t places[], first[], of 1 << log_slots places, four times K at least), int32_t slot[K] and the bits of the batches that the pass leaves out.
__host__ __device__ constexpr int rounded16(int bytes) { return (bytes + 15) / 16 * 16; }

// Exponentials of a batch's scores.
template <bool ORDINARY, int E>
__device__ __forceinline__ void exponentials(float (&v)[E], float m, float base, float c) {
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

// A barrier of the whole block, met by the teacher's warp and the others at different places.
__device__ __forceinline__ void bits_ready() { asm volatile("bar.sync 1;" ::: "memory"); }

// A row (or a part of it, by a cluster of blocks) by a block.  The sums of the exponentials take one pass over the scores as in the log probabilities; the
// gradient reads them once more, from L2, where the row has just passed.  One warp gathers the teacher's row and the scores of the listed items (indices, then what
// they point to: two latencies in a row); where a row has four warps or more it is one of its own, while the others sum.
// With the rest's weight given (REST) the sum over the items that are not listed is made without the listed ones and relative to their own largest: what is left of a
// difference, or relative to the row's largest, would lose its digits where the listed ones have almost everything.  Bits in shared memory, eight to a thread's group, say which batches hold a listed item; the pass
// leaves these out, and they are added afterwards item by item.
// The gradient is written as if nothing were listed, and the listed places once more.
// us: 4,096 x 65,536 bf16, 50 items, with gradient 209-218 (4.9-5.1 TB/s of its floor's bytes; 5% more reads than the scores, issue slots 48% busy: a block's warps sum, wait for each other and
// write in turn); 2,047 x 32,003 fp16, 64 items and the rest, 75-77, loss alone 40; 20,000 x 5,001 fp32, 20 and the rest, 187; 64 x 20,000 fp32, loss alone, 6-8: latency.  Rows kept in shared
// memory between the passes took longer (fewer blocks an SM), and so did clusters for many rows.
template <typename T, bool REST>
__global__ void __maxnreg__(64)                                // of (DISTILL_WARPS + 1) * 32 threads at most: 32 warps an SM
distill_loss(const T* logits, T* grad, const DistillCall a) {
  constexpr int E = RowBatches<T>::E, LOG_E = E == 8 ? 3 : 2, U = DISTILL_UNROLL;
  __shared__ DistillRoom room;
  extern __shared__ __align__(16) uint8_t behind[];
  float* const q = reinterpret_cast<float*>(behind);
  float* const score = q + a.K;
  float* const log_q = score + a.K;
  int32_t* const place = reinterpret_cast<int32_t*>(log_q + a.K);
  const int slots = 1 << a.log_slots;
  int32_t* const in_slot = reinterpret_cast<int32_t*>(behind + rounded16(16 * a.K));
  uint32_t* const places_of = reinterpret_cast<uint32_t*>(in_slot + slots);
  uint32_t* const first_of = places_of + slots;
  int32_t* const slot_of_place = reinterpret_cast<int32_t*>(first_of + slots);
  uint8_t* const left_out = reinterpret_cast<uint8_t*>(slot_of_place + a.K);
  const int tid = threadIdx.x, lane = lane_id(), warp = tid / 32, everyone = blockDim.x, warps = a.warps, threads = 32 * warps;
  const bool own_warp = everyone > threads;                    // of the teacher's row
  const int parts = 1 << a.log_parts, part = blockIdx.x & (parts - 1);
  const int64_t n = blockIdx.x >> a.log_parts;
  if (parts > 1) cluster_arrive();                             // all blocks have begun before others write to them
  const RowBatches<T, false> r(logits + n * a.row_stride, a.V);
  const int32_t b0 = min(r.whole_end, r.whole_begin + part * a.share), b1 = min(r.whole_end, b0 + a.share);
  const float c = a.scale * LOG2E;

  // the student's sums of this thread
  float m = -INFINITY, base = 0.f, m_listed = -INFINITY, listed = 0.f;
  Pair others(0.f, 0.f);
  const auto rescale = [&](float most) {
    others = Pair(scaled_to(others.sum(), m, most, c), 0.f);
    m = most;
    base = base_of(m, c);
  };

  if (warp == (own_warp ? warps : 0)) {
    // the teacher's row.  `place`: an item's number of elements from the first batch's begin, so that its batch is place / E; -1: not used
    if (REST) {
      const int bytes = min(LISTED_BYTES, (b1 - b0 + threads * U - 1) / (threads * U) * threads);
      for (int i = lane; i < bytes / 4; i += 32) reinterpret_cast<uint32_t*>(left_out)[i] = 0;
      if (lane == 0) room.edges_listed = 0;
    }
    float edge = -INFINITY;
    if (lane < 2 * E) {
      const int32_t i = r.edge(lane);
      if (i >= 0 && (lane < E ? part == 0 : part == parts - 1)) edge = to_f32(r.row[i]);
    }
    __syncwarp();
    float most = -INFINITY;
    bool wrong = false;
    for (int k = lane; k < a.K; k += 32) {
      const int64_t i = a.index[n * a.K + k];
      const float t = i >= 0 ? teacher_value(a.teacher, a.teacher_dtype, n * a.K + k) : -INFINITY;
      wrong |= i >= a.V || isnan(t);
      log_q[k] = t;
      place[k] = i >= 0 && i < a.V ? (int32_t)i + r.shift : -1;
      most = fmaxf(most, t);
      if (REST && i >= 0 && i < a.V) {
        const int32_t b = (((int32_t)i + r.shift) >> LOG_E) - b0, group = b / (threads * U), in = b - group * threads * U;
        const int64_t byte = (int64_t)group * threads + in % threads;
        if (i < r.first(r.whole_begin)) atomicOr(&room.edges_listed, 1u << i);
        else if (i >= r.first(r.whole_end)) atomicOr(&room.edges_listed, 1u << (E + i - r.first(r.whole_end)));
        else if (b >= 0 && b < b1 - b0 && byte < LISTED_BYTES) atomicOr(reinterpret_cast<uint32_t*>(left_out) + byte / 4, 1u << (in / threads + byte % 4 * 8));
      }
    }
    if (REST) bits_ready();                                    // the others may look at the bits and places
    const float t_rest = REST ? a.rest[n] : -INFINITY;
    for (int k = lane; k < a.K; k += 32) {
      score[k] = place[k] >= 0 ? to_f32(r.row[place[k] - r.shift]) : 0.f;
      if (REST && place[k] >= 0) m_listed = fmaxf(m_listed, score[k]);
    }
    if (REST) m_listed = warp_max(m_listed);
    const float base_listed = base_of(m_listed, c);
    most = warp_max(most);
    // Exponents relative to the best listed one, whose product with the scale need not be a number of fp32 (nor lose digits); where the rest has more, relative to that.
    const float top = most == -INFINITY ? 0.f : most;
    float d_rest = REST ? fmaf(-top, a.scale, t_rest) : -INFINITY, shift = 0.f;
    if (REST && t_rest > -INFINITY && (d_rest > 0.f || most == -INFINITY)) {
      shift = d_rest;
      d_rest = t_rest - t_rest;                                // 0, or NaN where the rest is infinite
    }
    const float e_rest = expf(d_rest);
    float total = 0.f;
    for (int k = lane; k < a.K; k += 32) {
      log_q[k] = scaled_difference(log_q[k], top, a.scale) - shift;
      total += expf(log_q[k]);
    }
    total = warp_sum(total) + e_rest;
    if (__any_sync(0xFFFFFFFFu, wrong)) total = NAN;
    const bool any = total != 0.f;                             // else nothing is left of the teacher's row
    const float log_total = any ? logf(total) : 0.f;
    for (int k = lane; k < a.K; k += 32) {
      const float d = log_q[k];
      q[k] = any ? expf(d) / total : 0.f;
      log_q[k] = d - log_total;
    }
    if (lane == 0) {
      room.total = total;
      room.q_rest = any ? e_rest / total : 0.f;
      room.log_q_rest = d_rest - log_total;
    }
    if (edge != -INFINITY) {
      if (REST && room.edges_listed >> lane & 1) {
        listed += power(edge, m_listed, base_listed, c);
      } else {
        if (edge > m) rescale(edge);
        others = others + Pair(power(edge, m, base, c), 0.f);
      }
    }
    if (REST) {
      // the batches that are left out, each for its first place, item by item: a table has the places of a batch's listed items and their first
      for (int i = lane; i < slots / 4; i += 32) {
        reinterpret_cast<int4*>(in_slot)[i] = make_int4(-1, -1, -1, -1);
        reinterpret_cast<uint4*>(places_of)[i] = make_uint4(0u, 0u, 0u, 0u);
        reinterpret_cast<uint4*>(first_of)[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
      }
      __syncwarp();
      const auto slot_of = [&](int32_t b) {
        uint32_t slot = (uint32_t)b * 2654435761u >> (32 - a.log_slots);
        for (;; slot = (slot + 1) & (slots - 1)) {             // at most a quarter of the slots are taken: it ends
          const int32_t was = atomicCAS(&in_slot[slot], -1, b);
          if (was == -1 || was == b) return slot;
        }
      };
      for (int k = lane; k < a.K; k += 32) {
        const int32_t b = place[k] >> LOG_E;
        if (b < b0 || b >= b1) continue;                       // -1 too
        const uint32_t slot = slot_of(b);
        slot_of_place[k] = (int32_t)slot;
        atomicOr(&places_of[slot], 1u << (place[k] & (E - 1)));
        atomicMin(&first_of[slot], (uint32_t)k);
      }
      __syncwarp();
      for (int k = lane; k < a.K; k += 32) {
        const int32_t b = place[k] >> LOG_E;
        if (b < b0 || b >= b1) continue;
        const uint32_t slot = slot_of_place[k], places = places_of[slot];
        if (first_of[slot] != k) continue;
        float v[E], top = -INFINITY;
        RowBatches<T>::unpack(r.raw(b), v);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (places >> e & 1) {
            listed += power(v[e], m_listed, base_listed, c);
            v[e] = -INFINITY;
          }
          top = fmaxf(top, v[e]);
        }
        if (top > m) rescale(top);
        if (ordinary(base)) exponentials<true>(v, m, base, c);
        else exponentials<false>(v, m, base, c);
        others = others + sum_of<T>(v);
      }
    }
  }
  if (warp < warps) {
    const uint4 nothing_there = make_uint4(RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW, RowBatches<T>::LOW);
    // whether batch b holds a listed item, where the bits do not reach
    const auto holds_listed = [&](int32_t b) {
      for (int k = 0; k < a.K; ++k)
        if (place[k] >> LOG_E == b) return true;          // -1 >> LOG_E is -1
      return false;
    };
    uint4 w[U];
    const auto load = [&](int32_t g) {
      const int32_t b = g + tid;
      const T* p = r.row + r.first(b);
      if (b1 - (b - lane) > (U - 1) * threads + 31) {
#pragma unroll
        for (int u = 0; u < U; ++u, p += threads * E) w[u] = r.load16(p);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u, p += threads * E) {
          w[u] = nothing_there;
          if (b + u * threads < b1) w[u] = r.load16(p);
        }
      }
    };
    if (b0 < b1) load(b0);
    if (REST && (own_warp || warp != 0)) bits_ready();
    int32_t byte = tid;
    for (int32_t g = b0; g < b1; g += threads * U) {
      const int32_t b = g + tid;
      if (g > b0) load(g);
      unsigned out = 0;
      if (REST) {
        if (byte < LISTED_BYTES) {
          out = left_out[byte];
        } else {
          for (int u = 0; u < U; ++u) out |= holds_listed(b + u * threads) << u;
        }
        byte += threads;
        if (out) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (out >> u & 1) w[u] = nothing_there;
        }
      }
      uint32_t most_bits = max_bits<T>(w[0]);
#pragma unroll
      for (int u = 1; u < U; ++u) most_bits = max_bits<T>(most_bits, w[u]);
      const float most = max_value<T>(most_bits);
      if (most > m) rescale(most);
      if (!ordinary(base)) {
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
          if (b + u * threads >= b1 || out >> u & 1) continue;
          float v[E];
          RowBatches<T>::unpack(r.raw(b + u * threads), v);
          exponentials<false>(v, m, base, c);
          others = others + sum_of<T>(v);
        }
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u * threads >= b1 - (b - lane)) break;
          float v[E];
          RowBatches<T>::unpack(w[u], v);
          exponentials<true>(v, m, base, c);
          others = others + sum_of<T>(v);
        }
      }
    }
  }
  const auto some_of = [&](const DistillSums* sums, int count) {
    DistillSums mine = {-INFINITY, 0.f, -INFINITY, 0.f};
    if (lane < count) {
      mine.m = sums[lane].m;
      mine.sum = sums[lane].sum;
      if (REST) {
        mine.m_listed = sums[lane].m_listed;
        mine.listed = sums[lane].listed;
      }
    }
    return join_lanes<REST>(mine, c);
  };
  DistillSums s = join_lanes<REST>({m, others.sum(), m_listed, listed}, c);
  if (lane == 0) room.of_warp[warp] = s;
  __syncthreads();
  s = some_of(room.of_warp, everyone / 32);
  if (parts > 1) {
    cluster_wait();
    if (tid < parts) {
      const uint32_t to = in_block(&room.of_part[part], tid);
      asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\tst.shared::cluster.f32 [%0 + 8], %3;\n\tst.shared::cluster.f32 [%0 + 12], %4;"
                   :: "r"(to), "f"(s.m), "f"(s.sum), "f"(s.m_listed), "f"(s.listed) : "memory");
    }
    cluster_arrive();
    cluster_wait();                                            // (and no block writes over scores that another still reads)
    s = some_of(room.of_part, parts);
  }
  // of all items, and what of it the ones that are not listed have (all, where they are not told apart)
  m = REST ? fmaxf(s.m, s.m_listed) : s.m;
  base = base_of(m, c);
  if (REST && change_of_base(s.m, m, c) <= LEAST_EXP) s.sum *= 0.f;      // ruled out; NaN stays
  const float sum = REST ? scaled_to(s.sum, s.m, m, c) : s.sum, all = REST ? sum + scaled_to(s.listed, s.m_listed, m, c) : sum, m0 = m == -INFINITY ? 0.f : m;
  const float base_rest = REST ? base_of(s.m, c) : base, m0_rest = REST ? (s.m == -INFINITY ? 0.f : s.m) : m0;
  if (warp == 0 && part == 0 && a.loss) {
    const float log_all = all == 0.f ? 0.f : logf(all) - log_excess(m, base, c);
    float loss = 0.f;
    for (int k = lane; k < a.K; k += 32) {
      if (q[k] != 0.f) loss += q[k] * (log_q[k] - (scaled_difference(score[k], m0, a.scale) - log_all));
    }
    if (REST && lane == 0 && room.q_rest != 0.f) {
      const float log_p = logf(s.sum) - log_excess(s.m, base_rest, c) + (s.m == -INFINITY ? 0.f : scaled_difference(s.m, m0, a.scale)) - log_all;
      loss += room.q_rest * (room.log_q_rest - log_p);
    }
    loss = warp_sum(loss);
    if (lane == 0) a.loss[n] = loss;
  }
  if (!grad) return;

  const RowBatches<T> to(grad + n * a.grad_stride, a.V);
  const RowUnder<T> under(r.row, to);
  const int32_t g0 = part * a.share, g1 = part == parts - 1 ? to.count : g0 + a.share;
  const float w = (a.weights ? a.weights[n] : 1.f) * a.scale, inv_all = all == 0.f ? 0.f : 1.f / all, total = room.total;
  if (w == 0.f || total == 0.f) {
    const float zero[E] = {};
    for (int32_t b = g0 + tid; b < g1; b += everyone) to.store(b, zero);
    return;
  }
  // of an item that is not listed: p - q_rest p / p_rest = (p_rest - q_rest) 2^(c x - base_rest) / (their sum)
  const float f = (!REST ? w * inv_all : s.sum == 0.f ? 0.f : w * (sum * inv_all - room.q_rest) / s.sum) + total * 0.f;
  const bool usual = ordinary(base_rest);
  const auto gradient = [&](const uint4& x, float (&v)[E]) {
    RowBatches<T>::unpack(x, v);
    const Pair minus(-base_rest, -base_rest), c2(c, c), f2(f, f);
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 d = usual ? fma2(Pair(v[e], v[e + 1]), c2, minus).get() : make_float2((v[e] - m0_rest) * c, (v[e + 1] - m0_rest) * c);
      const float2 g = (Pair(exp2_fast(d.x), exp2_fast(d.y)) * f2).get();
      v[e] = g.x;
      v[e + 1] = g.y;
    }
  };
  constexpr int GU = DISTILL_GRAD_UNROLL;
  int32_t in0, in1;
  under.inner(&in0, &in1);
  in1 = min(in1, g1);
  for (int32_t g = g0; g < g1; g += everyone * GU) {
    const int32_t b = g + tid;
    float v[E];
    if (usual && g >= in0 && g + everyone * GU <= in1) {        // nothing to test
      const T* from = r.row + (to.first(b) - under.ahead);
      T* at = grad + n * a.grad_stride + to.first(b);
      uint4 x[GU];
#pragma unroll
      for (int u = 0; u < GU; ++u, from += everyone * E) x[u] = under.inside(from);
#pragma unroll
      for (int u = 0; u < GU; ++u, at += everyone * E) {
        RowBatches<T>::unpack(x[u], v);
        const Pair minus(-base_rest, -base_rest), c2(c, c), f2(f, f);
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
      for (int32_t q = b; q < min(g1, g + everyone * GU); q += everyone) {
        gradient(under.raw(q), v);
        to.store(q, v);
      }
    }
  }
  __syncthreads();
  // the listed items' places once more, by the block that wrote them
  for (int k = tid; k < a.K; k += everyone) {
    if (place[k] < 0) continue;
    const int32_t i = place[k] - r.shift, b = (i + to.shift) >> LOG_E;
    if (b < g0 || b >= g1) continue;
    float want = 0.f;
#pragma unroll 4
    for (int j = 0; j < a.K; ++j) want += place[j] == place[k] ? q[j] : 0.f;
    const float p = power(score[k], m0, base, c) * inv_all;
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
  config.blockDim = dim3(32 * (warps + (warps >= 4)));
  const int64_t bits = ceil_div(a.share, 32 * warps * DISTILL_UNROLL) * 32 * warps;
  config.dynamicSmemBytes = (size_t)rounded16(16 * a.K) + (REST ? (size_t)(12 << a.log_slots) + 4 * a.K + (size_t)(bits < LISTED_BYTES ? bits : LISTED_BYTES) : 0);
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
    const int32_t share = (int32_t)ceil_div(V / RowBatches<T>::E, 1 << log_parts);
    // Warps that sum a row, with its gradient, us with 1, 4, 8 and 16: 20,000 rows of 625 batches 107, 144, 244, 630; 10,000 of 1,250 105, 114, 139, 349; 5,000 of
    // 2,000 102, 73, 89, 191; 4,000 of 5,000 183, 144, 148, 261; 4,096 of 8,192 289, 246, 220, 316; 1,000 of 25,000 330, 257, 212, 181.  More where SMs idle.
    int warps = share <= 1500 ? 1 : share <= 6000 ? 4 : share <= 20000 ? 8 : 16;
    while (warps < DISTILL_WARPS && (N << log_parts) * warps < 148 * 16 && share >= (warps < 8 ? 64 : 256) * warps) warps *= 2;
    int log_slots = 5;
    while (1 << log_slots < 4 * K) ++log_slots;
    const DistillCall a = {row_stride, grad_stride, teacher_index, teacher_logits, teacher_rest, weights, loss, (int32_t)V, K, teacher_dtype, log_parts, share, warps, log_slots, scale};
    const T* x = static_cast<const T*>(logits);
    T* d = static_cast<T*>(grad_logits);
    return teacher_rest ? launch_distill<T, true>(what, x, d, a, N, warps, s) : launch_distill<T, false>(what, x, d, a, N, warps, s);
  });
}
