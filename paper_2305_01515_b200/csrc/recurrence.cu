// Gated linear recurrence over packed ragged sequences, forward and backward:
//
//   z_t = 1 / (1 + exp(-gate_t)),  h_t = z_t value_t + (1 - z_t) h_{t-1}
//
// Any run of tokens maps the state before it to B + P * state, P the product of its 1 - z and B the state it reaches from 0; a run
// that contains a sequence's start forgets what came before it (a cut).  Runs compose, so the token axis is cut into chunks
// whatever the sequences are: one long sequence and a thousand short ones are the same work.  Two passes, a warp per chunk and strip of
// channels (8 bytes of a row per lane) in each:
//   maps: the map of every chunk whose last sequence goes on behind it, from that sequence's start on (what lies before it in the
//         chunk is forgotten).  The last warp of a group of 16 chunks composes the group's map, the last of a span of 16 groups the
//         span's, the last of all walks the spans: nobody waits.
//   walk: the state before the chunk from at most a span's state, 15 groups and 15 chunks, then its tokens.
// The association of the maps depends on the offsets alone, so the result is the same in every run.  Both passes stream at the memory's
// rate, which bounds them: the inputs are read twice.  The second pass takes the chunks in the opposite order, so that what the first
// read last is still in the L2 cache.  (Tried before: one pass, whose blocks kept their tokens in shared memory and waited for the
// maps of the blocks before them.  A word published by one SM is seen by another 1 to 2 us later, and a chain of three such steps per tile
// outlasts what shared memory can hold back: 424 to 690 us for 524,287 tokens x 256, fp16.)
#include <type_traits>

#include "dense.cuh"

namespace mts {

constexpr int REC_WARPS = 4;
constexpr int REC_CHUNK = 64;                     // tokens of a chunk at most: a bit mask of them is one word
constexpr int REC_BATCH = 8;                      // tokens loaded together, and between two states kept for the backward
constexpr int REC_RADIX = 16;                     // chunks per group, groups per span
constexpr int REC_SPAN = REC_RADIX * REC_RADIX;
#ifndef MTS_REC_WARPS_WANTED
#define MTS_REC_WARPS_WANTED 2368
#endif
constexpr int REC_STATUS_OFFSETS = 1;

struct RecArgs {
  const void* gate; int64_t gate_stride;
  const void* value; int64_t value_stride;
  const int64_t* offsets;
  const float* h0;
  int64_t N, S;
  int32_t D;
  int32_t chunk;               // tokens of a chunk
  int32_t chunks, strips, groups, spans;
  uint32_t* status;
  uint32_t* group_count;       // [groups, strips] chunks done, likewise groups of a span, spans
  uint32_t* span_count;
  uint32_t* total_count;
  int32_t* sequence;           // [chunks] a sequence at or before the chunk's first token
  float* chunk_P;              // [chunks, D]
  float* chunk_B;
  float* chunk_start;          // [chunks, D] state in which the chunk's last sequence starts
  float* group_P;
  float* group_B;
  float* span_P;
  float* span_B;
  float* span_state;           // [spans, D] the state before the span
};

// ------------------------------------------------------------------------------- V channels of a lane
// fp32 values in pairs, which sm_100 multiplies and adds two at a time.
template <int V>
struct Channels {
  static_assert(V % 2 == 0, "pairs");
  unsigned long long p[V / 2];
};
template <>
struct Channels<1> { float p[1]; };

__device__ __forceinline__ unsigned long long pair(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(unsigned long long v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }

template <int V>
__device__ __forceinline__ Channels<V> gathered(const float (&x)[V]) {
  Channels<V> r;
  if constexpr (V == 1) r.p[0] = x[0];
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) r.p[k] = pair(x[2 * k], x[2 * k + 1]);
  }
  return r;
}
template <int V>
__device__ __forceinline__ void scattered(Channels<V> v, float (&x)[V]) {
  if constexpr (V == 1) x[0] = v.p[0];
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) split(v.p[k], x[2 * k], x[2 * k + 1]);
  }
}
template <int V>
__device__ __forceinline__ Channels<V> all(float x) {
  Channels<V> r;
  if constexpr (V == 1) r.p[0] = x;
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) r.p[k] = pair(x, x);
  }
  return r;
}
template <int V>
__device__ __forceinline__ Channels<V> fma(Channels<V> a, Channels<V> b, Channels<V> c) {
  Channels<V> r;
  if constexpr (V == 1) r.p[0] = fmaf(a.p[0], b.p[0], c.p[0]);
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.p[k]) : "l"(a.p[k]), "l"(b.p[k]), "l"(c.p[k]));
  }
  return r;
}
template <int V>
__device__ __forceinline__ Channels<V> operator*(Channels<V> a, Channels<V> b) {
  Channels<V> r;
  if constexpr (V == 1) r.p[0] = a.p[0] * b.p[0];
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.p[k]) : "l"(a.p[k]), "l"(b.p[k]));
  }
  return r;
}
template <int V>
__device__ __forceinline__ Channels<V> operator+(Channels<V> a, Channels<V> b) {
  Channels<V> r;
  if constexpr (V == 1) r.p[0] = a.p[0] + b.p[0];
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.p[k]) : "l"(a.p[k]), "l"(b.p[k]));
  }
  return r;
}
template <int V, typename Fn>
__device__ __forceinline__ Channels<V> each(Channels<V> a, Fn&& fn) {
  if constexpr (V == 1) a.p[0] = fn(a.p[0]);
  else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      float x, y;
      split(a.p[k], x, y);
      a.p[k] = pair(fn(x), fn(y));
    }
  }
  return a;
}

// -z for gate logits g, through the hardware's 2^x and reciprocal, a few units of 2^-23 each, the gate's size times as much for
// large ones.  Denormals are flushed: a z below 2^-126.  Exactly -1 and -0 for gates of both infinities.
template <int V>
__device__ __forceinline__ Channels<V> minus_sigmoid(Channels<V> g) {
  const Channels<V> e = each(g * all<V>(-1.4426950408889634f), [](float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
  });
  return each(fma(e, all<V>(-1.f), all<V>(-1.f)), [](float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
  });
}
// z x + (1 - z) h for nz = -z and nx = -x, without rounding 1 - z: x itself for z = 1, h for z = 0.
template <int V>
__device__ __forceinline__ Channels<V> blend(Channels<V> nz, Channels<V> nx, Channels<V> h) { return fma(nz, nx, fma(nz, h, h)); }

// V consecutive elements as they lie in memory, in 32-bit words.
template <typename T, int V>
struct Raw { uint32_t w[(V * sizeof(T) + 3) / 4]; };

template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load_raw(const T* p) {
  Raw<T, V> r;
  constexpr int BYTES = V * sizeof(T);
  if constexpr (BYTES == 16) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
  } else if constexpr (BYTES == 8) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    r.w[0] = u.x; r.w[1] = u.y;
  } else if constexpr (BYTES == 4) {
    r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    r.w[0] = *reinterpret_cast<const uint16_t*>(p);
  }
  return r;
}
// NEGATE: minus the values (their sign bits flipped while still packed).
template <typename T, int V, bool NEGATE = false>
__device__ __forceinline__ Channels<V> unpack(Raw<T, V> r) {
  Channels<V> v;
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) v.p[0] = __uint_as_float(r.w[0] ^ (NEGATE ? 0x80000000u : 0u));
    else v.p[0] = unpack2<T>(r.w[0] ^ (NEGATE ? 0x8000u : 0u)).x;
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < V / 2; ++k)
      v.p[k] = pair(__uint_as_float(r.w[2 * k] ^ (NEGATE ? 0x80000000u : 0u)), __uint_as_float(r.w[2 * k + 1] ^ (NEGATE ? 0x80000000u : 0u)));
  } else {
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      const float2 f = unpack2<T>(r.w[k] ^ (NEGATE ? 0x80008000u : 0u));
      v.p[k] = pair(f.x, f.y);
    }
  }
  return v;
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, Channels<V> v) {
  if constexpr (V == 1) {
    *p = from_f32<T>(v.p[0]);
  } else {
    float x[V];
#pragma unroll
    for (int k = 0; k < V / 2; ++k) split(v.p[k], x[2 * k], x[2 * k + 1]);
    if constexpr (sizeof(T) == 4 && V == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
    else if constexpr (V == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]));
    else *reinterpret_cast<uint32_t*>(p) = pack2<T>(x[0], x[1]);
  }
}
template <int V>
__device__ __forceinline__ Channels<V> load_f32(const float* p) { return unpack<float, V>(load_raw<float, V>(p)); }
// The same in rows of D channels of which `left` begin at p: VEC = D and the row's base allow whole vectors, else one by one.
template <int V, bool VEC>
__device__ __forceinline__ Channels<V> get(const float* p, int left) {
  if (VEC) return left > 0 ? load_f32<V>(p) : all<V>(0.f);
  float x[V];
#pragma unroll
  for (int k = 0; k < V; ++k) x[k] = k < left ? p[k] : 0.f;
  return gathered<V>(x);
}
template <int V, bool VEC, typename T>
__device__ __forceinline__ void put(T* p, int left, Channels<V> v) {
  if (VEC) {
    if (left > 0) store(p, v);
  } else {
    float x[V];
    scattered(v, x);
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k < left) p[k] = from_f32<T>(x[k]);
  }
}
// The V channels of a row of which `left` begin at p (none: 0), as they lie in memory.
template <typename T, int V, bool VEC>
__device__ __forceinline__ Raw<T, V> get_raw(const T* p, int left) {
  Raw<T, V> r = {};
  if (VEC) {
    if (left > 0) r = load_raw<T, V>(p);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < V; ++k) r.w[k] = k < left ? __float_as_uint(p[k]) : 0u;
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k < left) r.w[k / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[k] << (16 * (k % 2));
  }
  return r;
}
// What another warp of the same launch has written: from L2, the L1 cache may hold what was there before.
template <int V, bool VEC>
__device__ __forceinline__ Channels<V> load_published(const float* p, int left) {
  float x[V];
  if constexpr (VEC && V == 4) {
    const float4 f = left > 0 ? __ldcg(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
    x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
  } else if constexpr (VEC && V == 2) {
    const float2 f = left > 0 ? __ldcg(reinterpret_cast<const float2*>(p)) : make_float2(0.f, 0.f);
    x[0] = f.x; x[1] = f.y;
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = k < left ? __ldcg(p + k) : 0.f;
  }
  return gathered<V>(x);
}

// ------------------------------------------------------------------------------- maps
// state -> B + P * state.  P >= 0 is a product of 1 - z; P = -0 marks a cut, whose result is B even where the state before it is
// infinite or NaN.
template <int V>
struct Map { Channels<V> P, B; };
constexpr float CUT = -0.f;

// first, then second; `first` may be a state (P = CUT).
template <int V>
__device__ __forceinline__ Map<V> then(Map<V> first, Map<V> second) {
  float P1[V], B1[V], P2[V], B2[V];
  scattered(first.P, P1);
  scattered(first.B, B1);
  scattered(second.P, P2);
  scattered(second.B, B2);
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const bool cut = __float_as_int(P2[k]) == (int)0x80000000;
    B1[k] = cut ? B2[k] : fmaf(P2[k], B1[k], B2[k]);
    P1[k] = cut || __float_as_int(P1[k]) == (int)0x80000000 ? CUT : P1[k] * P2[k];
  }
  return Map<V>{gathered<V>(P1), gathered<V>(B1)};
}

// Composition of n maps from row `lo` of [rows, D] arrays on, after `m`.
template <int V, bool VEC>
__device__ __forceinline__ Map<V> compose(const RecArgs& a, const float* P, const float* B, int lo, int n, int c, Map<V> m) {
  const int left = a.D - c;
  P += (int64_t)lo * a.D + c;
  B += (int64_t)lo * a.D + c;
#pragma unroll 4
  for (int k = 0; k < n; ++k, P += a.D, B += a.D) m = then(m, Map<V>{load_published<V, VEC>(P, left), load_published<V, VEC>(B, left)});
  return m;
}

// Whether this warp is the last of `members` to get here; if so, what the others wrote before is visible to it.
__device__ __forceinline__ bool last_of(uint32_t* count, int members) {
  uint32_t before = 0;
  __syncwarp();
  if (lane_id() == 0) {
    __threadfence();
    before = atomicAdd(count, 1u);
  }
  const bool last = __shfl_sync(0xFFFFFFFFu, before, 0) == (uint32_t)members - 1;
  if (last) __threadfence();
  return last;
}

// After a chunk's map (counted in the order of the walk) has been written: the maps of the group and span that it completes, and after the
// last of all the state before every span.
template <int V, bool VEC>
__device__ __forceinline__ void complete(const RecArgs& a, int index, int strip, int c) {
  if (a.groups == 1) return;                                            // the walk composes the chunks' maps itself
  const Map<V> identity = {all<V>(1.f), all<V>(0.f)};
  const int left = a.D - c, group = index / REC_RADIX, span = index / REC_SPAN;
  if (!last_of(a.group_count + (int64_t)group * a.strips + strip, min(REC_RADIX, a.chunks - group * REC_RADIX))) return;
  Map<V> m = compose<V, VEC>(a, a.chunk_P, a.chunk_B, group * REC_RADIX, min(REC_RADIX, a.chunks - group * REC_RADIX), c, identity);
  put<V, VEC>(a.group_P + (int64_t)group * a.D + c, left, m.P);
  put<V, VEC>(a.group_B + (int64_t)group * a.D + c, left, m.B);
  if (a.spans == 1) return;
  if (!last_of(a.span_count + (int64_t)span * a.strips + strip, min(REC_RADIX, a.groups - span * REC_RADIX))) return;
  m = compose<V, VEC>(a, a.group_P, a.group_B, span * REC_RADIX, min(REC_RADIX, a.groups - span * REC_RADIX), c, identity);
  put<V, VEC>(a.span_P + (int64_t)span * a.D + c, left, m.P);
  put<V, VEC>(a.span_B + (int64_t)span * a.D + c, left, m.B);
  if (!last_of(a.total_count + strip, a.spans)) return;
  m = {all<V>(CUT), all<V>(0.f)};
#pragma unroll 4
  for (int k = 0; k < a.spans; ++k) {
    put<V, VEC>(a.span_state + (int64_t)k * a.D + c, left, m.B);
    m = compose<V, VEC>(a, a.span_P, a.span_B, k, 1, c, m);
  }
}

// The state before tile `index`, whose first sequence (in the order of the walk) began in tile `from` < index.
template <int V, bool VEC>
__device__ __forceinline__ Channels<V> state_before(const RecArgs& a, int index, int from, int c) {
  from = max(0, min(from, index - 1));
  const int group = index / REC_RADIX, span = index / REC_SPAN, lo = max(from, group * REC_RADIX);
  Map<V> m = {all<V>(CUT), all<V>(0.f)};
  if (from < group * REC_RADIX) {
    if (from < span * REC_SPAN) m.B = load_published<V, VEC>(a.span_state + (int64_t)span * a.D + c, a.D - c);
    const int glo = max(from / REC_RADIX, span * REC_RADIX);
    m = compose<V, VEC>(a, a.group_P, a.group_B, glo, group - glo, c, m);
  }
  return compose<V, VEC>(a, a.chunk_P, a.chunk_B, lo, index - lo, c, m).B;
}

// ------------------------------------------------------------------------------- sequences of a chunk
struct ChunkSequences {
  unsigned long long first, last;      // tokens that begin / end their sequence
  int64_t head_begin;                  // of the sequence that holds the chunk's first token
  int64_t tail_end;                    // of the one that holds its last token
};

// One warp: the sequence of the chunk's first token, by a search with 32 probes a step.  Every index is bounded whatever the offsets hold.
__device__ __forceinline__ int find_sequence(const RecArgs& a, int64_t t0) {
  int64_t lo = 0, hi = a.S;
  while (hi - lo > 1) {                                               // offsets[lo] <= t0 < offsets[hi]
    const int64_t step = (hi - lo + 31) / 32, i = lo + lane_id() * step;
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, i < hi && a.offsets[i] <= t0));
    lo += (int64_t)max(n - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  return (int)lo;
}
// The sequences of a chunk from sequence `lo` on; their numbers go to first_of / last_of, by token.
__device__ __forceinline__ ChunkSequences find_borders(const RecArgs& a, int lo, int64_t t0, int64_t t1, int32_t* first_of, int32_t* last_of) {
  ChunkSequences q = {0, 0, t0, t1};
  for (int64_t base = lo; base < a.S; base += 32) {
    const int64_t s = base + lane_id();
    const int64_t b = s < a.S ? a.offsets[s] : a.N, e = s < a.S ? a.offsets[s + 1] : a.N;
    const bool some = e > b;
    if (some && b >= t0 && b < t1) { q.first |= 1ull << (b - t0); first_of[b - t0] = (int)s; }
    if (some && e > t0 && e <= t1) { q.last |= 1ull << (e - 1 - t0); last_of[e - 1 - t0] = (int)s; }
    const unsigned head = __ballot_sync(0xFFFFFFFFu, some && b <= t0 && e > t0), tail = __ballot_sync(0xFFFFFFFFu, some && b < t1 && e >= t1);
    if (head) q.head_begin = __shfl_sync(0xFFFFFFFFu, b, __ffs(head) - 1);
    if (tail) q.tail_end = __shfl_sync(0xFFFFFFFFu, e, __ffs(tail) - 1);
    if (__any_sync(0xFFFFFFFFu, b >= t1)) break;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    q.first |= __shfl_xor_sync(0xFFFFFFFFu, q.first, o);
    q.last |= __shfl_xor_sync(0xFFFFFFFFu, q.last, o);
  }
  q.head_begin = max(q.head_begin, (int64_t)0);
  q.tail_end = min(q.tail_end, a.N);
  __syncwarp();
  return q;
}

// Offsets in order, from 0 to N (each warp a share of them); `row(s)` for every empty sequence.
template <typename Fn>
__device__ __forceinline__ void check_offsets(const RecArgs& a, Fn&& row) {
  const int64_t warps = (int64_t)gridDim.x * REC_WARPS;
  bool bad = false;
  for (int64_t s0 = ((int64_t)blockIdx.x * REC_WARPS + threadIdx.x / 32) * 32; s0 < a.S; s0 += warps * 32) {
    const int64_t s = s0 + lane_id();
    const int64_t b = s < a.S ? a.offsets[s] : 0, e = s < a.S ? a.offsets[s + 1] : 1;
    if (s < a.S) bad |= b < 0 || e < b || (s == 0 && b != 0) || (s == a.S - 1 && e != a.N);
    unsigned empty = __ballot_sync(0xFFFFFFFFu, s < a.S && e <= b);
    while (empty) {
      row(s0 + __ffs(empty) - 1);
      empty &= empty - 1;
    }
  }
  if (bad) atomicOr(a.status, (uint32_t)REC_STATUS_OFFSETS);
}

// What a warp works on: chunk (counted from the end where BACKWARD) and strip of channels.
struct Item {
  int index, chunk, strip;
  int64_t t0, t1;
  __device__ __forceinline__ Item(const RecArgs& a, int64_t item, bool backward) {
    index = (int)(item / a.strips);
    strip = (int)(item - (int64_t)index * a.strips);
    chunk = backward ? a.chunks - 1 - index : index;
    t0 = (int64_t)chunk * a.chunk;
    t1 = min(t0 + a.chunk, a.N);
  }
};

// The rows of a batch of tokens, from row p on; rows that `live` does not name are not read and give 0.
template <typename T, int V, bool VEC>
__device__ __forceinline__ void load_rows(const T* p, int64_t stride, uint32_t live, int left, Raw<T, V> (&r)[REC_BATCH]) {
#pragma unroll
  for (int i = 0; i < REC_BATCH; ++i, p += stride) r[i] = (live >> i & 1) ? get_raw<T, V, VEC>(p, left) : Raw<T, V>{};
}
template <typename T, int V, bool VEC>
__device__ __forceinline__ void load_rows(const T* p, int64_t stride, int left, Raw<T, V> (&r)[REC_BATCH]) {
#pragma unroll
  for (int i = 0; i < REC_BATCH; ++i, p += stride) r[i] = get_raw<T, V, VEC>(p, left);
}

__device__ __forceinline__ uint32_t batch_bits(unsigned long long mask, int64_t rel) { return (uint32_t)(mask >> rel) & ((1u << REC_BATCH) - 1); }
constexpr uint32_t ALL_LIVE = (1u << REC_BATCH) - 1;

// ------------------------------------------------------------------------------- forward
template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(REC_WARPS * 32)
recurrence_forward_maps(const RecArgs a) {
  __shared__ int32_t borders[REC_WARPS][2][REC_CHUNK];
  int32_t* first_of = borders[threadIdx.x / 32][0];
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
  const int64_t item = (int64_t)blockIdx.x * REC_WARPS + threadIdx.x / 32;
  if (item >= (int64_t)a.chunks * a.strips) return;
  const Item it(a, item, false);
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c;
  const int lo = find_sequence(a, it.t0);
  if (it.strip == 0 && lane_id() == 0) a.sequence[it.chunk] = lo;
  const ChunkSequences q = find_borders(a, lo, it.t0, it.t1, first_of, borders[threadIdx.x / 32][1]);
  Map<V> m = {all<V>(CUT), all<V>(0.f)};
  if (q.tail_end > it.t1) {                                             // a whole chunk: the sequence goes on
    int start = 0;
    if (q.first) {
      start = 63 - __clzll(q.first);
      if (a.h0) m.B = get<V, VEC>(a.h0 + (int64_t)first_of[start] * a.D + c, left);
      put<V, VEC>(a.chunk_start + (int64_t)it.chunk * a.D + c, left, m.B);
    } else {
      m.P = all<V>(1.f);
    }
    Raw<T, V> g[REC_BATCH], x[REC_BATCH];
#pragma unroll 1
    for (int rel = start & ~(REC_BATCH - 1); rel < a.chunk; rel += REC_BATCH) {
      load_rows<T, V, VEC>(static_cast<const T*>(a.gate) + (it.t0 + rel) * a.gate_stride + c, a.gate_stride, left, g);
      load_rows<T, V, VEC>(static_cast<const T*>(a.value) + (it.t0 + rel) * a.value_stride + c, a.value_stride, left, x);
      const Channels<V> before = m.B;
#pragma unroll
      for (int i = 0; i < REC_BATCH; ++i) {
        const Channels<V> nz = minus_sigmoid(unpack<T, V>(g[i]));
        if (rel + i == start) m.B = before;
        m.B = blend(nz, unpack<T, V, true>(x[i]), m.B);
        m.P = fma(nz, m.P, m.P);
      }
    }
    if (q.first) m.P = all<V>(CUT);
  }
  put<V, VEC>(a.chunk_P + (int64_t)it.chunk * a.D + c, left, m.P);
  put<V, VEC>(a.chunk_B + (int64_t)it.chunk * a.D + c, left, m.B);
  complete<V, VEC>(a, it.index, it.strip, c);
}

template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(REC_WARPS * 32)
recurrence_forward_walk(const RecArgs a, T* __restrict__ out, int64_t out_stride, float* h_final, float* __restrict__ entry) {
  __shared__ int32_t borders[REC_WARPS][2][REC_CHUNK];
  int32_t* first_of = borders[threadIdx.x / 32][0];
  int32_t* last_of = borders[threadIdx.x / 32][1];
  if (h_final) {
    check_offsets(a, [&](int64_t s) {
      for (int d = lane_id(); d < a.D; d += 32) h_final[s * a.D + d] = a.h0 ? a.h0[s * a.D + d] : 0.f;
    });
  } else {
    check_offsets(a, [](int64_t) {});
  }
  const int64_t item = (int64_t)(gridDim.x - 1 - blockIdx.x) * REC_WARPS + threadIdx.x / 32;     // from the end: see above
  if (item >= (int64_t)a.chunks * a.strips) return;
  const Item it(a, item, false);
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c;
  const ChunkSequences q = find_borders(a, a.sequence[it.chunk], it.t0, it.t1, first_of, last_of);
  // the start of a sequence that goes on behind the chunk was kept by the first pass: h_final may be the same array as h0, and the
  // warp that writes it does not wait for this one
  const int kept = q.first && q.tail_end > it.t1 ? 63 - __clzll(q.first) : -1;
  Channels<V> h = all<V>(0.f);
  if (!(q.first & 1)) h = state_before<V, VEC>(a, it.index, (int)(q.head_begin / a.chunk), c);
  const T* gate = static_cast<const T*>(a.gate) + it.t0 * a.gate_stride + c;
  const T* value = static_cast<const T*>(a.value) + it.t0 * a.value_stride + c;
  T* to = out + it.t0 * out_stride + c;
  const int tokens = (int)(it.t1 - it.t0);
#pragma unroll 1
  for (int rel = 0; rel < tokens; rel += REC_BATCH, gate += REC_BATCH * a.gate_stride, value += REC_BATCH * a.value_stride, to += REC_BATCH * out_stride) {
    const uint32_t live = tokens - rel >= REC_BATCH ? ALL_LIVE : (1u << (tokens - rel)) - 1;
    const uint32_t firsts = batch_bits(q.first, rel), lasts = batch_bits(q.last, rel);
    if (entry) put<V, VEC>(entry + ((it.t0 + rel) / REC_BATCH) * a.D + c, left, h);
    Raw<T, V> g[REC_BATCH], x[REC_BATCH];
    if (live == ALL_LIVE && !(firsts | lasts)) {
      load_rows<T, V, VEC>(gate, a.gate_stride, left, g);
      load_rows<T, V, VEC>(value, a.value_stride, left, x);
      T* row = to;
#pragma unroll
      for (int i = 0; i < REC_BATCH; ++i, row += out_stride) {
        h = blend(minus_sigmoid(unpack<T, V>(g[i])), unpack<T, V, true>(x[i]), h);
        put<V, VEC>(row, left, h);
      }
    } else {
      load_rows<T, V, VEC>(gate, a.gate_stride, live, left, g);
      load_rows<T, V, VEC>(value, a.value_stride, live, left, x);
      T* row = to;
#pragma unroll
      for (int i0 = 0; i0 < REC_BATCH; i0 += 4) {
        Channels<V> s[4];
#pragma unroll
        for (int i = i0; i < i0 + 4; ++i) {
          s[i - i0] = all<V>(0.f);
          if (firsts >> i & 1) {
            if (rel + i == kept) s[i - i0] = load_published<V, VEC>(a.chunk_start + (int64_t)it.chunk * a.D + c, left);
            else if (a.h0) s[i - i0] = get<V, VEC>(a.h0 + (int64_t)first_of[rel + i] * a.D + c, left);
          }
        }
#pragma unroll
        for (int i = i0; i < i0 + 4; ++i, row += out_stride) {
          if (live >> i & 1) {
            if (firsts >> i & 1) h = s[i - i0];
            h = blend(minus_sigmoid(unpack<T, V>(g[i])), unpack<T, V, true>(x[i]), h);
            put<V, VEC>(row, left, h);
            if ((lasts >> i & 1) && h_final) put<V, VEC>(h_final + (int64_t)last_of[rel + i] * a.D + c, left, h);
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------- backward
// What a token hands to the one before it, c_t = (1 - z_t) G_t = (1 - z_t) (grad_out_t + c_{t+1}), is the same kind of map, walked from
// the last chunk to the first; its cut is a sequence's last token, which starts from grad_final.
template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(REC_WARPS * 32)
recurrence_backward_maps(const RecArgs a, const T* __restrict__ grad_out, int64_t grad_out_stride, const float* __restrict__ grad_final) {
  __shared__ int32_t borders[REC_WARPS][2][REC_CHUNK];
  int32_t* last_of = borders[threadIdx.x / 32][1];
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
  const int64_t item = (int64_t)blockIdx.x * REC_WARPS + threadIdx.x / 32;
  if (item >= (int64_t)a.chunks * a.strips) return;
  const Item it(a, item, true);
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c;
  const int lo = find_sequence(a, it.t0);
  if (it.strip == 0 && lane_id() == 0) a.sequence[it.chunk] = lo;
  const ChunkSequences q = find_borders(a, lo, it.t0, it.t1, borders[threadIdx.x / 32][0], last_of);
  Map<V> m = {all<V>(CUT), all<V>(0.f)};
  if (q.head_begin < it.t0) {
    int end = (int)(it.t1 - it.t0) - 1;
    if (q.last) {
      end = __ffsll(q.last) - 1;
      if (grad_final) m.B = get<V, VEC>(grad_final + (int64_t)last_of[end] * a.D + c, left);
    } else {
      m.P = all<V>(1.f);
    }
    Raw<T, V> g[REC_BATCH], d[REC_BATCH];
#pragma unroll 1
    for (int rel = end & ~(REC_BATCH - 1); rel >= 0; rel -= REC_BATCH) {
      const uint32_t live = end - rel >= REC_BATCH - 1 ? ALL_LIVE : (1u << (end - rel + 1)) - 1;
      load_rows<T, V, VEC>(static_cast<const T*>(a.gate) + (it.t0 + rel) * a.gate_stride + c, a.gate_stride, live, left, g);
      load_rows<T, V, VEC>(grad_out + (it.t0 + rel) * grad_out_stride + c, grad_out_stride, live, left, d);
#pragma unroll
      for (int i = REC_BATCH - 1; i >= 0; --i) {
        if (live >> i & 1) {
          const Channels<V> nz = minus_sigmoid(unpack<T, V>(g[i])), G = unpack<T, V>(d[i]) + m.B;
          m.B = fma(nz, G, G);
          m.P = fma(nz, m.P, m.P);
        }
      }
    }
    if (q.last) m.P = all<V>(CUT);
  }
  put<V, VEC>(a.chunk_P + (int64_t)it.index * a.D + c, left, m.P);
  put<V, VEC>(a.chunk_B + (int64_t)it.index * a.D + c, left, m.B);
  complete<V, VEC>(a, it.index, it.strip, c);
}

// A batch is walked forward from the state that the forward left before it, for -z and the distance from value to state, then backward.
template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(REC_WARPS * 32)
recurrence_backward_walk(const RecArgs a, const float* __restrict__ entry, const T* __restrict__ grad_out, int64_t grad_out_stride,
                         const float* __restrict__ grad_final, T* __restrict__ grad_gate, int64_t grad_gate_stride,
                         T* __restrict__ grad_value, int64_t grad_value_stride, float* __restrict__ grad_h0) {
  __shared__ int32_t borders[REC_WARPS][2][REC_CHUNK];
  int32_t* first_of = borders[threadIdx.x / 32][0];
  int32_t* last_of = borders[threadIdx.x / 32][1];
  if (grad_h0) {
    check_offsets(a, [&](int64_t s) {
      for (int d = lane_id(); d < a.D; d += 32) grad_h0[s * a.D + d] = grad_final ? grad_final[s * a.D + d] : 0.f;
    });
  } else {
    check_offsets(a, [](int64_t) {});
  }
  const int64_t item = (int64_t)(gridDim.x - 1 - blockIdx.x) * REC_WARPS + threadIdx.x / 32;
  if (item >= (int64_t)a.chunks * a.strips) return;
  const Item it(a, item, true);
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c, tokens = (int)(it.t1 - it.t0);
  const ChunkSequences q = find_borders(a, a.sequence[it.chunk], it.t0, it.t1, first_of, last_of);
  Channels<V> carry = all<V>(0.f);
  if (!(q.last >> (tokens - 1) & 1))
    carry = state_before<V, VEC>(a, it.index, a.chunks - 1 - (int)min((q.tail_end - 1) / a.chunk, (int64_t)a.chunks - 1), c);
#pragma unroll 1
  for (int rel = (tokens - 1) & ~(REC_BATCH - 1); rel >= 0; rel -= REC_BATCH) {
    const int64_t t = it.t0 + rel;
    const uint32_t live = tokens - rel >= REC_BATCH ? ALL_LIVE : (1u << (tokens - rel)) - 1;
    const uint32_t firsts = batch_bits(q.first, rel), lasts = batch_bits(q.last, rel);
    Raw<T, V> g[REC_BATCH], x[REC_BATCH], d[REC_BATCH];
    load_rows<T, V, VEC>(static_cast<const T*>(a.gate) + t * a.gate_stride + c, a.gate_stride, live, left, g);
    load_rows<T, V, VEC>(static_cast<const T*>(a.value) + t * a.value_stride + c, a.value_stride, live, left, x);
    load_rows<T, V, VEC>(grad_out + t * grad_out_stride + c, grad_out_stride, live, left, d);
    Channels<V> h = all<V>(0.f);
    if (!(firsts & 1)) h = get<V, VEC>(entry + t / REC_BATCH * a.D + c, left);
    Channels<V> nz[REC_BATCH], away[REC_BATCH];                         // away: - (value - state before the token)
#pragma unroll
    for (int i = 0; i < REC_BATCH; ++i) {
      if (firsts >> i & 1) h = a.h0 ? get<V, VEC>(a.h0 + (int64_t)first_of[rel + i] * a.D + c, left) : all<V>(0.f);
      const Channels<V> nx = unpack<T, V, true>(x[i]);
      nz[i] = minus_sigmoid(unpack<T, V>(g[i]));
      away[i] = nx + h;
      h = blend(nz[i], nx, h);
    }
    T* to_gate = grad_gate + t * grad_gate_stride + c;
    T* to_value = grad_value + t * grad_value_stride + c;
#pragma unroll
    for (int i = REC_BATCH - 1; i >= 0; --i) {
      if (live >> i & 1) {
        if (lasts >> i & 1) carry = grad_final ? get<V, VEC>(grad_final + (int64_t)last_of[rel + i] * a.D + c, left) : all<V>(0.f);
        const Channels<V> G = unpack<T, V>(d[i]) + carry, nG = nz[i] * G;          // -z G
        carry = fma(nz[i], G, G);
        put<V, VEC>(to_value + i * grad_value_stride, left, nG * all<V>(-1.f));
        put<V, VEC>(to_gate + i * grad_gate_stride, left, nG * fma(nz[i], away[i], away[i]));
        if ((firsts >> i & 1) && grad_h0) put<V, VEC>(grad_h0 + (int64_t)first_of[rel + i] * a.D + c, left, carry);
      }
    }
  }
}

}  // namespace mts

using namespace mts;

namespace {

int check_sizes(const char* what, int64_t N, int64_t S, int32_t D, int32_t dtype) {
  if (N < 0 || S < 0 || D < 1 || !known_dtype(dtype))
    return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, S %lld, D %d, dtype %d", what, (long long)N, (long long)S, D, dtype);
  if (N >= (1ll << 31) - (1 << 16) || S >= (1ll << 31) - (1 << 16) || D > (1 << 20) ||
      ceil_div(N, REC_BATCH) * ceil_div(D, 32) >= (1ll << 31))
    return set_error(MTS_ERR_UNSUPPORTED, "%s: N %lld, S %lld, D %d", what, (long long)N, (long long)S, D);
  if (S == 0 && N > 0) return set_error(MTS_ERR_INVALID_ARG, "%s: %lld tokens in no sequence", what, (long long)N);
  return MTS_OK;
}

int check_workspace(const char* what, const void* workspace, size_t have, size_t need) {
  if (!workspace || have < need) return set_error(MTS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed", what, have, need);
  if ((uintptr_t)workspace & 255) return set_error(MTS_ERR_ALIGNMENT, "%s: the workspace must be 256-byte aligned", what);
  return MTS_OK;
}

// An [N, D] argument: present when there are tokens, rows that do not overlap, elements on their own boundary.
int check_rows(const char* what, const char* name, const void* p, int64_t stride, int64_t N, int32_t D, int32_t dtype) {
  if (N == 0) return MTS_OK;
  if (!p || stride < D) return set_error(MTS_ERR_INVALID_ARG, "%s: %s is null or its rows overlap (stride %lld, D %d)", what, name, (long long)stride, D);
  if ((uintptr_t)p % dtype_bytes(dtype)) return set_error(MTS_ERR_ALIGNMENT, "%s: %s is no multiple of its element size", what, name);
  return MTS_OK;
}

int check_states(const char* what, const void* a, const void* b, const void* c) {
  if (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 3) return set_error(MTS_ERR_ALIGNMENT, "%s: an fp32 array is not 4-byte aligned", what);
  return MTS_OK;
}

// Alignment of all rows at once: bases and strides (in bytes) or-ed together.
struct Alignment {
  uintptr_t rows = 0, states = 0;
  void row(const void* p, int64_t stride, int bytes) { rows |= (uintptr_t)p | (uintptr_t)(stride * bytes); }
  void state(const void* p) { states |= (uintptr_t)p; }
};

// Tokens of a chunk: 64, fewer where that would leave most of the GPU without a warp (a strip is 256 bytes of a row).
int chunk_tokens(int64_t N, int32_t D, int32_t dtype) {
  const int64_t strips = ceil_div((int64_t)D * dtype_bytes(dtype), 256);
  int chunk = REC_CHUNK;
  while (chunk > 2 * REC_BATCH && ceil_div(N, chunk) * strips < MTS_REC_WARPS_WANTED) chunk /= 2;
  return chunk;
}

// Parts of the workspace, in bytes: status | counters | maps.  Strips of 32 channels are the narrowest.
struct Workspace {
  int chunk;
  int64_t chunks, groups, spans, counters, total;
  Workspace(int64_t N, int32_t D, int32_t dtype) {
    chunk = chunk_tokens(N, D, dtype);
    chunks = ceil_div(N, chunk);
    groups = ceil_div(chunks, REC_RADIX);
    spans = ceil_div(groups, REC_RADIX);
    counters = (int64_t)align_up(256 + 4 * (size_t)(groups + spans + 1) * (size_t)ceil_div(D, 32), 256);
    total = counters + (int64_t)align_up(4 * (size_t)chunks, 256) + 4 * (3 * chunks + 2 * groups + 3 * spans) * (int64_t)align_up(D, 4);
  }
};

RecArgs arguments(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride, const int64_t* offsets, const float* h0,
                  int64_t N, int64_t S, int32_t D, int32_t dtype, int vec, void* workspace) {
  RecArgs a = {gate, gate_stride, value, value_stride, offsets, h0, N, S, D};
  const Workspace w(N, D, dtype);
  a.chunk = w.chunk;
  a.chunks = (int32_t)w.chunks;
  a.strips = (int32_t)ceil_div(D, 32 * vec);
  a.groups = (int32_t)w.groups;
  a.spans = (int32_t)w.spans;
  char* p = static_cast<char*>(workspace);
  a.status = reinterpret_cast<uint32_t*>(p);
  a.group_count = reinterpret_cast<uint32_t*>(p + 256);
  a.span_count = a.group_count + w.groups * a.strips;
  a.total_count = a.span_count + w.spans * a.strips;
  a.sequence = reinterpret_cast<int32_t*>(p + w.counters);
  a.chunk_P = reinterpret_cast<float*>(p + w.counters + align_up(4 * (size_t)w.chunks, 256));
  a.chunk_B = a.chunk_P + w.chunks * D;
  a.chunk_start = a.chunk_B + w.chunks * D;
  a.group_P = a.chunk_start + w.chunks * D;
  a.group_B = a.group_P + w.groups * D;
  a.span_P = a.group_B + w.groups * D;
  a.span_B = a.span_P + w.spans * D;
  a.span_state = a.span_B + w.spans * D;
  return a;
}

// One warp per chunk and strip, at least one for the check of the offsets.
template <typename Kernel, typename... Args>
int launch_pass(const char* what, int trace_id, Kernel kernel, const RecArgs& a, cudaStream_t s, Args... args) {
  const int64_t blocks = ceil_div((int64_t)a.chunks * a.strips, REC_WARPS);
  LaunchScope scope(trace_id, s);
  kernel<<<(unsigned)(blocks < 1 ? 1 : blocks), REC_WARPS * 32, 0, s>>>(a, args...);
  return check_launch(what);
}

// fn(V, VEC): a lane holds `most` channels, fewer where a row has no use for all lanes.
template <int MOST, typename Fn>
int with_channels(int32_t D, const Alignment& al, int bytes, Fn&& fn) {
  auto vec = [&](int v) { return D % v == 0 && al.rows % (v * bytes) == 0 && al.states % (v * 4) == 0; };
  if constexpr (MOST >= 4)
    if (D > 64) return vec(4) ? fn(std::integral_constant<int, 4>(), std::true_type()) : fn(std::integral_constant<int, 4>(), std::false_type());
  if constexpr (MOST >= 2)
    if (D > 32) return vec(2) ? fn(std::integral_constant<int, 2>(), std::true_type()) : fn(std::integral_constant<int, 2>(), std::false_type());
  return fn(std::integral_constant<int, 1>(), std::true_type());
}

}  // namespace

extern "C" int64_t mts_recurrence_chunks(int64_t N, int32_t D, int32_t dtype) {
  return N < 0 || D < 1 || !known_dtype(dtype) ? 0 : ceil_div(N, REC_BATCH);
}

extern "C" size_t mts_recurrence_workspace_bytes(int64_t N, int64_t S, int32_t D, int32_t dtype) {
  if (N < 0 || S < 0 || D < 1 || !known_dtype(dtype)) return 0;
  const Workspace w(N, D, dtype);
  return (size_t)w.total;
}

extern "C" int mts_recurrence_forward(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride, int32_t dtype,
                                      int64_t N, int32_t D, const int64_t* offsets, int64_t S, const float* h0, void* out,
                                      int64_t out_stride, float* h_final, float* entry_states, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  const char* what = "recurrence_forward";
  int rc = check_sizes(what, N, S, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "gate", gate, gate_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "value", value, value_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "out", out, out_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_states(what, h0, h_final, entry_states);
  if (rc == MTS_OK && S > 0 && !offsets) rc = set_error(MTS_ERR_INVALID_ARG, "%s: null offsets", what);
  const size_t need = mts_recurrence_workspace_bytes(N, S, D, dtype);
  if (rc == MTS_OK) rc = check_workspace(what, workspace, workspace_bytes, need);
  if (rc != MTS_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Workspace w(N, D, dtype);
  if (w.groups > 1 || S == 0) rc = check_cuda(cudaMemsetAsync(workspace, 0, (size_t)w.counters, s), "cudaMemsetAsync(recurrence counters)");
  if (rc != MTS_OK || S == 0) return rc;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    Alignment al;
    al.row(gate, gate_stride, sizeof(T));
    al.row(value, value_stride, sizeof(T));
    al.row(out, out_stride, sizeof(T));
    al.state(h0);
    al.state(h_final);
    al.state(entry_states);
    return with_channels<8 / sizeof(T)>(D, al, sizeof(T), [&](auto v, auto q) {
      constexpr int V = decltype(v)::value;
      constexpr bool VEC = decltype(q)::value;
      const RecArgs a = arguments(gate, gate_stride, value, value_stride, offsets, h0, N, S, D, dtype, V, workspace);
      const int e = launch_pass(what, K_RECURRENCE_FWD, recurrence_forward_maps<T, V, VEC>, a, s);
      return e != MTS_OK ? e : launch_pass(what, K_RECURRENCE_FWD, recurrence_forward_walk<T, V, VEC>, a, s, static_cast<T*>(out), out_stride,
                                           h_final, entry_states);
    });
  });
}

extern "C" int mts_recurrence_backward(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride, int32_t dtype,
                                       int64_t N, int32_t D, const int64_t* offsets, int64_t S, const float* h0,
                                       const float* entry_states, const void* grad_out, int64_t grad_out_stride,
                                       const float* grad_final, void* grad_gate, int64_t grad_gate_stride, void* grad_value,
                                       int64_t grad_value_stride, float* grad_h0, void* workspace, size_t workspace_bytes,
                                       void* stream) {
  const char* what = "recurrence_backward";
  int rc = check_sizes(what, N, S, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "gate", gate, gate_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "value", value, value_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "grad_out", grad_out, grad_out_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "grad_gate", grad_gate, grad_gate_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_rows(what, "grad_value", grad_value, grad_value_stride, N, D, dtype);
  if (rc == MTS_OK) rc = check_states(what, h0, entry_states, grad_final);
  if (rc == MTS_OK) rc = check_states(what, grad_h0, nullptr, nullptr);
  if (rc == MTS_OK && ((S > 0 && !offsets) || (N > 0 && !entry_states)))
    rc = set_error(MTS_ERR_INVALID_ARG, "%s: null offsets or entry_states", what);
  const size_t need = mts_recurrence_workspace_bytes(N, S, D, dtype);
  if (rc == MTS_OK) rc = check_workspace(what, workspace, workspace_bytes, need);
  if (rc != MTS_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Workspace w(N, D, dtype);
  if (w.groups > 1 || S == 0) rc = check_cuda(cudaMemsetAsync(workspace, 0, (size_t)w.counters, s), "cudaMemsetAsync(recurrence counters)");
  if (rc != MTS_OK || S == 0) return rc;
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    Alignment al;
    al.row(gate, gate_stride, sizeof(T));
    al.row(value, value_stride, sizeof(T));
    al.row(grad_out, grad_out_stride, sizeof(T));
    al.row(grad_gate, grad_gate_stride, sizeof(T));
    al.row(grad_value, grad_value_stride, sizeof(T));
    al.state(h0);
    al.state(entry_states);
    al.state(grad_final);
    al.state(grad_h0);
    return with_channels<8 / sizeof(T)>(D, al, sizeof(T), [&](auto v, auto q) {
      constexpr int V = decltype(v)::value;
      constexpr bool VEC = decltype(q)::value;
      const RecArgs a = arguments(gate, gate_stride, value, value_stride, offsets, h0, N, S, D, dtype, V, workspace);
      const int e = launch_pass(what, K_RECURRENCE_BWD, recurrence_backward_maps<T, V, VEC>, a, s, static_cast<const T*>(grad_out),
                                grad_out_stride, grad_final);
      return e != MTS_OK ? e : launch_pass(what, K_RECURRENCE_BWD, recurrence_backward_walk<T, V, VEC>, a, s, entry_states,
                                           static_cast<const T*>(grad_out), grad_out_stride, grad_final, static_cast<T*>(grad_gate),
                                           grad_gate_stride, static_cast<T*>(grad_value), grad_value_stride, grad_h0);
    });
  });
}

extern "C" int mts_recurrence_status(const void* workspace, int32_t* host_status, void* stream) {
  if (!workspace || !host_status) return set_error(MTS_ERR_INVALID_ARG, "recurrence_status: null argument");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint32_t word = 0;
  int rc = check_cuda(cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, s), "cudaMemcpyAsync(status)");
  if (rc == MTS_OK) rc = check_cuda(cudaStreamSynchronize(s), "cudaStreamSynchronize(status)");
  *host_status = rc == MTS_OK ? (int32_t)word : 0;
  return rc;
}
