// Gated linear recurrence over packed ragged sequences, forward and backward:
//
//   z_t = 1 / (1 + exp(-gate_t)),  h_t = z_t value_t + (1 - z_t) h_{t-1}
//
// Any run of tokens maps the state before it to B + P * state, P the product of its 1 - z and B the state it reaches from 0; a run
// that contains a sequence's start forgets what came before it (a cut).  Runs compose, so the token axis is cut into chunks
// whatever the sequences are: one long sequence and a thousand short ones are the same work.  A chunk x a strip of channels (8 bytes
// of a row per lane) is two pieces of work for a warp:
//   map:  the chunk's map, if its last sequence goes on behind it, from that sequence's start on (what lies before it in the chunk is
//         forgotten).  The last warp of eight neighbours composes their map, and so on; behind every 512 chunks a state is kept.
//   walk: the state before the chunk from at most seven maps of each of three levels and a kept state, then the chunk's tokens.
// Warps take the pieces from a counter: all maps, then all walks in calls of up to REC_LAG pieces of a kind, else in turn, a walk REC_LAG
// pieces behind its chunk's map.  By then the maps it needs have long been published (a word written by one SM is seen by another only 1 to
// 2 us later).  The association of the maps depends on the
// offsets alone: the result is the same in every run.
//
// What bounds it: memory.  A chunk's rows are read for its map and again for its walk (in the backward: gate and gradient, then all
// three), which the L2 cache does not hold in between.  524,287 tokens x 256 in fp16, one sequence: 218 to 228 us on different GPUs, 5.9 to
// 6.1 TB/s of what is moved (reads from memory are twice the inputs), 3.5 to 3.7 TB/s of each input once; 1,000 histories of 120,007 tokens
// in bf16: 69 us (1.8 times the inputs); forward and backward of 2,048 histories, 250,001 x 200: 106 + 160 us (1.7 and 1.4 times).  In all of
// these every map comes before the walks; 262,143 x 1,024 in bf16, in turn: 420 us.  Ragged calls of that size are one wave of warps, whose
// tokens go one after the other.
//
// Waiting: a piece waits only for pieces of lower numbers, which running or finished warps have taken, and the lowest unfinished one
// waits for nothing.  Every wait has a limit all the same, after which the status word says so.
//
// Tried before (524,287 x 256): one pass that keeps its rows in shared memory, with maps gathered over levels of groups by every tile
// (424 to 690 us: three publications in a row per tile outlast what shared memory can hold back), or linked in order by dedicated
// warps (321 us: 40 ns a link); two launches, maps and walks (250 us: the composition at the end of the first leaves SMs idle).
#include <type_traits>

#include "dense.cuh"

namespace mts {

// Measured on 250,001 tokens x 200 and 524,287 x 256 (16-bit): 12, 14, 16 blocks of one warp per SM take 120 / 109 / 108 us and 223 / 219 / 219 us
// in the forward, 20 and 24 of them a tenth more than 16 (registers spill); 10, 11, 12, 14 take 177 / 167 / 168 / 184 us in the backward.
constexpr int FWD_BLOCKS = 16, BWD_BLOCKS = 12;
constexpr int REC_WARPS_WANTED = 2368;            // chunks are halved until there are so many pieces of a kind: 16 per SM
// Pieces between a chunk's map and its walk; calls with fewer of a kind take all maps first.  512, 2,048, 4,096 and all of them: one sequence of
// 524,287 x 256 in bf16 (4,096 of a kind) 255 / 227 / 218 / 218 us, with its backward 640 / 581 / 566 / 566; 262,143 x 1,024 (8,192) 460 / 424 / 420 / 427
// and 1,198 / 1,102 / 1,090 / 1,095; 1,048,575 x 256 (8,192) 469 / 428 / 420 / 426: a walk must not wait for its maps, and a short way does not
// keep the rows in the L2 cache.
constexpr int REC_LAG = 4096;
constexpr int REC_CHUNK = 256;                    // tokens of a chunk at most
constexpr int REC_PART = 64;                      // tokens whose borders are looked up together: a bit mask of them is one word
constexpr int REC_BATCH = 8;                      // tokens in registers, and between two states kept for the backward
constexpr int REC_SHORT = 4096;                   // tokens of a call that threads may walk one by one
constexpr int REC_RADIX_BITS = 3;
constexpr int REC_RADIX = 1 << REC_RADIX_BITS;    // maps composed into one of the next level
constexpr int REC_LEVELS = 4;                     // levels of maps, chunks included; a state is kept behind every map of the highest, 512 chunks
constexpr int REC_STATUS_OFFSETS = 1, REC_STATUS_TIMEOUT = 2;
constexpr int REC_POLLS = 1 << 21;                // polls before a wait gives up (about a second)
constexpr uint32_t READY_MAP = 1, READY_CUT = 2;  // a published map, and one that contains a cut

// One level of maps, or (P unused) the kept states.
struct RecLevel {
  uint32_t* ready;             // [n, strips]
  uint32_t* done;              // [n, strips] parts of the map that are ready
  float* P;                    // [n, D]
  float* B;
};

struct RecArgs {
  const void* gate; int64_t gate_stride;
  const void* value; int64_t value_stride;
  const int64_t* offsets;
  const float* h0;
  int64_t N, S;
  int32_t D;
  int32_t chunk;               // tokens of a chunk
  int32_t chunks, strips;
  int32_t lag;                 // pieces between the map of a chunk and its walk
  uint32_t* status;
  uint32_t* ticket;
  float* chunk_start;          // [chunks, D] state in which the chunk's last sequence starts
  RecLevel level[REC_LEVELS + 1];
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
  if constexpr (VEC) {
    return left > 0 ? load_f32<V>(p) : all<V>(0.f);
  } else {
    float x[V];
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] = k < left ? p[k] : 0.f;
    return gathered<V>(x);
  }
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
// What another warp of the same launch has published, after the flag that says so.
template <int V, bool VEC>
__device__ __forceinline__ Channels<V> load_published(const float* p, int left) {
  float x[V];
  if constexpr (VEC && V == 4) {
    if (left <= 0) return all<V>(0.f);
    asm volatile("ld.relaxed.gpu.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "l"(p) : "memory");
  } else if constexpr (VEC && V == 2) {
    if (left <= 0) return all<V>(0.f);
    asm volatile("ld.relaxed.gpu.global.v2.f32 {%0, %1}, [%2];" : "=f"(x[0]), "=f"(x[1]) : "l"(p) : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      x[k] = 0.f;
      if (k < left) asm volatile("ld.relaxed.gpu.global.f32 %0, [%1];" : "=f"(x[k]) : "l"(p + k) : "memory");
    }
  }
  return gathered<V>(x);
}

// ------------------------------------------------------------------------------- maps
template <int V>
struct Map { Channels<V> P, B; };

// After this warp's writes to what `flag` stands for.
__device__ __forceinline__ void set_ready(uint32_t* flag, uint32_t how) {
  __syncwarp();
  if (lane_id() == 0) {
    __threadfence();
    asm volatile("st.release.gpu.global.u32 [%0], %1;" :: "l"(flag), "r"(how) : "memory");
  }
}
// Every lane waits for a flag of its own (null: none) and gets what it says.
__device__ __forceinline__ uint32_t wait_ready(const RecArgs& a, const uint32_t* flag) {
  uint32_t v = flag ? 0u : READY_MAP;
  for (int polls = 1;; ++polls) {
    if (!v) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(flag) : "memory");
    if (__all_sync(0xFFFFFFFFu, v != 0)) break;
    // offsets out of order may name chunks that publish nothing; once a wait has run out the others give up soon, too
    const uint32_t status = polls % 64 ? 0u : *reinterpret_cast<volatile uint32_t*>(a.status);
    if (polls >= REC_POLLS || status) {
      if (lane_id() == 0 && !status) atomicOr(a.status, (uint32_t)REC_STATUS_TIMEOUT);
      break;
    }
  }
  __syncwarp();
  return v;
}

// Publishes the map of chunk `index` (counted in the order of the walk) and those of the higher levels that it completes.
template <int V, bool VEC>
__device__ __forceinline__ void publish(const RecArgs& a, int index, int strip, int c, Map<V> m, bool cut) {
  const int left = a.D - c;
#pragma unroll 1
  for (int l = 0;; ++l) {
    const RecLevel& to = a.level[l];
    put<V, VEC>(to.P + (int64_t)index * a.D + c, left, m.P);
    put<V, VEC>(to.B + (int64_t)index * a.D + c, left, m.B);
    set_ready(to.ready + (int64_t)index * a.strips + strip, cut ? READY_CUT : READY_MAP);
    if (l + 1 == REC_LEVELS) break;
    // the last of eight to come here goes on (a set that the end of the tokens leaves short is never needed)
    const int parent = index >> REC_RADIX_BITS;
    uint32_t before = 0;
    if (lane_id() == 0)
      asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.level[l + 1].done + (int64_t)parent * a.strips + strip) : "memory");
    if (__shfl_sync(0xFFFFFFFFu, before, 0) != REC_RADIX - 1) return;
    const uint32_t how = wait_ready(a, lane_id() < REC_RADIX ? to.ready + ((int64_t)parent * REC_RADIX + lane_id()) * a.strips + strip : nullptr);
    const uint32_t cuts = __ballot_sync(0xFFFFFFFFu, how == READY_CUT);
    m = {all<V>(1.f), all<V>(0.f)};
    const float* P = to.P + (int64_t)parent * REC_RADIX * a.D + c;
    const float* B = to.B + (int64_t)parent * REC_RADIX * a.D + c;
#pragma unroll
    for (int k = 0; k < REC_RADIX; ++k, P += a.D, B += a.D) {
      const Channels<V> Pk = load_published<V, VEC>(P, left), Bk = load_published<V, VEC>(B, left);
      if (cuts >> k & 1) m.B = Bk;
      else m = {Pk * m.P, fma(Pk, m.B, Bk)};
    }
    cut = cuts != 0;
    index = parent;
  }
  // the state behind a map of the highest level: the next one kept
  const RecLevel& kept = a.level[REC_LEVELS];
  if (!cut && index > 0) {
    wait_ready(a, lane_id() == 0 ? kept.ready + (int64_t)index * a.strips + strip : nullptr);
    m.B = fma(m.P, load_published<V, VEC>(kept.B + (int64_t)index * a.D + c, left), m.B);
  }
  put<V, VEC>(kept.B + (int64_t)(index + 1) * a.D + c, left, m.B);
  set_ready(kept.ready + (int64_t)(index + 1) * a.strips + strip, READY_MAP);
}

// The state before chunk `index`, whose first sequence (in the order of the walk) began in chunk `from` < index.
template <int V, bool VEC>
__device__ __forceinline__ Channels<V> state_before(const RecArgs& a, int index, int strip, int from, int c) {
  from = max(0, min(from, index - 1));
  // lane 8 l + k: map k of level l, of those between the start of the next level's map (or `from`) and the chunk, seven at most; lane 31:
  // the kept state
  const int l = lane_id() / REC_RADIX, shift = l * REC_RADIX_BITS, k = lane_id() % REC_RADIX;
  const int at = index >> shift, parent = at >> REC_RADIX_BITS << REC_RADIX_BITS;
  // a level is used where the one below does not reach back to `from`
  const bool used = l < REC_LEVELS - 1 && from >> shift < at && (l == 0 || from >> (shift - REC_RADIX_BITS) < (index >> (shift - REC_RADIX_BITS) >> REC_RADIX_BITS << REC_RADIX_BITS));
  const int lo = max(from >> shift, parent);
  const bool mine = used && k < REC_RADIX - 1 && lo + k < at;
  constexpr int TOP = (REC_LEVELS - 1) * REC_RADIX_BITS;
  const int top = index >> TOP;
  const bool kept = from < top << TOP;
  const uint32_t* flag = mine ? a.level[l].ready + (int64_t)(lo + k) * a.strips + strip : nullptr;
  if (lane_id() == 31 && kept) flag = a.level[REC_LEVELS].ready + (int64_t)top * a.strips + strip;
  const uint32_t how = wait_ready(a, flag);
  Channels<V> h = all<V>(0.f);
  const uint32_t maps = __ballot_sync(0xFFFFFFFFu, mine), cuts = __ballot_sync(0xFFFFFFFFu, mine && how == READY_CUT);
  const int left = a.D - c;
  if (kept) h = load_published<V, VEC>(a.level[REC_LEVELS].B + (int64_t)top * a.D + c, left);
#pragma unroll
  for (int i = REC_LEVELS - 2; i >= 0; --i) {
    const int n = __popc(maps >> (i * REC_RADIX) & 0xFF), first = __shfl_sync(0xFFFFFFFFu, lo, i * REC_RADIX);
    const float* P = a.level[i].P + (int64_t)first * a.D + c;
    const float* B = a.level[i].B + (int64_t)first * a.D + c;
#pragma unroll 4
    for (int j = 0; j < n; ++j, P += a.D, B += a.D) {
      const Channels<V> Pj = load_published<V, VEC>(P, left), Bj = load_published<V, VEC>(B, left);
      h = cuts >> (i * REC_RADIX + j) & 1 ? Bj : fma(Pj, h, Bj);
    }
  }
  return h;
}

// ------------------------------------------------------------------------------- sequences
// One warp: the last sequence that begins at or before token t, by a search with 32 probes a step.  Every index is bounded whatever the
// offsets hold.
__device__ __forceinline__ int find_sequence(const RecArgs& a, int64_t t) {
  int64_t lo = 0, hi = a.S;
  while (hi - lo > 1) {                                               // offsets[lo] <= t < offsets[hi]
    const int64_t step = (hi - lo + 31) / 32, i = lo + lane_id() * step;
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, i < hi && a.offsets[i] <= t));
    lo += (int64_t)max(n - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  return (int)lo;
}

// The borders among the tokens [t0, t1) of a part.
struct Borders {
  unsigned long long first, last;      // tokens that begin / end their sequence
  int64_t head_begin;                  // of the sequence that holds the part's first token
  int64_t tail_end;                    // of the one that holds its last token
  int32_t lo;                          // in: a sequence at or before the part's first token; out: the one of its last token
};
// Looked up by one warp from sequence `lo` on; the sequences' numbers go to first_of / last_of, by token, and those of sequences that
// begin here and end behind `kept_end` bitwise inverted to first_of.
__device__ __forceinline__ Borders find_borders(const RecArgs& a, int lo, int64_t t0, int64_t t1, int64_t kept_end, int32_t* first_of, int32_t* last_of) {
  Borders q = {0, 0, t0, t1, lo};
  __syncwarp();
  for (int64_t base = lo; base < a.S; base += 32) {
    const int64_t s = base + lane_id();
    const int64_t b = s < a.S ? a.offsets[s] : a.N, e = s < a.S ? a.offsets[s + 1] : a.N;
    const bool some = e > b;
    if (some && b >= t0 && b < t1) { q.first |= 1ull << (b - t0); first_of[b - t0] = e > kept_end ? ~(int)s : (int)s; }
    if (some && e > t0 && e <= t1) { q.last |= 1ull << (e - 1 - t0); last_of[e - 1 - t0] = (int)s; }
    const unsigned head = __ballot_sync(0xFFFFFFFFu, some && b <= t0 && e > t0), tail = __ballot_sync(0xFFFFFFFFu, some && b < t1 && e >= t1);
    if (head) q.head_begin = __shfl_sync(0xFFFFFFFFu, b, __ffs(head) - 1);
    if (tail) {
      q.tail_end = __shfl_sync(0xFFFFFFFFu, e, __ffs(tail) - 1);
      q.lo = (int)base + __ffs(tail) - 1;
    }
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

// Offsets in order, from 0 to N; `row(s)` for every empty sequence.  Warp `number` of n takes an even share of the sequences.
template <typename Fn>
__device__ __forceinline__ void check_offsets(const RecArgs& a, int64_t number, int64_t n, Fn&& row) {
  const int64_t share = (a.S + n - 1) / n, end = min(a.S, (number + 1) * share);
  bool bad = false;
  for (int64_t s0 = number * share; s0 < end; s0 += 32) {
    const int64_t s = s0 + lane_id();
    const int64_t b = s < end ? a.offsets[s] : 0, e = s < end ? a.offsets[s + 1] : 1;
    if (s < end) bad |= b < 0 || e < b || (s == 0 && b != 0) || (s == a.S - 1 && e != a.N);
    unsigned empty = __ballot_sync(0xFFFFFFFFu, s < end && e <= b);
    while (empty) {
      row(s0 + __ffs(empty) - 1);
      empty &= empty - 1;
    }
  }
  if (bad) atomicOr(a.status, (uint32_t)REC_STATUS_OFFSETS);
}

// What a warp works on: the map or the walk of a chunk (counted from the end where BACKWARD) and a strip of channels.
struct Piece {
  bool walk;
  int index, chunk, strip;
  int64_t t0, t1, number;      // number: of the walk, for the share of the offsets to check
  __device__ __forceinline__ Piece(const RecArgs& a, bool backward) {
    uint32_t t = 0;
    if (lane_id() == 0) t = atomicAdd(a.ticket, 1u);
    t = __shfl_sync(0xFFFFFFFFu, t, 0);
    // the first maps; walks and maps in turn; the last walks
    const int64_t n = (int64_t)a.chunks * a.strips, u = (int64_t)t - a.lag;
    const bool mixed = u >= 0 && t < 2 * n - a.lag;
    walk = u >= 0 && (!mixed || u % 2 == 0);
    number = u < 0 ? t : mixed ? (walk ? u / 2 : a.lag + u / 2) : t - n;
    index = (int)(number / a.strips);
    strip = (int)(number - (int64_t)index * a.strips);
    chunk = backward ? a.chunks - 1 - index : index;
    t0 = (int64_t)chunk * a.chunk;
    t1 = min(t0 + a.chunk, a.N);
  }
};

// A lane's channels of the rows of an [N, D] array, from one row on, walked up or down by a pointer.  A lane behind the last channel
// reads the first ones: no test where rows are read.
template <typename T, int V, bool VEC>
struct Rows {
  T* at;
  int64_t stride;
  int left;
  __device__ __forceinline__ Rows(const void* p, int64_t stride_, int64_t row, int c, int left_)
      : at(static_cast<T*>(const_cast<void*>(p)) + row * stride_ + (left_ > 0 ? c : 0)), stride(stride_), left(left_) {}
  __device__ __forceinline__ void move(int rows) { at += rows * stride; }
  __device__ __forceinline__ Raw<T, V> get() const { return VEC ? load_raw<T, V>(at) : get_raw<T, V, VEC>(at, left); }
  __device__ __forceinline__ Raw<T, V> next() { const Raw<T, V> r = get(); at += stride; return r; }
  __device__ __forceinline__ Raw<T, V> previous() { at -= stride; return get(); }
  __device__ __forceinline__ void put(Channels<V> v) const { mts::put<V, VEC>(at, left, v); }
  // A batch of n rows from here on, the first `live` of them; the others give 0.  Moves behind the batch.
  template <int N>
  __device__ __forceinline__ void load(int live, Raw<T, V> (&r)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i, at += stride) r[i] = i < live ? get() : Raw<T, V>{};
  }
};
// Brings rows 8 to 15 behind where two arrays stand towards the L2 cache: every lane asks for half a strip of one row.  The registers
// hold a batch on its way, which is less than the memory's latency needs: 524,287 tokens x 256 take 219 us with it, on the same GPU 233 without and 226 from eight rows
// further on.  In the backward it costs as much as it gives (169 / 168 us), but for the kept states (164).
template <typename T, int V, bool VEC>
struct Ahead {
  using R = Rows<T, V, VEC>;
  int64_t by;
  bool second;
  __device__ __forceinline__ Ahead(const R& a, const R& b, int c, int D) : second(lane_id() & 1) {
    const int own = a.left > 0 ? c : 0, half = min(c - lane_id() * V + (lane_id() >> 1 & 1) * 16 * V, D - 1), row = 8 + (lane_id() >> 2);
    by = row * (second ? b.stride : a.stride) + half - own;
  }
  __device__ __forceinline__ void operator()(const R& a, const R& b) const {
    asm volatile("prefetch.global.L2 [%0];" :: "l"((second ? b.at : a.at) + by));
  }
};
// Bits of n tokens from token `rel` of a part on.
template <int N>
__device__ __forceinline__ uint32_t batch_bits(unsigned long long mask, int rel) { return (uint32_t)(mask >> (rel % REC_PART)) & ((1u << N) - 1); }

// In all four walks a row's registers take the row one batch ahead as soon as they have been read: a batch is always on its way.

// ------------------------------------------------------------------------------- forward
constexpr int FWD_BATCH = 8;           // rows on their way; 4 leave room for more warps and take as long
constexpr int FWD_STEP = REC_BATCH;    // tokens of one turn of the inner loops
static_assert(FWD_STEP % FWD_BATCH == 0, "a state is kept where a batch begins");
static_assert(FWD_STEP == 8 && FWD_BATCH == 8, "eight rows are asked for ahead");

template <typename T, int V, bool VEC>
__device__ __forceinline__ void forward_map(const RecArgs& a, const Piece& it) {
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c;
  const int s = find_sequence(a, it.t1 - 1);
  const int64_t begin = a.offsets[s], end = min(a.offsets[s + 1], a.N);
  const bool goes_on = end > it.t1, cut = !goes_on || (begin >= it.t0 && begin < it.t1);
  Map<V> m = {all<V>(1.f), all<V>(0.f)};
  if (goes_on) {                                                    // a whole chunk: the sequence goes on
    const int start = cut ? (int)(begin - it.t0) : 0;
    Channels<V> from = all<V>(0.f);
    if (cut) {
      if (a.h0) from = get<V, VEC>(a.h0 + (int64_t)s * a.D + c, left);
      put<V, VEC>(a.chunk_start + (int64_t)it.chunk * a.D + c, left, from);
    }
    int rel = start & ~(FWD_BATCH - 1);
    Rows<T, V, VEC> gate(a.gate, a.gate_stride, it.t0 + rel, c, left), value(a.value, a.value_stride, it.t0 + rel, c, left);
    Raw<T, V> g[FWD_BATCH], x[FWD_BATCH];
    gate.load(FWD_BATCH, g);
    value.load(FWD_BATCH, x);
    // the batch with the start: what is before it there is forgotten
    const int later = a.chunk - rel - FWD_BATCH;                        // tokens behind this batch
#pragma unroll
    for (int i = 0; i < FWD_BATCH; ++i) {
      const Channels<V> nz = minus_sigmoid(unpack<T, V>(g[i])), nx = unpack<T, V, true>(x[i]);
      if (rel + i == start) m = {all<V>(1.f), from};
      m.B = blend(nz, nx, m.B);
      m.P = fma(nz, m.P, m.P);
    }
    gate.load(later, g);
    value.load(later, x);
    const auto step = [&](int i) {
      const Channels<V> nz = minus_sigmoid(unpack<T, V>(g[i])), nx = unpack<T, V, true>(x[i]);
      m.B = blend(nz, nx, m.B);
      m.P = fma(nz, m.P, m.P);
    };
    rel = later;                                                        // tokens to go, FWD_BATCH of them in registers
    const Ahead<T, V, VEC> ahead(gate, value, c, a.D);
#pragma unroll 1
    for (; rel >= FWD_STEP + FWD_BATCH; rel -= FWD_STEP) {
      if (rel >= FWD_STEP + 2 * FWD_BATCH) ahead(gate, value);
#pragma unroll
      for (int i = 0; i < FWD_STEP; ++i) {
        step(i % FWD_BATCH);
        g[i % FWD_BATCH] = gate.next();
        x[i % FWD_BATCH] = value.next();
      }
    }
#pragma unroll 1
    for (; rel > 0; rel -= FWD_BATCH) {
#pragma unroll
      for (int i = 0; i < FWD_BATCH; ++i) step(i);
      gate.load(rel - FWD_BATCH, g);
      value.load(rel - FWD_BATCH, x);
    }
  }
  publish<V, VEC>(a, it.index, it.strip, c, m, cut);
}

template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(32, FWD_BLOCKS)
recurrence_forward_kernel(const RecArgs a, T* __restrict__ out, int64_t out_stride, float* h_final, float* __restrict__ entry) {
  __shared__ int32_t first_of[REC_PART], last_of[REC_PART];
  const Piece it(a, false);
  if (!it.walk) return forward_map<T, V, VEC>(a, it);
  const auto empty_row = [&](int64_t s) {
    if (h_final)
      for (int d = lane_id(); d < a.D; d += 32) h_final[s * a.D + d] = a.h0 ? a.h0[s * a.D + d] : 0.f;
  };
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c, tokens = (int)(it.t1 - it.t0);
  Rows<T, V, VEC> gate(a.gate, a.gate_stride, it.t0, c, left), value(a.value, a.value_stride, it.t0, c, left), to(out, out_stride, it.t0, c, left);
  Raw<T, V> g[FWD_BATCH], x[FWD_BATCH];
  gate.load(tokens, g);
  value.load(tokens, x);
  check_offsets(a, it.number, (int64_t)a.chunks * a.strips, empty_row);
  const Ahead<T, V, VEC> ahead(gate, value, c, a.D);
  Borders q = {0, 0, 0, 0, find_sequence(a, it.t0)};
  Channels<V> h = all<V>(0.f);
#pragma unroll 1
  for (int rel = 0; rel < tokens;) {
    if (rel % REC_PART == 0) {
      q = find_borders(a, q.lo, it.t0 + rel, min(it.t0 + rel + REC_PART, it.t1), it.t1, first_of, last_of);
      if (rel == 0 && !(q.first & 1)) h = state_before<V, VEC>(a, it.index, it.strip, (int)(q.head_begin / a.chunk), c);
    }
    // tokens of the part before the next border; FWD_STEP at a time as long as the FWD_BATCH behind them exist
    const unsigned long long borders = (q.first | q.last) >> (rel % REC_PART);
    const int clear = min(borders ? __ffsll(borders) - 1 : REC_PART - rel % REC_PART, tokens - rel - FWD_BATCH);
    if (clear >= FWD_STEP && rel % FWD_STEP == 0) {
#pragma unroll 1
      for (const int end = rel + clear / FWD_STEP * FWD_STEP; rel < end; rel += FWD_STEP) {
        if (entry) put<V, VEC>(entry + ((it.t0 + rel) / REC_BATCH) * a.D + c, left, h);
        if (rel + FWD_STEP + 2 * FWD_BATCH <= tokens) ahead(gate, value);
#pragma unroll
        for (int i = 0; i < FWD_STEP; ++i, to.at += to.stride) {
          const Channels<V> nz = minus_sigmoid(unpack<T, V>(g[i % FWD_BATCH])), nx = unpack<T, V, true>(x[i % FWD_BATCH]);
          g[i % FWD_BATCH] = gate.next();
          x[i % FWD_BATCH] = value.next();
          h = blend(nz, nx, h);
          to.put(h);
        }
      }
    } else {
      const uint32_t firsts = batch_bits<FWD_BATCH>(q.first, rel), lasts = batch_bits<FWD_BATCH>(q.last, rel);
      if (entry && rel % REC_BATCH == 0) put<V, VEC>(entry + ((it.t0 + rel) / REC_BATCH) * a.D + c, left, h);
      const int live = tokens - rel;
      Channels<V> s[FWD_BATCH];
#pragma unroll
      for (int i = 0; i < FWD_BATCH; ++i) {
        s[i] = all<V>(0.f);
        if (firsts >> i & 1) {
          // the start of a sequence that goes on behind the chunk was kept with the chunk's map: h_final may be the same array as h0,
          // and the warp that writes it does not wait for this one
          const int f = first_of[rel % REC_PART + i];
          if (f < 0) {
            wait_ready(a, lane_id() == 0 ? a.level[0].ready + (int64_t)it.index * a.strips + it.strip : nullptr);
            s[i] = load_published<V, VEC>(a.chunk_start + (int64_t)it.chunk * a.D + c, left);
          } else if (a.h0) s[i] = get<V, VEC>(a.h0 + (int64_t)f * a.D + c, left);
        }
      }
#pragma unroll
      for (int i = 0; i < FWD_BATCH; ++i, to.at += to.stride) {
        if (i < live) {
          if (firsts >> i & 1) h = s[i];
          h = blend(minus_sigmoid(unpack<T, V>(g[i])), unpack<T, V, true>(x[i]), h);
          to.put(h);
          if ((lasts >> i & 1) && h_final) put<V, VEC>(h_final + (int64_t)last_of[rel % REC_PART + i] * a.D + c, left, h);
        }
      }
      gate.load(live - FWD_BATCH, g);
      value.load(live - FWD_BATCH, x);
      rel += FWD_BATCH;
    }
  }
}

// Single tokens: a thread for every channel of every sequence.  One launch, no counters to clear, and no search: 192 sequences of one token
// x 128 take a third of the pieces' time.  A long sequence among empty ones would be walked token by token, so the host takes this only
// where sequences hold one token on average and REC_SHORT in all.
template <typename T>
__global__ void __launch_bounds__(128)
recurrence_forward_short(const RecArgs a, T* __restrict__ out, int64_t out_stride, float* h_final, float* __restrict__ entry) {
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    bool bad = false;
    for (int64_t s = threadIdx.x; s < a.S; s += blockDim.x) {
      const int64_t b = a.offsets[s], e = a.offsets[s + 1];
      bad |= b < 0 || e < b || (s == 0 && b != 0) || (s == a.S - 1 && e != a.N);
    }
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) *a.status = any ? (uint32_t)REC_STATUS_OFFSETS : 0u;
  }
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.D) return;
  for (int64_t s = blockIdx.y; s < a.S; s += gridDim.y) {
    const int64_t begin = min(max(a.offsets[s], (int64_t)0), a.N), end = min(max(a.offsets[s + 1], begin), a.N);
    Channels<1> h = {{a.h0 ? a.h0[s * a.D + c] : 0.f}};
    const T* gate = static_cast<const T*>(a.gate) + begin * a.gate_stride + c;
    const T* value = static_cast<const T*>(a.value) + begin * a.value_stride + c;
    for (int64_t t = begin; t < end; ++t, gate += a.gate_stride, value += a.value_stride) {
      if (entry && t % REC_BATCH == 0) entry[t / REC_BATCH * a.D + c] = h.p[0];
      h = blend(minus_sigmoid(Channels<1>{{to_f32(*gate)}}), Channels<1>{{-to_f32(*value)}}, h);
      out[t * out_stride + c] = from_f32<T>(h.p[0]);
    }
    if (h_final) h_final[s * a.D + c] = h.p[0];
  }
}

// ------------------------------------------------------------------------------- backward
// What a token hands to the one before it, c_t = (1 - z_t) G_t = (1 - z_t) (grad_out_t + c_{t+1}), is the same kind of map, walked from
// the last chunk to the first; its cut is a sequence's last token, which starts from grad_final.
template <typename T, int V, bool VEC>
__device__ __forceinline__ void backward_map(const RecArgs& a, const Piece& it, const T* grad_out, int64_t grad_out_stride, const float* grad_final) {
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c;
  const int s = find_sequence(a, it.t0);
  const int64_t begin = a.offsets[s], end = a.offsets[s + 1];
  const bool goes_on = begin < it.t0, cut = !goes_on || (end > it.t0 && end <= it.t1);
  Map<V> m = {all<V>(1.f), all<V>(0.f)};
  if (goes_on) {
    const int tokens = (int)((cut ? end : it.t1) - it.t0);
    if (cut && grad_final) m.B = get<V, VEC>(grad_final + (int64_t)s * a.D + c, left);
    int rel = (tokens - 1) & ~(REC_BATCH - 1);
    Rows<T, V, VEC> gate(a.gate, a.gate_stride, it.t0 + rel, c, left), grad(grad_out, grad_out_stride, it.t0 + rel, c, left);
    Raw<T, V> g[REC_BATCH], d[REC_BATCH];
    gate.load(tokens - rel, g);
    grad.load(tokens - rel, d);
    gate.move(-REC_BATCH);                                              // to the batch's first row: rows before it come next
    grad.move(-REC_BATCH);
#pragma unroll 1
    for (; rel >= 0; rel -= REC_BATCH) {
      const int here = tokens - rel;
#pragma unroll
      for (int i = REC_BATCH - 1; i >= 0; --i) {
        const Channels<V> nz = minus_sigmoid(unpack<T, V>(g[i])), dv = unpack<T, V>(d[i]);
        if (rel > 0) {
          g[i] = gate.previous();
          d[i] = grad.previous();
        }
        if (i < here) {
          const Channels<V> G = dv + m.B;
          m.B = fma(nz, G, G);
          m.P = fma(nz, m.P, m.P);
        }
      }
    }
  }
  publish<V, VEC>(a, it.index, it.strip, c, m, cut);
}

// A batch is walked forward from the state that the forward left before it, for -z and the distance from value to state, then backward.
template <typename T, int V, bool VEC>
__global__ void __launch_bounds__(32, BWD_BLOCKS)
recurrence_backward_kernel(const RecArgs a, const float* __restrict__ entry, const T* __restrict__ grad_out, int64_t grad_out_stride,
                           const float* __restrict__ grad_final, T* __restrict__ grad_gate, int64_t grad_gate_stride,
                           T* __restrict__ grad_value, int64_t grad_value_stride, float* __restrict__ grad_h0) {
  __shared__ int32_t first_of[REC_PART], last_of[REC_PART];
  const Piece it(a, true);
  if (!it.walk && a.chunks > 0) return backward_map<T, V, VEC>(a, it, grad_out, grad_out_stride, grad_final);
  const auto empty_row = [&](int64_t s) {
    if (grad_h0)
      for (int d = lane_id(); d < a.D; d += 32) grad_h0[s * a.D + d] = grad_final ? grad_final[s * a.D + d] : 0.f;
  };
  if (a.chunks == 0) return check_offsets(a, blockIdx.x, gridDim.x, empty_row);
  const int c = (it.strip * 32 + lane_id()) * V, left = a.D - c, tokens = (int)(it.t1 - it.t0);
  int rel = (tokens - 1) & ~(REC_BATCH - 1);
  Rows<T, V, VEC> gate(a.gate, a.gate_stride, it.t0 + rel, c, left), value(a.value, a.value_stride, it.t0 + rel, c, left),
      grad(grad_out, grad_out_stride, it.t0 + rel, c, left), to_gate(grad_gate, grad_gate_stride, it.t0 + rel + REC_BATCH, c, left),
      to_value(grad_value, grad_value_stride, it.t0 + rel + REC_BATCH, c, left);
  Raw<T, V> g[REC_BATCH], x[REC_BATCH], d[REC_BATCH];
  gate.load(tokens - rel, g);
  value.load(tokens - rel, x);
  grad.load(tokens - rel, d);
  gate.move(-2 * REC_BATCH);                                            // to the batch before; the gradient to the first row of this one
  value.move(-2 * REC_BATCH);
  grad.move(-REC_BATCH);
  check_offsets(a, it.number, (int64_t)a.chunks * a.strips, empty_row);
  const int lo = find_sequence(a, it.t0);
  Borders q = {0, 0, 0, 0, lo};
  Channels<V> carry = all<V>(0.f);
#pragma unroll 1
  for (bool start = true; rel >= 0; rel -= REC_BATCH, start = false) {
    if (start || rel % REC_PART == REC_PART - REC_BATCH) {
      const int64_t p0 = it.t0 + rel / REC_PART * REC_PART;
      q = find_borders(a, lo, p0, min(p0 + REC_PART, it.t1), INT64_MAX, first_of, last_of);
      if (start && !(q.last >> ((tokens - 1) % REC_PART) & 1))
        carry = state_before<V, VEC>(a, it.index, it.strip, a.chunks - 1 - (int)min((q.tail_end - 1) / a.chunk, (int64_t)a.chunks - 1), c);
    }
    const int live = tokens - rel;
    const uint32_t firsts = batch_bits<REC_BATCH>(q.first, rel), lasts = batch_bits<REC_BATCH>(q.last, rel);
    Channels<V> h = all<V>(0.f), nz[REC_BATCH], away[REC_BATCH];        // away: - (value - state before the token)
    const float* kept = entry + (it.t0 + rel) / REC_BATCH * a.D + c;
    if (!(firsts & 1)) h = get<V, VEC>(kept, left);
    if (rel >= 2 * REC_BATCH && left > 0) asm volatile("prefetch.global.L2 [%0];" :: "l"(kept - 2 * a.D));     // registers for it are not to be had
    if (!(firsts | lasts) && live >= REC_BATCH && rel > 0) {
#pragma unroll
      for (int i = 0; i < REC_BATCH; ++i) {
        const Channels<V> nx = unpack<T, V, true>(x[i]);
        nz[i] = minus_sigmoid(unpack<T, V>(g[i]));
        g[i] = gate.next();
        x[i] = value.next();
        away[i] = nx + h;
        h = blend(nz[i], nx, h);
      }
#pragma unroll
      for (int i = REC_BATCH - 1; i >= 0; --i) {
        const Channels<V> G = unpack<T, V>(d[i]) + carry, nG = nz[i] * G;          // -z G
        d[i] = grad.previous();
        carry = fma(nz[i], G, G);
        to_value.at -= to_value.stride;
        to_gate.at -= to_gate.stride;
        to_value.put(nG * all<V>(-1.f));
        to_gate.put(nG * fma(nz[i], away[i], away[i]));
      }
      gate.move(-2 * REC_BATCH);
      value.move(-2 * REC_BATCH);
    } else {
#pragma unroll
      for (int i = 0; i < REC_BATCH; ++i) {
        if (firsts >> i & 1) h = a.h0 ? get<V, VEC>(a.h0 + (int64_t)first_of[rel % REC_PART + i] * a.D + c, left) : all<V>(0.f);
        const Channels<V> nx = unpack<T, V, true>(x[i]);
        nz[i] = minus_sigmoid(unpack<T, V>(g[i]));
        away[i] = nx + h;
        h = blend(nz[i], nx, h);
      }
#pragma unroll
      for (int i = REC_BATCH - 1; i >= 0; --i) {
        to_value.at -= to_value.stride;
        to_gate.at -= to_gate.stride;
        if (i < live) {
          if (lasts >> i & 1) carry = grad_final ? get<V, VEC>(grad_final + (int64_t)last_of[rel % REC_PART + i] * a.D + c, left) : all<V>(0.f);
          const Channels<V> G = unpack<T, V>(d[i]) + carry, nG = nz[i] * G;
          carry = fma(nz[i], G, G);
          to_value.put(nG * all<V>(-1.f));
          to_gate.put(nG * fma(nz[i], away[i], away[i]));
          if ((firsts >> i & 1) && grad_h0) put<V, VEC>(grad_h0 + (int64_t)first_of[rel % REC_PART + i] * a.D + c, left, carry);
        }
      }
      const int next = rel > 0 ? REC_BATCH : 0;
      grad.move(-REC_BATCH);
      gate.load(next, g);
      value.load(next, x);
      grad.load(next, d);
      gate.move(-2 * REC_BATCH);
      value.move(-2 * REC_BATCH);
      grad.move(-REC_BATCH);
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
      ceil_div(N, 2 * REC_BATCH) * ceil_div(D, 32) >= (1ll << 30))
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

// Tokens of a chunk: 256, fewer where that would leave most of the GPU without a warp (a strip is 256 bytes of a row).
int chunk_tokens(int64_t N, int32_t D, int32_t dtype) {
  const int64_t strips = ceil_div((int64_t)D * dtype_bytes(dtype), 256);
  int chunk = REC_CHUNK;
  while (chunk > 2 * REC_BATCH && ceil_div(N, chunk) * strips < REC_WARPS_WANTED) chunk /= 2;
  return chunk;
}

// Parts of the workspace, in bytes: status and ticket | flags and counts | maps.  Strips of 32 channels are the narrowest.
struct Workspace {
  int chunk;
  int64_t n[REC_LEVELS + 1], counters, total;
  Workspace(int64_t N, int32_t D, int32_t dtype) {
    chunk = chunk_tokens(N, D, dtype);
    n[0] = ceil_div(N, chunk);
    for (int l = 1; l < REC_LEVELS; ++l) n[l] = ceil_div(n[l - 1], REC_RADIX);
    n[REC_LEVELS] = n[REC_LEVELS - 1] + 1;
    int64_t all = 0;
    for (int l = 0; l <= REC_LEVELS; ++l) all += n[l];
    counters = (int64_t)align_up(256 + 8 * (size_t)all * (size_t)ceil_div(D, 32), 256);
    total = counters + 4 * (n[0] + 2 * all) * (int64_t)align_up(D, 4);
  }
};

RecArgs arguments(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride, const int64_t* offsets, const float* h0,
                  int64_t N, int64_t S, int32_t D, int32_t dtype, int vec, void* workspace) {
  RecArgs a = {gate, gate_stride, value, value_stride, offsets, h0, N, S, D};
  const Workspace w(N, D, dtype);
  a.chunk = w.chunk;
  a.chunks = (int32_t)w.n[0];
  a.strips = (int32_t)ceil_div(D, 32 * vec);
  const int64_t pieces = w.n[0] * a.strips;
  a.lag = (int32_t)(pieces < REC_LAG ? pieces : REC_LAG);
  char* p = static_cast<char*>(workspace);
  a.status = reinterpret_cast<uint32_t*>(p);
  a.ticket = a.status + 1;
  uint32_t* flags = reinterpret_cast<uint32_t*>(p + 256);
  a.chunk_start = reinterpret_cast<float*>(p + w.counters);
  float* maps = a.chunk_start + w.n[0] * D;
  for (int l = 0; l <= REC_LEVELS; ++l) {
    a.level[l].ready = flags;
    a.level[l].done = flags + w.n[l] * a.strips;
    flags += 2 * w.n[l] * a.strips;
    a.level[l].P = maps;
    a.level[l].B = maps + w.n[l] * D;
    maps += 2 * w.n[l] * D;
  }
  return a;
}

// A warp for every piece of work; without tokens (the backward's, the forward then takes the single-token kernel) one for the offsets.
template <typename Kernel, typename... Args>
int launch_pieces(const char* what, int trace_id, Kernel kernel, const RecArgs& a, cudaStream_t s, Args... args) {
  const int64_t warps = 2 * (int64_t)a.chunks * a.strips;
  LaunchScope scope(trace_id, s);
  kernel<<<(unsigned)(warps < 1 ? 1 : warps), 32, 0, s>>>(a, args...);
  return check_launch(what);
}

// fn(V, VEC): a lane holds MOST channels, fewer where a row has no use for all lanes: 200,000 tokens in bf16 with 32 and 64 channels take 34.9
// and 40.7 us with one and two of them a lane, 51.1 and 52.6 us with four.
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
  if (N <= S && N <= REC_SHORT && S > 0) {
    const RecArgs a = arguments(gate, gate_stride, value, value_stride, offsets, h0, N, S, D, dtype, 1, workspace);
    return with_dtype(dtype, [&](auto t) {
      using T = decltype(t);
      LaunchScope scope(K_RECURRENCE_FWD, s);
      recurrence_forward_short<T><<<dim3((unsigned)ceil_div(D, 128), (unsigned)(S < 65535 ? S : 65535)), 128, 0, s>>>(a, static_cast<T*>(out), out_stride,
                                                                                                                  h_final, entry_states);
      return check_launch(what);
    });
  }
  const Workspace w(N, D, dtype);
  rc = check_cuda(cudaMemsetAsync(workspace, 0, (size_t)w.counters, s), "cudaMemsetAsync(recurrence counters)");
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
      return launch_pieces(what, K_RECURRENCE_FWD, recurrence_forward_kernel<T, V, VEC>, a, s, static_cast<T*>(out), out_stride, h_final,
                           entry_states);
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
  rc = check_cuda(cudaMemsetAsync(workspace, 0, (size_t)w.counters, s), "cudaMemsetAsync(recurrence counters)");
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
      return launch_pieces(what, K_RECURRENCE_BWD, recurrence_backward_kernel<T, V, VEC>, a, s, entry_states, static_cast<const T*>(grad_out),
                           grad_out_stride, grad_final, static_cast<T*>(grad_gate), grad_gate_stride, static_cast<T*>(grad_value),
                           grad_value_stride, grad_h0);
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
  if (rc == MTS_OK && (*host_status & REC_STATUS_TIMEOUT))
    rc = set_error(MTS_ERR_TIMEOUT, "recurrence: a bounded wait ran out, the results of the last call are incomplete");
  return rc;
}
