// Gated linear recurrence over packed ragged sequences, forward and backward:
//
//   z_t = 1 / (1 + exp(-gate_t)),  h_t = z_t value_t + (1 - z_t) h_{t-1}
//
// Composition of steps: any run of tokens maps the state before it to B + P * state, P the product of its 1 - z and B the state
// it reaches from 0; a run that contains a sequence's start forgets what came before it (a cut).  Runs compose, so the token
// axis is split into chunks of 64 tokens whatever the sequences are: one long sequence and a thousand short ones are the same
// work.  A block owns a tile (a chunk x a strip of channels): it computes the maps of its 8 runs of 8 tokens, publishes the
// map of the chunk, gathers the maps before it back to the start of its sequence (at most 15 chunks, 15 groups of 16 chunks and the
// state after 256 of them), and walks its tokens once more from the state they give.  Everything is read once and written
// once: memory traffic bounds it.  The association of the maps depends on the offsets alone, so the result is the
// same in every run.
//
// Waiting: published words are single 64-bit stores into memory that was filled with 0xFF; a reader polls the word itself.  All blocks
// are resident (cooperative launch) and take their tiles in ascending order, and a tile waits for lower ones only: the
// lowest unfinished tile never waits.  Every poll loop has a limit all the same.
#include <type_traits>

#include "dense.cuh"

namespace mts {

constexpr int REC_RUN = 8;                        // tokens of one thread
constexpr int REC_RUNS = 8;
constexpr int REC_CHUNK = REC_RUN * REC_RUNS;     // tokens of a tile
constexpr int REC_RADIX = 16;                     // chunks per group, groups per span
constexpr int REC_SPAN = REC_RADIX * REC_RADIX;   // chunks between two published states
constexpr int REC_STATUS_OFFSETS = 1, REC_STATUS_TIMEOUT = 2;
constexpr int REC_POLLS = 1 << 21;                // polls of one word before a wait gives up (about a second)
constexpr uint32_t REC_UNPUBLISHED = 0xFFFFFFFFu;

struct RecArgs {
  const void* gate; int64_t gate_stride;
  const void* value; int64_t value_stride;
  const int64_t* offsets;
  const float* h0;
  int64_t N, S;
  int32_t D;
  int32_t chunks, strips;
  int32_t wide;                // rows, strides and bases on 16-byte boundaries (else 4-element ones, or none: template)
  uint32_t* status;            // status bits, inverted: the workspace starts as all ones
  unsigned long long* chunk_map;   // [chunks, D], [groups, D], [spans, D]
  unsigned long long* group_map;
  unsigned long long* span_state;
};

__device__ __forceinline__ void raise_status(const RecArgs& a, int bit) { atomicAnd(a.status, ~(uint32_t)bit); }

// exp through the hardware's 2^x and the reciprocal: a few units of 2^-23, the gate's size times as much for large ones.
__device__ __forceinline__ float sigmoid_f32(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

// h + z (x - h) as z x + (1 - z) h without rounding 1 - z: x itself for z = 1, h for z = 0.
__device__ __forceinline__ float blend(float z, float x, float h) { return fmaf(z, x, fmaf(-z, h, h)); }

// A map state -> B + P * state.  P >= 0 is a product of 1 - z; P = -0 marks a cut, whose result is B even if the state before it is
// infinite or NaN.
struct Map { float P, B; };
__device__ __forceinline__ bool is_cut(float P) { return __float_as_int(P) < 0; }
__device__ __forceinline__ float apply(Map m, float h) { return is_cut(m.P) ? m.B : fmaf(m.P, h, m.B); }
__device__ __forceinline__ Map then(Map first, Map second) {          // first, then second
  return Map{is_cut(second.P) ? -0.f : first.P * second.P, apply(second, first.B)};
}
constexpr float CUT = -0.f;

__device__ __forceinline__ void publish(unsigned long long* at, Map m) {
  uint32_t p = __float_as_uint(m.P);
  if (p == REC_UNPUBLISHED) p = 0x7FFFFFFFu;                          // a NaN of the one pattern that means "not yet"
  const unsigned long long w = ((unsigned long long)__float_as_uint(m.B) << 32) | p;
  asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" :: "l"(at), "l"(w) : "memory");
}
__device__ __forceinline__ unsigned long long peek(const unsigned long long* at) {
  unsigned long long w;
  asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(w) : "l"(at) : "memory");
  return w;
}

__device__ __forceinline__ bool timed_out(const RecArgs& a) {
  return !(*reinterpret_cast<volatile uint32_t*>(a.status) & REC_STATUS_TIMEOUT);
}

// Composition of the published maps at[0], at[step], ..., count of them (count <= 16), in that order; waits for those still missing.
__device__ __forceinline__ Map gather(const RecArgs& a, const unsigned long long* at, int64_t step, int count) {
  Map m = {1.f, 0.f};
  for (int i = 0; i < count; i += 8) {
    unsigned long long w[8];
    int polls = 0;
    bool missing;
    do {
      missing = false;
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = i + k < count ? peek(at + (i + k) * step) : 0ull;
#pragma unroll
      for (int k = 0; k < 8; ++k) missing |= (uint32_t)w[k] == REC_UNPUBLISHED;
      ++polls;                          // once a wait has run out the others give up soon, too
    } while (missing && polls < REC_POLLS && (polls % 1024 || !timed_out(a)));
    if (missing) raise_status(a, REC_STATUS_TIMEOUT);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k < count) m = then(m, Map{__uint_as_float((uint32_t)w[k]), __uint_as_float((uint32_t)(w[k] >> 32))});
  }
  return m;
}

// One channel of a tile, whose maps are counted by `index` in the order of the walk, by two threads.  The near one publishes the tile's own
// map and returns the composition of those before it in its group; the far one returns (as B) the state before the group.  Both
// begin at `from`, the tile where the sequence began, and the association is the same whatever is published when.
__device__ __forceinline__ Map join(const RecArgs& a, int index, int from, bool near, int channel, Map own) {
  Map m = {1.f, 0.f};
  if (channel < 0) return m;
  const int group = index / REC_RADIX, span = index / REC_SPAN;
  from = min(max(from, 0), index);
  if (near) {
    const bool ends_group = index % REC_RADIX == REC_RADIX - 1;
    if (!ends_group) publish(a.chunk_map + (int64_t)index * a.D + channel, own);
    const int lo = max(from, group * REC_RADIX);
    m = gather(a, a.chunk_map + (int64_t)lo * a.D + channel, a.D, index - lo);
    if (ends_group) publish(a.group_map + (int64_t)group * a.D + channel, then(m, own));
  } else if (from < group * REC_RADIX) {
    if (from < span * REC_SPAN) m = gather(a, a.span_state + (int64_t)(span - 1) * a.D + channel, 0, 1);
    const int lo = max(from / REC_RADIX, span * REC_RADIX);
    m = then(m, gather(a, a.group_map + (int64_t)lo * a.D + channel, a.D, group - lo));
  }
  return m;
}

// What a tile knows of the sequences in its chunk.
struct ChunkSequences {
  unsigned long long first, last;      // tokens that begin / end their sequence
  int64_t far;                         // forward: first token of the sequence that holds the chunk's first token;
                                       // backward: last token of the one that holds the chunk's last token
  int32_t first_of[REC_CHUNK];         // sequence that begins at the token
  int32_t last_of[REC_CHUNK];          // sequence that ends at the token
};

// One warp: the sequence of the chunk's first token by a search with 32 probes a step, then the sequences up to the chunk's end.  Every
// index is bounded whatever the offsets hold.
template <bool BACKWARD>
__device__ void find_sequences(const RecArgs& a, int chunk, ChunkSequences* out) {
  const int lane = lane_id();
  const int64_t t0 = (int64_t)chunk * REC_CHUNK, t1 = min(t0 + REC_CHUNK, a.N);
  int64_t lo = 0, hi = a.S;
  while (hi - lo > 1) {                                               // offsets[lo] <= t0 < offsets[hi]
    const int64_t step = (hi - lo + 31) / 32, i = lo + lane * step;
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, i < hi && a.offsets[i] <= t0));
    lo += (int64_t)max(n - 1, 0) * step;
    hi = min(hi, lo + step);
  }
  unsigned long long first = 0, last = 0;
  int64_t far = BACKWARD ? t1 - 1 : t0;
  for (int64_t base = lo; base < a.S; base += 32) {
    const int64_t s = base + lane;
    const int64_t b = s < a.S ? a.offsets[s] : a.N, e = s < a.S ? a.offsets[s + 1] : a.N;
    if (e > b) {
      if (b >= t0 && b < t1) { first |= 1ull << (b - t0); out->first_of[b - t0] = (int)s; }
      if (e > t0 && e <= t1) { last |= 1ull << (e - 1 - t0); out->last_of[e - 1 - t0] = (int)s; }
      if (!BACKWARD && b <= t0 && e > t0) far = b;
      if (BACKWARD && b < t1 && e >= t1) far = e - 1;
    }
    if (__any_sync(0xFFFFFFFFu, b >= t1)) break;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    first |= __shfl_xor_sync(0xFFFFFFFFu, first, o);
    last |= __shfl_xor_sync(0xFFFFFFFFu, last, o);
    const int64_t f = __shfl_xor_sync(0xFFFFFFFFu, far, o);
    far = BACKWARD ? max(far, f) : min(far, f);
  }
  if (lane == 0) { out->first = first; out->last = last; out->far = far; }
}

// Offsets in order, from 0 to N (each thread a share of them); `row(s)` for every empty sequence, one warp each.
template <typename Fn>
__device__ void check_offsets(const RecArgs& a, Fn&& row) {
  const int64_t warps = (int64_t)gridDim.x * (blockDim.x / 32);
  bool bad = false;
  for (int64_t s0 = ((int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32) * 32; s0 < a.S; s0 += warps * 32) {
    const int64_t s = s0 + lane_id();
    const int64_t b = s < a.S ? a.offsets[s] : 0, e = s < a.S ? a.offsets[s + 1] : 1;
    if (s < a.S) bad |= b < 0 || e < b || (s == 0 && b != 0) || (s == a.S - 1 && e != a.N);
    unsigned empty = __ballot_sync(0xFFFFFFFFu, s < a.S && e <= b);
    while (empty) {
      row(s0 + __ffs(empty) - 1);
      empty &= empty - 1;
    }
  }
  if (bad) raise_status(a, REC_STATUS_OFFSETS);
}

__device__ __forceinline__ void copy_async(void* smem, const void* global, int bytes, bool wide) {
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(smem);
  if (wide) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(global), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" :: "r"(to), "l"(global), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

// Four channels of one row.
template <typename T>
__device__ __forceinline__ void read4(const T* p, float (&v)[4]) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const float2 a = unpack2<T>(w.x), b = unpack2<T>(w.y);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
template <>
__device__ __forceinline__ void read4<float>(const float* p, float (&v)[4]) {
  const float4 w = *reinterpret_cast<const float4*>(p);
  v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
}
template <typename T>
__device__ __forceinline__ void write4(T* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
}
template <>
__device__ __forceinline__ void write4<float>(float* p, const float (&v)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
// The same in global memory: QUADS = rows begin on 4-element boundaries and D is a multiple of 4, else the first `left` of the
// four one by one.
template <bool QUADS, typename T>
__device__ __forceinline__ void get4(const T* p, int left, float (&v)[4]) {
  if (QUADS) {
    if (left > 0) read4(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) v[k] = to_f32(p[k]);
  }
}
template <bool QUADS, typename T>
__device__ __forceinline__ void put4(T* p, int left, const float (&v)[4]) {
  if (QUADS) {
    if (left > 0) write4(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) p[k] = from_f32<T>(v[k]);
  }
}

// A tile's [64, 4 LANES] part of an [N, D] array to shared memory; what lies outside reads as 0.
template <typename T, int LANES, bool QUADS>
__device__ __forceinline__ void fetch_rows(const RecArgs& a, const void* src, int64_t stride, int64_t t0, int c0, T* to) {
  constexpr int W = 4 * LANES, THREADS = REC_RUNS * LANES;
  const T* from = static_cast<const T*>(src);
  if (QUADS) {
    const bool wide = sizeof(T) == 4 || a.wide;
    const int per = wide ? 16 / (int)sizeof(T) : 4;                                  // elements of one copy
    const int pieces = W / per;
    for (int i = threadIdx.x; i < REC_CHUNK * pieces; i += THREADS) {
      const int r = i / pieces, c = (i - r * pieces) * per;
      const bool in = t0 + r < a.N && c0 + c < a.D;
      copy_async(to + r * W + c, in ? from + (t0 + r) * stride + c0 + c : from, in ? per * (int)sizeof(T) : 0, wide);
    }
  } else {
    for (int i = threadIdx.x; i < REC_CHUNK * W; i += THREADS) {
      const int r = i / W, c = i % W;
      to[i] = t0 + r < a.N && c0 + c < a.D ? from[(t0 + r) * stride + c0 + c] : from_f32<T>(0.f);
    }
  }
}

template <int THREADS>
__device__ __forceinline__ void worker_barrier() { asm volatile("bar.sync 1, %0;" :: "n"(THREADS) : "memory"); }

// Threads: 8 runs x LANES, four channels each, and one more warp that looks up the sequences of the block's next tile.
template <typename T, int LANES, bool QUADS>
__global__ void __launch_bounds__(REC_RUNS * LANES + 32)
recurrence_forward_scan(const RecArgs a, T* __restrict__ out, int64_t out_stride, float* h_final, float* __restrict__ entry) {
  constexpr int W = 4 * LANES, WORKERS = REC_RUNS * LANES, TILE = REC_CHUNK * W;
  extern __shared__ __align__(16) unsigned char smem[];
  T* rows = reinterpret_cast<T*>(smem);                               // [2 stages][gate, value][64][W]
  float* run_P = reinterpret_cast<float*>(rows + 4 * TILE);           // [8][W]
  float* run_B = run_P + REC_RUNS * W;
  float* near_P = run_B + REC_RUNS * W;                               // [W]: the chunks before this one in its group
  float* near_B = near_P + W;
  float* far_h = near_B + W;                                          // [W]: the state before the group
  ChunkSequences* seqs = reinterpret_cast<ChunkSequences*>(far_h + W);
  const int tiles = a.chunks * a.strips;
  const bool worker = threadIdx.x < WORKERS;
  const int run = threadIdx.x / LANES, lane4 = (threadIdx.x % LANES) * 4;

  auto fetch = [&](int tile, int stage) {
    if (tile < tiles) {
      const int64_t t0 = (int64_t)(tile / a.strips) * REC_CHUNK;
      const int c0 = tile % a.strips * W;
      fetch_rows<T, LANES, QUADS>(a, a.gate, a.gate_stride, t0, c0, rows + stage * 2 * TILE);
      fetch_rows<T, LANES, QUADS>(a, a.value, a.value_stride, t0, c0, rows + (stage * 2 + 1) * TILE);
    }
    copy_commit();
  };

  if (worker) fetch(blockIdx.x, 0);
  else if (blockIdx.x < tiles) find_sequences<false>(a, blockIdx.x / a.strips, &seqs[0]);
  if (h_final) {
    check_offsets(a, [&](int64_t s) {
      for (int d = lane_id(); d < a.D; d += 32) h_final[s * a.D + d] = a.h0 ? a.h0[s * a.D + d] : 0.f;
    });
  } else {
    check_offsets(a, [](int64_t) {});
  }
  __syncthreads();

  int stage = 0;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, stage ^= 1) {
    const int next = tile + gridDim.x;
    if (!worker) {
      if (next < tiles) find_sequences<false>(a, next / a.strips, &seqs[stage ^ 1]);
      __syncthreads();
      continue;
    }
    fetch(next, stage ^ 1);
    copy_wait<1>();
    worker_barrier<WORKERS>();

    const int chunk = tile / a.strips, c0 = tile % a.strips * W;
    const int64_t t0 = (int64_t)chunk * REC_CHUNK;
    const ChunkSequences& sq = seqs[stage];
    const T* gate = rows + stage * 2 * TILE + run * REC_RUN * W + lane4;
    const T* value = gate + TILE;
    const uint32_t firsts = (uint32_t)(sq.first >> (run * REC_RUN)) & 0xFF;
    const int left = a.D - c0 - lane4;                                // channels of this thread that exist
    const int tokens = (int)min((int64_t)REC_RUN, a.N - t0 - run * REC_RUN);

    // the maps of the runs; z is kept, in its place the state itself where a sequence begins (h0 is read once, before anything
    // that depends on it is published: h_final may be the same array)
    float z[REC_RUN][4];
#pragma unroll
    for (int i = 0; i < REC_RUN; ++i) {
#pragma unroll
      for (int k = 0; k < 4; ++k) z[i][k] = 0.f;
      if ((firsts >> i & 1) && a.h0) get4<QUADS>(a.h0 + (int64_t)sq.first_of[run * REC_RUN + i] * a.D + c0 + lane4, left, z[i]);
    }
    float P[4] = {1.f, 1.f, 1.f, 1.f}, B[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < REC_RUN; ++i) {
      float g[4], x[4];
      read4(gate + i * W, g);
      read4(value + i * W, x);
      if (firsts >> i & 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          B[k] = z[i][k] = blend(sigmoid_f32(g[k]), x[k], z[i][k]);
          P[k] = CUT;
        }
      } else if (i < tokens) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          z[i][k] = sigmoid_f32(g[k]);
          B[k] = blend(z[i][k], x[k], B[k]);
          P[k] *= 1.f - z[i][k];
        }
      }
    }
    *reinterpret_cast<float4*>(run_P + run * W + lane4) = make_float4(P[0], P[1], P[2], P[3]);
    *reinterpret_cast<float4*>(run_B + run * W + lane4) = make_float4(B[0], B[1], B[2], B[3]);
    worker_barrier<WORKERS>();

    const int ch = threadIdx.x % W;
    const bool near = threadIdx.x < W, exists = c0 + ch < a.D;
    Map own = {1.f, 0.f};
    if (near)
#pragma unroll
      for (int r = 0; r < REC_RUNS; ++r) own = then(own, Map{run_P[r * W + ch], run_B[r * W + ch]});
    const int from = sq.first & 1 ? chunk : (int)(sq.far / REC_CHUNK);
    const Map nearby = join(a, chunk, from, near, exists ? c0 + ch : -1, own);
    if (near) {
      near_P[ch] = nearby.P;
      near_B[ch] = nearby.B;
    } else {
      far_h[ch] = nearby.B;
    }
    worker_barrier<WORKERS>();
    if (near && exists && (entry || chunk % REC_SPAN == REC_SPAN - 1)) {
      const float h = apply(nearby, far_h[ch]);
      if (entry) entry[(int64_t)chunk * a.D + c0 + ch] = h;
      if (chunk % REC_SPAN == REC_SPAN - 1) publish(a.span_state + (int64_t)(chunk / REC_SPAN) * a.D + c0 + ch, Map{CUT, apply(own, h)});
    }

    // the state before the run, then its tokens
    float h[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) h[k] = apply(Map{near_P[lane4 + k], near_B[lane4 + k]}, far_h[lane4 + k]);
    for (int r = 0; r < run; ++r) {
      const float4 p = *reinterpret_cast<const float4*>(run_P + r * W + lane4);
      const float4 b = *reinterpret_cast<const float4*>(run_B + r * W + lane4);
      h[0] = apply(Map{p.x, b.x}, h[0]);
      h[1] = apply(Map{p.y, b.y}, h[1]);
      h[2] = apply(Map{p.z, b.z}, h[2]);
      h[3] = apply(Map{p.w, b.w}, h[3]);
    }
    const uint32_t lasts = (uint32_t)(sq.last >> (run * REC_RUN)) & 0xFF;
    T* to = out + (t0 + run * REC_RUN) * out_stride + c0 + lane4;
#pragma unroll
    for (int i = 0; i < REC_RUN; ++i) {
      if (i < tokens) {
        float x[4];
        read4(value + i * W, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = (firsts >> i & 1) ? z[i][k] : blend(z[i][k], x[k], h[k]);
        put4<QUADS>(to + i * out_stride, left, h);
        if ((lasts >> i & 1) && h_final) put4<QUADS>(h_final + (int64_t)sq.last_of[run * REC_RUN + i] * a.D + c0 + lane4, left, h);
      }
    }
    __syncthreads();
  }
  copy_wait<0>();
}

// The backward walks the chunks from the last to the first.  What a token hands to the one before it, c_t = (1 - z_t) G_t =
// (1 - z_t) (grad_out_t + c_{t+1}), is the same kind of map; its cut is a sequence's last token, which starts from grad_final.
// The states come from the forward's entry states, by the runs' forward maps inside the chunk.
template <typename T, int LANES, bool QUADS>
__global__ void __launch_bounds__(REC_RUNS * LANES + 32)
recurrence_backward_scan(const RecArgs a, const float* __restrict__ entry, const T* __restrict__ grad_out, int64_t grad_out_stride,
                         const float* __restrict__ grad_final, T* __restrict__ grad_gate, int64_t grad_gate_stride,
                         T* __restrict__ grad_value, int64_t grad_value_stride, float* __restrict__ grad_h0) {
  constexpr int W = 4 * LANES, WORKERS = REC_RUNS * LANES, TILE = REC_CHUNK * W;
  extern __shared__ __align__(16) unsigned char smem[];
  T* rows = reinterpret_cast<T*>(smem);                               // [2 stages][gate, value, grad_out][64][W]
  float* run_P = reinterpret_cast<float*>(rows + 6 * TILE);           // [8][W] products of 1 - z
  float* run_B = run_P + REC_RUNS * W;                                // [8][W] states
  float* run_C = run_B + REC_RUNS * W;                                // [8][W] what the run hands back
  float* near_P = run_C + REC_RUNS * W;
  float* near_B = near_P + W;
  float* far_c = near_B + W;
  ChunkSequences* seqs = reinterpret_cast<ChunkSequences*>(far_c + W);
  const int tiles = a.chunks * a.strips;
  const bool worker = threadIdx.x < WORKERS;
  const int run = threadIdx.x / LANES, lane4 = (threadIdx.x % LANES) * 4;

  auto fetch = [&](int tile, int stage) {
    if (tile < tiles) {
      const int64_t t0 = (int64_t)(a.chunks - 1 - tile / a.strips) * REC_CHUNK;
      const int c0 = tile % a.strips * W;
      fetch_rows<T, LANES, QUADS>(a, a.gate, a.gate_stride, t0, c0, rows + stage * 3 * TILE);
      fetch_rows<T, LANES, QUADS>(a, a.value, a.value_stride, t0, c0, rows + (stage * 3 + 1) * TILE);
      fetch_rows<T, LANES, QUADS>(a, grad_out, grad_out_stride, t0, c0, rows + (stage * 3 + 2) * TILE);
    }
    copy_commit();
  };

  if (worker) fetch(blockIdx.x, 0);
  else if (blockIdx.x < tiles) find_sequences<true>(a, a.chunks - 1 - blockIdx.x / a.strips, &seqs[0]);
  if (grad_h0) {
    check_offsets(a, [&](int64_t s) {
      for (int d = lane_id(); d < a.D; d += 32) grad_h0[s * a.D + d] = grad_final ? grad_final[s * a.D + d] : 0.f;
    });
  } else {
    check_offsets(a, [](int64_t) {});
  }
  __syncthreads();

  int stage = 0;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, stage ^= 1) {
    const int next = tile + gridDim.x;
    if (!worker) {
      if (next < tiles) find_sequences<true>(a, a.chunks - 1 - next / a.strips, &seqs[stage ^ 1]);
      __syncthreads();
      continue;
    }
    fetch(next, stage ^ 1);
    copy_wait<1>();
    worker_barrier<WORKERS>();

    const int back = tile / a.strips, chunk = a.chunks - 1 - back, c0 = tile % a.strips * W;     // back: chunks from the end
    const int64_t t0 = (int64_t)chunk * REC_CHUNK;
    const ChunkSequences& sq = seqs[stage];
    const T* gate = rows + stage * 3 * TILE + run * REC_RUN * W + lane4;
    const T* value = gate + TILE;
    const T* grad = value + TILE;
    const uint32_t firsts = (uint32_t)(sq.first >> (run * REC_RUN)) & 0xFF, lasts = (uint32_t)(sq.last >> (run * REC_RUN)) & 0xFF;
    const int left = a.D - c0 - lane4;
    const int tokens = (int)min((int64_t)REC_RUN, a.N - t0 - run * REC_RUN);
    auto start_state = [&](int i, float (&h)[4]) {                    // h0 of the sequence that begins at token i of the run
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = 0.f;
      if (a.h0) get4<QUADS>(a.h0 + (int64_t)sq.first_of[run * REC_RUN + i] * a.D + c0 + lane4, left, h);
    };
    auto end_gradient = [&](int i, float (&c)[4]) {                   // grad_final of the sequence that ends there
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] = 0.f;
      if (grad_final) get4<QUADS>(grad_final + (int64_t)sq.last_of[run * REC_RUN + i] * a.D + c0 + lane4, left, c);
    };

    // the runs' maps in both directions
    float z[REC_RUN][4], P[4] = {1.f, 1.f, 1.f, 1.f}, h[4] = {0.f, 0.f, 0.f, 0.f}, c[4] = {0.f, 0.f, 0.f, 0.f}, before[4] = {0.f, 0.f, 0.f, 0.f};
    if (entry) get4<QUADS>(entry + (int64_t)chunk * a.D + c0 + lane4, left, before);
#pragma unroll
    for (int i = 0; i < REC_RUN; ++i) {
      float g[4], x[4];
      read4(gate + i * W, g);
      read4(value + i * W, x);
      if (firsts >> i & 1) start_state(i, h);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        z[i][k] = i < tokens ? sigmoid_f32(g[k]) : 0.f;
        h[k] = blend(z[i][k], x[k], h[k]);
        P[k] *= 1.f - z[i][k];
      }
    }
#pragma unroll
    for (int i = REC_RUN - 1; i >= 0; --i) {
      float d[4];
      read4(grad + i * W, d);
      if (lasts >> i & 1) end_gradient(i, c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float G = i < tokens ? d[k] + c[k] : c[k];
        c[k] = fmaf(-z[i][k], G, G);
      }
    }
    *reinterpret_cast<float4*>(run_P + run * W + lane4) = make_float4(P[0], P[1], P[2], P[3]);
    *reinterpret_cast<float4*>(run_B + run * W + lane4) = make_float4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<float4*>(run_C + run * W + lane4) = make_float4(c[0], c[1], c[2], c[3]);
    worker_barrier<WORKERS>();

    const int ch = threadIdx.x % W;
    const bool near = threadIdx.x < W, exists = c0 + ch < a.D;
    Map own = {1.f, 0.f};
    if (near)
#pragma unroll
      for (int r = REC_RUNS - 1; r >= 0; --r)
        own = then(own, Map{sq.last >> (r * REC_RUN) & 0xFF ? CUT : run_P[r * W + ch], run_C[r * W + ch]});
    const int end = (int)(min(t0 + REC_CHUNK, a.N) - 1 - t0);         // the chunk's last token
    const int from = sq.last >> end & 1 ? back : a.chunks - 1 - (int)min(sq.far / REC_CHUNK, (int64_t)a.chunks - 1);
    const Map nearby = join(a, back, from, near, exists ? c0 + ch : -1, own);
    if (near) {
      near_P[ch] = nearby.P;
      near_B[ch] = nearby.B;
    } else {
      far_c[ch] = nearby.B;
    }

    // meanwhile the states before the run's tokens: value - h
    float away[REC_RUN][4];
    for (int r = 0; r < run; ++r) {
      const bool cut = sq.first >> (r * REC_RUN) & 0xFF;
      const float4 p = *reinterpret_cast<const float4*>(run_P + r * W + lane4);
      const float4 b = *reinterpret_cast<const float4*>(run_B + r * W + lane4);
      before[0] = cut ? b.x : fmaf(p.x, before[0], b.x);
      before[1] = cut ? b.y : fmaf(p.y, before[1], b.y);
      before[2] = cut ? b.z : fmaf(p.z, before[2], b.z);
      before[3] = cut ? b.w : fmaf(p.w, before[3], b.w);
    }
#pragma unroll
    for (int i = 0; i < REC_RUN; ++i) {
      float x[4];
      read4(value + i * W, x);
      if (firsts >> i & 1) start_state(i, before);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        away[i][k] = x[k] - before[k];
        before[k] = blend(z[i][k], x[k], before[k]);
      }
    }
    worker_barrier<WORKERS>();
    if (near && exists && back % REC_SPAN == REC_SPAN - 1)
      publish(a.span_state + (int64_t)(back / REC_SPAN) * a.D + c0 + ch, Map{CUT, apply(own, apply(nearby, far_c[ch]))});

#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = apply(Map{near_P[lane4 + k], near_B[lane4 + k]}, far_c[lane4 + k]);
    for (int r = REC_RUNS - 1; r > run; --r) {
      const bool cut = sq.last >> (r * REC_RUN) & 0xFF;
      const float4 p = *reinterpret_cast<const float4*>(run_P + r * W + lane4);
      const float4 b = *reinterpret_cast<const float4*>(run_C + r * W + lane4);
      c[0] = cut ? b.x : fmaf(p.x, c[0], b.x);
      c[1] = cut ? b.y : fmaf(p.y, c[1], b.y);
      c[2] = cut ? b.z : fmaf(p.z, c[2], b.z);
      c[3] = cut ? b.w : fmaf(p.w, c[3], b.w);
    }
    T* to_gate = grad_gate + (t0 + run * REC_RUN) * grad_gate_stride + c0 + lane4;
    T* to_value = grad_value + (t0 + run * REC_RUN) * grad_value_stride + c0 + lane4;
#pragma unroll
    for (int i = REC_RUN - 1; i >= 0; --i) {
      if (i < tokens) {
        float d[4], gv[4], gg[4];
        read4(grad + i * W, d);
        if (lasts >> i & 1) end_gradient(i, c);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float G = d[k] + c[k], keep = 1.f - z[i][k];
          gv[k] = z[i][k] * G;
          gg[k] = gv[k] * (keep * away[i][k]);
          c[k] = fmaf(-z[i][k], G, G);
        }
        put4<QUADS>(to_value + i * grad_value_stride, left, gv);
        put4<QUADS>(to_gate + i * grad_gate_stride, left, gg);
        if ((firsts >> i & 1) && grad_h0) put4<QUADS>(grad_h0 + (int64_t)sq.first_of[run * REC_RUN + i] * a.D + c0 + lane4, left, c);
      }
    }
    __syncthreads();
  }
  copy_wait<0>();
}

}  // namespace mts

using namespace mts;

namespace {

int check_sizes(const char* what, int64_t N, int64_t S, int32_t D, int32_t dtype) {
  if (N < 0 || S < 0 || D < 1 || !known_dtype(dtype))
    return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, S %lld, D %d, dtype %d", what, (long long)N, (long long)S, D, dtype);
  if (N >= (1ll << 31) - (1 << 16) || S >= (1ll << 31) - (1 << 16) || D > (1 << 20) ||
      ceil_div(N, REC_CHUNK) * ceil_div(D, 32) >= (1ll << 30))
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

RecArgs arguments(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride, const int64_t* offsets, const float* h0,
                  int64_t N, int64_t S, int32_t D, void* workspace) {
  RecArgs a = {gate, gate_stride, value, value_stride, offsets, h0, N, S, D};
  a.chunks = (int32_t)ceil_div(N, REC_CHUNK);
  char* w = static_cast<char*>(workspace);
  a.status = reinterpret_cast<uint32_t*>(w);
  a.chunk_map = reinterpret_cast<unsigned long long*>(w + 256);
  a.group_map = a.chunk_map + (int64_t)a.chunks * D;
  a.span_state = a.group_map + ceil_div(a.chunks, REC_RADIX) * D;
  return a;
}

// One block per tile up to what the device holds at once (the blocks of one launch wait for one another).
template <typename Kernel>
int launch_scan(const char* what, int trace_id, Kernel kernel, int threads, size_t smem, const RecArgs& a, void** args, cudaStream_t s) {
  int dev = 0, sms = 0, per_sm = 0;
  int rc = check_cuda(cudaGetDevice(&dev), "cudaGetDevice");
  if (rc == MTS_OK) rc = check_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), "sm count");
  if (rc == MTS_OK) rc = check_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem), "shared memory size");
  if (rc == MTS_OK) rc = check_cuda(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem), "occupancy");
  if (rc != MTS_OK) return rc;
  const int64_t tiles = (int64_t)a.chunks * a.strips, room = (int64_t)sms * per_sm;
  const unsigned grid = (unsigned)(tiles < 1 ? 1 : tiles < room ? tiles : room);
  LaunchScope scope(trace_id, s);
  return check_cuda(cudaLaunchCooperativeKernel((const void*)kernel, dim3(grid), dim3(threads), args, smem, s), what);
}

template <typename T, int LANES, bool BACKWARD>
constexpr size_t scan_smem() {
  constexpr size_t W = 4 * LANES;
  return 2 * (BACKWARD ? 3 : 2) * REC_CHUNK * W * sizeof(T) + ((BACKWARD ? 3 : 2) * REC_RUNS + 3) * W * sizeof(float) + 2 * sizeof(ChunkSequences);
}

// fn(LANES, QUADS) as compile-time constants.  A strip of channels is 256 bytes of a row wide, less for rows that are narrower.
template <typename T, typename Fn>
int with_shape(int32_t D, bool quads, Fn&& fn) {
  using L8 = std::integral_constant<int, 8>;
  using L16 = std::integral_constant<int, 16>;
  using L32 = std::integral_constant<int, 32>;
  if (D <= 32) return quads ? fn(L8(), std::true_type()) : fn(L8(), std::false_type());
  if constexpr (sizeof(T) == 2)
    if (D > 64) return quads ? fn(L32(), std::true_type()) : fn(L32(), std::false_type());
  return quads ? fn(L16(), std::true_type()) : fn(L16(), std::false_type());
}

}  // namespace

extern "C" int64_t mts_recurrence_chunks(int64_t N, int32_t D, int32_t dtype) {
  return N < 0 || D < 1 || !known_dtype(dtype) ? 0 : ceil_div(N, REC_CHUNK);
}

extern "C" size_t mts_recurrence_workspace_bytes(int64_t N, int64_t S, int32_t D, int32_t dtype) {
  if (N < 0 || S < 0 || D < 1 || !known_dtype(dtype)) return 0;
  const int64_t chunks = ceil_div(N, REC_CHUNK);
  return 256 + sizeof(unsigned long long) * (size_t)(chunks + ceil_div(chunks, REC_RADIX) + ceil_div(chunks, REC_SPAN)) * (size_t)D;
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
  rc = check_cuda(cudaMemsetAsync(workspace, 0xFF, need, s), "cudaMemsetAsync(recurrence maps)");
  if (rc != MTS_OK || S == 0) return rc;
  RecArgs a = arguments(gate, gate_stride, value, value_stride, offsets, h0, N, S, D, workspace);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    Alignment al;
    al.row(gate, gate_stride, sizeof(T));
    al.row(value, value_stride, sizeof(T));
    al.row(out, out_stride, sizeof(T));
    al.state(h0);
    al.state(h_final);
    al.state(entry_states);
    a.wide = al.rows % 16 == 0 && D % (16 / (int)sizeof(T)) == 0;
    const bool quads = al.rows % (4 * sizeof(T)) == 0 && D % 4 == 0 && al.states % 16 == 0;
    return with_shape<T>(D, quads, [&](auto lanes, auto q) {
      constexpr int LANES = decltype(lanes)::value;
      a.strips = (int32_t)ceil_div(D, 4 * LANES);
      T* o = static_cast<T*>(out);
      void* args[] = {&a, &o, &out_stride, &h_final, &entry_states};
      return launch_scan(what, K_RECURRENCE_FWD, recurrence_forward_scan<T, LANES, decltype(q)::value>, REC_RUNS * LANES + 32,
                         scan_smem<T, LANES, false>(), a, args, s);
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
  rc = check_cuda(cudaMemsetAsync(workspace, 0xFF, need, s), "cudaMemsetAsync(recurrence maps)");
  if (rc != MTS_OK || S == 0) return rc;
  RecArgs a = arguments(gate, gate_stride, value, value_stride, offsets, h0, N, S, D, workspace);
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
    a.wide = al.rows % 16 == 0 && D % (16 / (int)sizeof(T)) == 0;
    const bool quads = al.rows % (4 * sizeof(T)) == 0 && D % 4 == 0 && al.states % 16 == 0;
    return with_shape<T>(D, quads, [&](auto lanes, auto q) {
      constexpr int LANES = decltype(lanes)::value;
      a.strips = (int32_t)ceil_div(D, 4 * LANES);
      const T* go = static_cast<const T*>(grad_out);
      T* gg = static_cast<T*>(grad_gate);
      T* gv = static_cast<T*>(grad_value);
      void* args[] = {&a, &entry_states, &go, &grad_out_stride, &grad_final, &gg, &grad_gate_stride, &gv, &grad_value_stride, &grad_h0};
      return launch_scan(what, K_RECURRENCE_BWD, recurrence_backward_scan<T, LANES, decltype(q)::value>, REC_RUNS * LANES + 32,
                         scan_smem<T, LANES, true>(), a, args, s);
    });
  });
}

extern "C" int mts_recurrence_status(const void* workspace, int32_t* host_status, void* stream) {
  if (!workspace || !host_status) return set_error(MTS_ERR_INVALID_ARG, "recurrence_status: null argument");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint32_t word = 0;
  int rc = check_cuda(cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, s), "cudaMemcpyAsync(status)");
  if (rc == MTS_OK) rc = check_cuda(cudaStreamSynchronize(s), "cudaStreamSynchronize(status)");
  *host_status = rc == MTS_OK ? (int32_t)~word : 0;
  if (rc == MTS_OK && (*host_status & REC_STATUS_TIMEOUT))
    rc = set_error(MTS_ERR_TIMEOUT, "recurrence: a bounded wait ran out, the results of the last call are incomplete");
  return rc;
}
