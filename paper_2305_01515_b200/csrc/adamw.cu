// AdamW over many tensors in one launch, moments in 32 or in 8 bits.
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
//   p = p - lr wd p - (lr / (1 - beta1^t)) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Every element is read and written once and costs a few dozen instructions, so the memory traffic bounds it: 28 bytes
// per element with fp32 parameters, gradients and moments, 16 with 8-bit moments.  A warp owns one block of 256 elements, eight
// consecutive ones per lane (one 16- or 32-byte access per array); in 8 bits the block is also the unit that shares a scale, so its
// largest moment is one warp reduction and nothing leaves the registers.  A block of threads owns eight such blocks of
// one tensor, found through a map made once, so that tensors of any number and size share one launch.
//
// Parameters in 16 bits with fp32 masters and moments, 120 M elements of 28 bytes: 521 to 533 us on different GPUs, 96 to 98.6% of the copy rate.  8-bit moments with
// fp32 parameters and bf16 gradients, 100 M elements of 14 bytes: step 320 to 325 us, 4.4 TB/s: 80 instructions per element, a third of them for
// the codes, keep the integer units busy (113 with correctly rounded root and quotient and the check for finite values by element:
// 437 us); their export, 10 bytes per element, 152 us at the copy rate.
#include <math.h>

#include <new>

#include "dense.cuh"

namespace mts {

constexpr int ADAM_WARPS = 8;
constexpr int ADAM_BLOCK = MTS_ADAMW_BLOCK;
static_assert(ADAM_BLOCK == 32 * 8, "a block is one warp of eight elements per lane");

struct AdamTensor {
  void* param;
  float* master;
  int64_t n;
  int64_t first;       // first element of the tensor in the state
  int32_t decays;
};

struct AdamChunk { int32_t tensor, index; };      // eight blocks of a tensor: blocks [8 index, 8 index + 8)

struct AdamState {
  float* m32;
  float* v32;
  uint8_t* m8;
  uint8_t* v8;
  float* m_scale;
  float* v_scale;
};

struct AdamConstants {
  float beta1, one_minus_beta1, beta2, one_minus_beta2;
  float inv_root2;     // 1 / sqrt(1 - beta2^step)
  float eps;
  float rate;          // lr / (1 - beta1^step)
  float decay;         // lr * weight_decay
  uint32_t seed_word;
};

// ------------------------------------------------------------------------------- 8-bit moments
// Codes stand for fp32 numbers in (0, 1] of which the exponent and the three leading mantissa bits are kept: value of
// code c > 0 = bits ((c + base) << 20), the largest code being 1.0.  First moments: 7 bits and a sign, 15 octaves
// under the block's largest; second moments: 8 bits, 31 octaves (the update divides by their root, so they need twice the range).
constexpr uint32_t CODE_ONE = 0x3F8;                    // 1.0f >> 20
constexpr uint32_t BASE_M = CODE_ONE - 127, BASE_V = CODE_ONE - 255;
constexpr uint32_t SMALLEST_TOP = 0x03800000;           // 2^-120: below it the inverse of the scale would overflow

__device__ __forceinline__ float decode_first(uint32_t code, float scale) {      // -0 for code 0x80
  const uint32_t mag = code & 0x7F, bits = mag ? (mag + BASE_M) << 20 : 0u;
  return __fmul_rn(__uint_as_float(bits | ((code << 24) & 0x80000000u)), scale);
}
__device__ __forceinline__ float decode_second(uint32_t code, float scale) {
  return __fmul_rn(__uint_as_float(code ? (code + BASE_V) << 20 : 0u), scale);
}
// inv: 1 / the block's largest magnitude, so that |x| inv is 1 at most, or the number after it.  Rounded to nearest (halves away from
// zero): half a step is put on top of the 20 dropped bits.
__device__ __forceinline__ uint32_t encode_first(float x, float inv) {
  const uint32_t bits = __float_as_uint(__fmul_rn(x, inv));
  return (max(((bits & 0x7FFFFFFFu) + 0x80000u) >> 20, BASE_M) - BASE_M) | ((bits >> 24) & 0x80u);
}
// add: half a step, or random bits below a whole step.  Not 0 for x > 0.
__device__ __forceinline__ uint32_t encode_second(float x, float inv, uint32_t add) {
  const uint32_t q = max((__float_as_uint(__fmul_rn(x, inv)) + add) >> 20, BASE_V + 1u) - BASE_V;
  return x > 0.f ? q : 0u;
}
// 16 random bits of (element, seed) in the upper half of the word: two rounds of multiply and shift, with the 32-bit pair of multipliers and
// shifts that C. Wellons published in "Prospecting for Hash Functions" (2018).
__device__ __forceinline__ uint32_t mix(uint32_t element, uint32_t seed_word) {
  uint32_t w = element * 0x9E3779B1u + seed_word;
  w = (w ^ (w >> 15)) * 0x2C1B3C6Du;
  w = (w ^ (w >> 12)) * 0x297A2D39u;
  return w;
}
// A warp's block of moments to codes and scales.  RANDOM: second moments by random bits, else to nearest.  fp32 magnitudes compare like
// their bits; what is not finite is above all others.
template <bool RANDOM>
__device__ __forceinline__ void encode_block(float (&m)[8], float (&v)[8], int64_t block, uint32_t seed_word, const AdamState& st) {
  constexpr uint32_t NOT_FINITE = 0x7F800000u;
  uint32_t tm = 0, tv = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    tm = max(tm, __float_as_uint(m[k]) & 0x7FFFFFFFu);
    tv = max(tv, __float_as_uint(v[k]));
  }
  tm = __reduce_max_sync(0xFFFFFFFFu, tm);
  tv = __reduce_max_sync(0xFFFFFFFFu, tv);
  if (max(tm, tv) >= NOT_FINITE) {                                      // the whole warp: both moments of such an element are stored as 0
    tm = tv = 0;                                                        // (one without the other is a step of its own size), the rest by the largest
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (max(__float_as_uint(m[k]) & 0x7FFFFFFFu, __float_as_uint(v[k])) >= NOT_FINITE) m[k] = v[k] = 0.f;
      tm = max(tm, __float_as_uint(m[k]) & 0x7FFFFFFFu);
      tv = max(tv, __float_as_uint(v[k]));
    }
    tm = __reduce_max_sync(0xFFFFFFFFu, tm);
    tv = __reduce_max_sync(0xFFFFFFFFu, tv);
  }
  const int64_t at = block * ADAM_BLOCK + lane_id() * 8;
  uint32_t cm[2] = {0, 0}, cv[2] = {0, 0};
  if (tm >= SMALLEST_TOP) {
    const float inv = __frcp_rn(__uint_as_float(tm));
#pragma unroll
    for (int k = 0; k < 8; ++k) cm[k / 4] |= encode_first(m[k], inv) << (8 * (k % 4));
  } else {
    tm = 0;
  }
  if (tv >= SMALLEST_TOP) {
    const float inv = __frcp_rn(__uint_as_float(tv));
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t add = RANDOM ? (mix((uint32_t)at + k, seed_word) >> 12) & 0xFFFF0u : 0x80000u;
      cv[k / 4] |= encode_second(v[k], inv, add) << (8 * (k % 4));
    }
  } else {
    tv = 0;
  }
  *reinterpret_cast<uint2*>(st.m8 + at) = make_uint2(cm[0], cm[1]);
  *reinterpret_cast<uint2*>(st.v8 + at) = make_uint2(cv[0], cv[1]);
  if (lane_id() == 0) {
    st.m_scale[block] = __uint_as_float(tm);
    st.v_scale[block] = __uint_as_float(tv);
  }
}

__device__ __forceinline__ void decode_block(const uint2 cm, const uint2 cv, float sm, float sv, float (&m)[8], float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t a = k < 4 ? cm.x : cm.y, b = k < 4 ? cv.x : cv.y;
    m[k] = decode_first((a >> (8 * (k % 4))) & 0xFF, sm);
    v[k] = decode_second((b >> (8 * (k % 4))) & 0xFF, sv);
  }
}

// ------------------------------------------------------------------------------- the step
// Up to eight elements of a tensor; what is behind its end reads as 0 and is not written.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int count, float (&v)[8]) {
  if (count == 8 && aligned8(p)) {
    load8(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < count ? to_f32(p[k]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, int count, const float (&v)[8]) {
  if (count == 8 && aligned8(p)) {
    store8(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < count) p[k] = from_f32<T>(v[k]);
  }
}

template <typename P, typename G, int BITS>
__global__ void __launch_bounds__(ADAM_WARPS * 32)
adamw_step_kernel(const AdamTensor* __restrict__ tensors, const void* const* __restrict__ grads,
                  const AdamChunk* __restrict__ chunks, AdamState st, AdamConstants c, const float* __restrict__ grad_scale) {
  const AdamChunk ch = chunks[blockIdx.x];
  const AdamTensor t = tensors[ch.tensor];
  const int64_t e = ((int64_t)ch.index * ADAM_WARPS + threadIdx.x / 32) * ADAM_BLOCK + lane_id() * 8;
  if (e - lane_id() * 8 >= t.n) return;                     // the whole warp
  const int count = (int)max((int64_t)0, min((int64_t)8, t.n - e));
  const int64_t at = t.first + e;
  float g[8], p[8], m[8], v[8];
  load_some(static_cast<const G*>(grads[ch.tensor]) + e, count, g);
  P* param = static_cast<P*>(t.param) + e;
  if (t.master) load_some(t.master + e, count, p);
  else load_some(param, count, p);
  if (BITS == 32) {
    load8_f32(st.m32 + at, m);
    load8_f32(st.v32 + at, v);
  } else {
    const int64_t block = at / ADAM_BLOCK;
    decode_block(*reinterpret_cast<const uint2*>(st.m8 + at), *reinterpret_cast<const uint2*>(st.v8 + at),
                 st.m_scale[block], st.v_scale[block], m, v);
  }
  const float scale = grad_scale ? *grad_scale : 1.f;
  const float decay = t.decays ? c.decay : 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    // the moments in separately rounded products and sums: the 8-bit codes then depend on the formula alone and not on
    // which product a compiler contracts
    const float gk = __fmul_rn(g[k], scale);
    m[k] = __fadd_rn(__fmul_rn(m[k], c.beta1), __fmul_rn(gk, c.one_minus_beta1));
    v[k] = __fadd_rn(__fmul_rn(v[k], c.beta2), __fmul_rn(__fmul_rn(gk, gk), c.one_minus_beta2));
    // hardware root and reciprocal: an update's last two units of 2^-23, far below the fp32 parameter's own rounding of the sum
    float root, inv;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v[k]));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(fmaf(root, c.inv_root2, c.eps)));
    p[k] = fmaf(-c.rate, m[k] * inv, fmaf(-decay, p[k], p[k]));
  }
  if (t.master) store_some(t.master + e, count, p);
  store_some(param, count, p);
  if (BITS == 32) {
    store8_f32(st.m32 + at, m);
    store8_f32(st.v32 + at, v);
  } else {
    encode_block<true>(m, v, at / ADAM_BLOCK, c.seed_word, st);
  }
}

// The moments as fp32 arrays, one warp per block.
__global__ void __launch_bounds__(ADAM_WARPS * 32)
adamw_export_kernel(AdamState st, int64_t blocks, float* __restrict__ m_out, float* __restrict__ v_out) {
  const int64_t block = (int64_t)blockIdx.x * ADAM_WARPS + threadIdx.x / 32;
  if (block >= blocks) return;
  const int64_t at = block * ADAM_BLOCK + lane_id() * 8;
  float m[8], v[8];
  decode_block(*reinterpret_cast<const uint2*>(st.m8 + at), *reinterpret_cast<const uint2*>(st.v8 + at),
               st.m_scale[block], st.v_scale[block], m, v);
  store_some(m_out + at, 8, m);
  store_some(v_out + at, 8, v);
}

__global__ void __launch_bounds__(ADAM_WARPS * 32)
adamw_import_kernel(AdamState st, int64_t blocks, const float* __restrict__ m_in, const float* __restrict__ v_in) {
  const int64_t block = (int64_t)blockIdx.x * ADAM_WARPS + threadIdx.x / 32;
  if (block >= blocks) return;
  const int64_t at = block * ADAM_BLOCK + lane_id() * 8;
  float m[8], v[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float4 a = *reinterpret_cast<const float4*>(m_in + at + 4 * h), b = *reinterpret_cast<const float4*>(v_in + at + 4 * h);
    m[4 * h] = a.x; m[4 * h + 1] = a.y; m[4 * h + 2] = a.z; m[4 * h + 3] = a.w;
    v[4 * h] = b.x; v[4 * h + 1] = b.y; v[4 * h + 2] = b.z; v[4 * h + 3] = b.w;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = v[k] <= 0.f ? 0.f : v[k];          // -0 among them: the codes have no sign
  encode_block<false>(m, v, block, 0u, st);
}

}  // namespace mts

struct mts_adamw {
  int32_t n_tensors = 0;
  int32_t param_dtype = 0, grad_dtype = 0, bits = 32;
  int64_t elements = 0;          // P: with every tensor rounded up to whole blocks
  int64_t n_chunks = 0;
  std::vector<int64_t> sizes;
  void* block = nullptr;         // the one device allocation: tensors, gradient pointers, chunks
  mts::AdamTensor* d_tensors = nullptr;
  const void** d_grads = nullptr;
  mts::AdamChunk* d_chunks = nullptr;
};

using namespace mts;

namespace {

size_t state_bytes_of(const mts_adamw* h) {
  if (h->bits == 32) return (size_t)h->elements * 8;
  return (size_t)h->elements * 2 + (size_t)(h->elements / ADAM_BLOCK) * 8;
}

AdamState state_of(const mts_adamw* h, void* state) {
  AdamState st = {};
  const int64_t P = h->elements;
  if (h->bits == 32) {
    st.m32 = static_cast<float*>(state);
    st.v32 = st.m32 + P;
  } else {
    st.m8 = static_cast<uint8_t*>(state);
    st.v8 = st.m8 + P;
    st.m_scale = reinterpret_cast<float*>(st.v8 + P);
    st.v_scale = st.m_scale + P / ADAM_BLOCK;
  }
  return st;
}

int check_state(const char* what, const mts_adamw* h, const void* state, size_t state_bytes) {
  if (!h || (!state && h->elements > 0)) return set_error(MTS_ERR_INVALID_ARG, "%s: null argument", what);
  if ((uintptr_t)state & 255) return set_error(MTS_ERR_ALIGNMENT, "%s: the state must be 256-byte aligned", what);
  if (state_bytes < state_bytes_of(h))
    return set_error(MTS_ERR_WORKSPACE, "%s: the state has %zu bytes, %zu are needed", what, state_bytes, state_bytes_of(h));
  return MTS_OK;
}

int upload(const char* what, void* dst, const void* src, size_t bytes) {
  return bytes ? check_cuda(cudaMemcpy(dst, src, bytes, cudaMemcpyHostToDevice), what) : MTS_OK;
}

}  // namespace

extern "C" int mts_adamw_create(const mts_adamw_desc* d, mts_adamw** out) {
  if (!d || !out) return set_error(MTS_ERR_INVALID_ARG, "adamw_create: null argument");
  *out = nullptr;
  if (d->n_tensors < 1 || !d->host_sizes || !d->host_params || !d->host_grads)
    return set_error(MTS_ERR_INVALID_ARG, "adamw_create: n_tensors = %d, or null sizes/params/grads", d->n_tensors);
  if (!known_dtype(d->param_dtype) || !known_dtype(d->grad_dtype))
    return set_error(MTS_ERR_INVALID_ARG, "adamw_create: param dtype %d, grad dtype %d", d->param_dtype, d->grad_dtype);
  if (d->state_bits != 32 && d->state_bits != 8)
    return set_error(MTS_ERR_INVALID_ARG, "adamw_create: state_bits = %d", d->state_bits);
  const int pb = dtype_bytes(d->param_dtype), gb = dtype_bytes(d->grad_dtype);
  int64_t elements = 0, n_chunks = 0;
  for (int k = 0; k < d->n_tensors; ++k) {
    const int64_t n = d->host_sizes[k];
    if (n < 0) return set_error(MTS_ERR_INVALID_ARG, "adamw_create: tensor %d has %lld elements", k, (long long)n);
    if (n >= (1ll << 40) || elements + ceil_div(n, ADAM_BLOCK) * ADAM_BLOCK >= (1ll << 40))
      return set_error(MTS_ERR_UNSUPPORTED, "adamw_create: 2^40 elements or more");
    if (n > 0 && (!d->host_params[k] || !d->host_grads[k] || (d->host_masters && !d->host_masters[k])))
      return set_error(MTS_ERR_INVALID_ARG, "adamw_create: null pointer of tensor %d", k);
    if (n > 0 && (((uintptr_t)d->host_params[k] % pb) || ((uintptr_t)d->host_grads[k] % gb) ||
                  (d->host_masters && ((uintptr_t)d->host_masters[k] % 4))))
      return set_error(MTS_ERR_ALIGNMENT, "adamw_create: a pointer of tensor %d is no multiple of its element size", k);
    elements += ceil_div(n, ADAM_BLOCK) * ADAM_BLOCK;
    n_chunks += ceil_div(n, ADAM_BLOCK * ADAM_WARPS);
  }
  mts_adamw* h = nullptr;
  try {
    std::vector<AdamTensor> tensors(d->n_tensors);
    std::vector<const void*> grads(d->n_tensors);
    std::vector<AdamChunk> chunks;
    chunks.reserve((size_t)n_chunks);
    int64_t first = 0;
    for (int k = 0; k < d->n_tensors; ++k) {
      const int64_t n = d->host_sizes[k];
      tensors[k] = AdamTensor{d->host_params[k], d->host_masters ? d->host_masters[k] : nullptr, n, first,
                              d->host_decays ? (d->host_decays[k] != 0) : 1};
      grads[k] = d->host_grads[k];
      for (int64_t i = 0; i < ceil_div(n, ADAM_BLOCK * ADAM_WARPS); ++i) chunks.push_back(AdamChunk{k, (int32_t)i});
      first += ceil_div(n, ADAM_BLOCK) * ADAM_BLOCK;
    }
    h = new mts_adamw();
    h->n_tensors = d->n_tensors;
    h->param_dtype = d->param_dtype;
    h->grad_dtype = d->grad_dtype;
    h->bits = d->state_bits;
    h->elements = elements;
    h->n_chunks = n_chunks;
    h->sizes.assign(d->host_sizes, d->host_sizes + d->n_tensors);
    const size_t tb = align_up(sizeof(AdamTensor) * tensors.size(), 256), pbytes = align_up(sizeof(void*) * grads.size(), 256);
    char* blk = nullptr;
    int rc = check_cuda(cudaMalloc(&blk, tb + pbytes + sizeof(AdamChunk) * chunks.size() + 256), "cudaMalloc(adamw)");
    if (rc == MTS_OK) {
      h->block = blk;
      h->d_tensors = reinterpret_cast<AdamTensor*>(blk);
      h->d_grads = reinterpret_cast<const void**>(blk + tb);
      h->d_chunks = reinterpret_cast<AdamChunk*>(blk + tb + pbytes);
      rc = upload("cudaMemcpy(adamw tensors)", h->d_tensors, tensors.data(), sizeof(AdamTensor) * tensors.size());
      if (rc == MTS_OK) rc = upload("cudaMemcpy(adamw gradients)", h->d_grads, grads.data(), sizeof(void*) * grads.size());
      if (rc == MTS_OK) rc = upload("cudaMemcpy(adamw chunks)", h->d_chunks, chunks.data(), sizeof(AdamChunk) * chunks.size());
      // a copy from pageable memory returns once it is staged; streams that do not wait for the default one may run the first step
      if (rc == MTS_OK) rc = check_cuda(cudaStreamSynchronize(cudaStreamLegacy), "cudaStreamSynchronize(adamw)");
    }
    if (rc != MTS_OK) {
      if (h->block) cudaFree(h->block);
      delete h;
      return rc;
    }
  } catch (const std::bad_alloc&) {
    delete h;
    return set_error(MTS_ERR_INVALID_ARG, "adamw_create: out of host memory");
  }
  *out = h;
  return MTS_OK;
}

extern "C" int mts_adamw_destroy(mts_adamw* h) {
  if (!h) return MTS_OK;
  const int rc = h->block ? check_cuda(cudaFree(h->block), "cudaFree(adamw)") : MTS_OK;
  delete h;
  return rc;
}

extern "C" int64_t mts_adamw_state_elements(const mts_adamw* h) { return h ? h->elements : 0; }
extern "C" size_t mts_adamw_state_bytes(const mts_adamw* h) { return h ? state_bytes_of(h) : 0; }

extern "C" int mts_adamw_set_grads(mts_adamw* h, const void* const* host_grads, void* stream) {
  if (!h || !host_grads) return set_error(MTS_ERR_INVALID_ARG, "adamw_set_grads: null argument");
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  const int rc = check_cuda(cudaStreamIsCapturing(static_cast<cudaStream_t>(stream), &capture), "cudaStreamIsCapturing(adamw gradients)");
  if (rc != MTS_OK) return rc;
  // a captured copy would read the caller's array at every replay, long after this call
  if (capture != cudaStreamCaptureStatusNone) return set_error(MTS_ERR_UNSUPPORTED, "adamw_set_grads: the stream is being captured");
  const int gb = dtype_bytes(h->grad_dtype);
  for (int k = 0; k < h->n_tensors; ++k) {
    if (h->sizes[k] > 0 && !host_grads[k]) return set_error(MTS_ERR_INVALID_ARG, "adamw_set_grads: null gradient of tensor %d", k);
    if (h->sizes[k] > 0 && (uintptr_t)host_grads[k] % gb)
      return set_error(MTS_ERR_ALIGNMENT, "adamw_set_grads: gradient %d is no multiple of its element size", k);
  }
  return check_cuda(cudaMemcpyAsync(h->d_grads, host_grads, sizeof(void*) * (size_t)h->n_tensors, cudaMemcpyHostToDevice,
                                    static_cast<cudaStream_t>(stream)), "cudaMemcpyAsync(adamw gradients)");
}

extern "C" int mts_adamw_step(mts_adamw* h, void* state, size_t state_bytes, double lr, double beta1, double beta2, double eps,
                              double weight_decay, int64_t step, const float* grad_scale, uint32_t seed, void* stream) {
  int rc = check_state("adamw_step", h, state, state_bytes);
  if (rc != MTS_OK) return rc;
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !isfinite(lr) ||
      !isfinite(weight_decay) || !isfinite(eps) || step < 1)
    return set_error(MTS_ERR_INVALID_ARG, "adamw_step: lr %g, betas %g %g, eps %g, weight_decay %g, step %lld", lr, beta1, beta2,
                     eps, weight_decay, (long long)step);
  if (h->n_chunks == 0) return MTS_OK;
  AdamConstants c;
  c.beta1 = (float)beta1;
  c.one_minus_beta1 = (float)(1.0 - beta1);
  c.beta2 = (float)beta2;
  c.one_minus_beta2 = (float)(1.0 - beta2);
  c.inv_root2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  c.eps = (float)eps;
  c.rate = (float)(lr / (1.0 - pow(beta1, (double)step)));
  c.decay = (float)(lr * weight_decay);
  c.seed_word = seed * 0x85EBCA77u;
  const AdamState st = state_of(h, state);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_dtype(h->param_dtype, [&](auto p) {
    return with_dtype(h->grad_dtype, [&](auto g) {
      using P = decltype(p);
      using G = decltype(g);
      LaunchScope scope(K_ADAMW, s);
      if (h->bits == 32)
        adamw_step_kernel<P, G, 32><<<(unsigned)h->n_chunks, ADAM_WARPS * 32, 0, s>>>(h->d_tensors, h->d_grads, h->d_chunks, st, c, grad_scale);
      else
        adamw_step_kernel<P, G, 8><<<(unsigned)h->n_chunks, ADAM_WARPS * 32, 0, s>>>(h->d_tensors, h->d_grads, h->d_chunks, st, c, grad_scale);
      return check_launch("adamw_step");
    });
  });
}

extern "C" int mts_adamw_export_state(mts_adamw* h, const void* state, size_t state_bytes, float* m_out, float* v_out, void* stream) {
  int rc = check_state("adamw_export_state", h, state, state_bytes);
  if (rc != MTS_OK) return rc;
  if (h->elements == 0) return MTS_OK;
  if (!m_out || !v_out) return set_error(MTS_ERR_INVALID_ARG, "adamw_export_state: null output");
  if (((uintptr_t)m_out | (uintptr_t)v_out) & 15) return set_error(MTS_ERR_ALIGNMENT, "adamw_export_state: outputs must be 16-byte aligned");
  const AdamState st = state_of(h, const_cast<void*>(state));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (h->bits == 32) {
    rc = check_cuda(cudaMemcpyAsync(m_out, st.m32, (size_t)h->elements * 4, cudaMemcpyDeviceToDevice, s), "cudaMemcpyAsync(adamw m)");
    return rc != MTS_OK ? rc : check_cuda(cudaMemcpyAsync(v_out, st.v32, (size_t)h->elements * 4, cudaMemcpyDeviceToDevice, s), "cudaMemcpyAsync(adamw v)");
  }
  const int64_t blocks = h->elements / ADAM_BLOCK;
  LaunchScope scope(K_ADAMW_STATE, s);
  adamw_export_kernel<<<(unsigned)ceil_div(blocks, ADAM_WARPS), ADAM_WARPS * 32, 0, s>>>(st, blocks, m_out, v_out);
  return check_launch("adamw_export_state");
}

extern "C" int mts_adamw_import_state(mts_adamw* h, void* state, size_t state_bytes, const float* m, const float* v, void* stream) {
  int rc = check_state("adamw_import_state", h, state, state_bytes);
  if (rc != MTS_OK) return rc;
  if (h->elements == 0) return MTS_OK;
  if (!m || !v) return set_error(MTS_ERR_INVALID_ARG, "adamw_import_state: null input");
  if (((uintptr_t)m | (uintptr_t)v) & 15) return set_error(MTS_ERR_ALIGNMENT, "adamw_import_state: inputs must be 16-byte aligned");
  const AdamState st = state_of(h, state);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (h->bits == 32) {
    rc = check_cuda(cudaMemcpyAsync(st.m32, m, (size_t)h->elements * 4, cudaMemcpyDeviceToDevice, s), "cudaMemcpyAsync(adamw m)");
    return rc != MTS_OK ? rc : check_cuda(cudaMemcpyAsync(st.v32, v, (size_t)h->elements * 4, cudaMemcpyDeviceToDevice, s), "cudaMemcpyAsync(adamw v)");
  }
  const int64_t blocks = h->elements / ADAM_BLOCK;
  LaunchScope scope(K_ADAMW_STATE, s);
  adamw_import_kernel<<<(unsigned)ceil_div(blocks, ADAM_WARPS), ADAM_WARPS * 32, 0, s>>>(st, blocks, m, v);
  return check_launch("adamw_import_state");
}
