// Gated linear recurrence over packed ragged sequences, forward and backward:
//
//   z_t = 1 / (1 + exp(-gate_t)),  h_t = h_{t-1} + z_t (value_t - h_{t-1})
//
// A thread walks one channel of one sequence.
#include "dense.cuh"

namespace mts {

constexpr int REC_CHUNK = 64;          // tokens between two kept states
constexpr int REC_STATUS_OFFSETS = 1, REC_STATUS_TIMEOUT = 2;

struct RecArgs {
  const void* gate; int64_t gate_stride;
  const void* value; int64_t value_stride;
  const int64_t* offsets;
  const float* h0;
  int64_t N, S;
  int32_t D;
  int32_t* status;
};

__device__ __forceinline__ float sigmoid_f32(float g) { return __frcp_rn(1.f + __expf(-g)); }

// h + z (x - h) as z x + (1 - z) h without rounding 1 - z: x itself for z = 1, h for z = 0.
__device__ __forceinline__ float blend(float z, float x, float h) { return fmaf(z, x, fmaf(-z, h, h)); }

// Tokens of sequence s, clamped into [0, N).
__device__ __forceinline__ void sequence_range(const RecArgs& a, int64_t s, int64_t& begin, int64_t& end) {
  const int64_t b = a.offsets[s], e = a.offsets[s + 1];
  begin = min(max(b, (int64_t)0), a.N);
  end = min(max(e, begin), a.N);
  if (b != begin || e != end || (s == 0 && b != 0) || (s == a.S - 1 && e != a.N)) atomicOr(a.status, REC_STATUS_OFFSETS);
}

template <typename T>
__global__ void recurrence_forward_serial(RecArgs a, T* __restrict__ out, int64_t out_stride, float* h_final, float* __restrict__ entry) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.S * a.D) return;
  const int64_t s = i / a.D;
  const int d = (int)(i % a.D);
  int64_t begin, end;
  sequence_range(a, s, begin, end);
  float h = a.h0 ? a.h0[i] : 0.f;
  const T* gate = static_cast<const T*>(a.gate);
  const T* value = static_cast<const T*>(a.value);
  for (int64_t t = begin; t < end; ++t) {
    if (entry && t % REC_CHUNK == 0) entry[t / REC_CHUNK * a.D + d] = h;
    const float z = sigmoid_f32(to_f32(gate[t * a.gate_stride + d]));
    h = blend(z, to_f32(value[t * a.value_stride + d]), h);
    out[t * out_stride + d] = from_f32<T>(h);
  }
  if (h_final) h_final[i] = h;
}

template <typename T>
__global__ void recurrence_backward_serial(RecArgs a, const float* __restrict__ entry, const T* __restrict__ grad_out, int64_t grad_out_stride,
                                           const float* __restrict__ grad_final, T* __restrict__ grad_gate, int64_t grad_gate_stride,
                                           T* __restrict__ grad_value, int64_t grad_value_stride, float* __restrict__ grad_h0) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.S * a.D) return;
  const int64_t s = i / a.D;
  const int d = (int)(i % a.D);
  int64_t begin, end;
  sequence_range(a, s, begin, end);
  const T* gate = static_cast<const T*>(a.gate);
  const T* value = static_cast<const T*>(a.value);
  float carry = grad_final ? grad_final[i] : 0.f;        // what reaches h_t from the right
  float before[REC_CHUNK];
  for (int64_t hi = end; hi > begin;) {
    const int64_t lo = max(begin, (hi - 1) / REC_CHUNK * REC_CHUNK);
    float h = lo == begin ? (a.h0 ? a.h0[i] : 0.f) : entry[lo / REC_CHUNK * a.D + d];
    for (int64_t t = lo; t < hi; ++t) {
      before[t - lo] = h;
      h = blend(sigmoid_f32(to_f32(gate[t * a.gate_stride + d])), to_f32(value[t * a.value_stride + d]), h);
    }
    for (int64_t t = hi - 1; t >= lo; --t) {
      const float z = sigmoid_f32(to_f32(gate[t * a.gate_stride + d]));
      const float G = to_f32(grad_out[t * grad_out_stride + d]) + carry;
      grad_value[t * grad_value_stride + d] = from_f32<T>(z * G);
      grad_gate[t * grad_gate_stride + d] = from_f32<T>(z * (1.f - z) * (to_f32(value[t * a.value_stride + d]) - before[t - lo]) * G);
      carry = fmaf(-z, G, G);
    }
    hi = lo;
  }
  if (grad_h0) grad_h0[i] = carry;
}

}  // namespace mts

using namespace mts;

namespace {

int check_sizes(const char* what, int64_t N, int64_t S, int32_t D, int32_t dtype) {
  if (N < 0 || S < 0 || D < 1 || !known_dtype(dtype))
    return set_error(MTS_ERR_INVALID_ARG, "%s: N %lld, S %lld, D %d, dtype %d", what, (long long)N, (long long)S, D, dtype);
  if (N >= (1ll << 31) - (1 << 16) || S >= (1ll << 31) - (1 << 16) || D > (1 << 20))
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

}  // namespace

extern "C" int64_t mts_recurrence_chunks(int64_t N, int32_t D, int32_t dtype) {
  return N < 0 || D < 1 || !known_dtype(dtype) ? 0 : ceil_div(N, REC_CHUNK);
}

extern "C" size_t mts_recurrence_workspace_bytes(int64_t N, int64_t S, int32_t D, int32_t dtype) {
  return N < 0 || S < 0 || D < 1 || !known_dtype(dtype) ? 0 : 256;
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
  if (rc == MTS_OK && S > 0 && !offsets) rc = set_error(MTS_ERR_INVALID_ARG, "%s: null offsets", what);
  if (rc == MTS_OK) rc = check_workspace(what, workspace, workspace_bytes, mts_recurrence_workspace_bytes(N, S, D, dtype));
  if (rc != MTS_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  rc = check_cuda(cudaMemsetAsync(workspace, 0, 256, s), "cudaMemsetAsync(recurrence status)");
  if (rc != MTS_OK || S == 0) return rc;
  const RecArgs a = {gate, gate_stride, value, value_stride, offsets, h0, N, S, D, static_cast<int32_t*>(workspace)};
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    LaunchScope scope(K_RECURRENCE_FWD, s);
    recurrence_forward_serial<T><<<(unsigned)ceil_div(S * D, 128), 128, 0, s>>>(a, static_cast<T*>(out), out_stride, h_final, entry_states);
    return check_launch("recurrence_forward");
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
  if (rc == MTS_OK && ((S > 0 && !offsets) || (N > 0 && !entry_states)))
    rc = set_error(MTS_ERR_INVALID_ARG, "%s: null offsets or entry_states", what);
  if (rc == MTS_OK) rc = check_workspace(what, workspace, workspace_bytes, mts_recurrence_workspace_bytes(N, S, D, dtype));
  if (rc != MTS_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  rc = check_cuda(cudaMemsetAsync(workspace, 0, 256, s), "cudaMemsetAsync(recurrence status)");
  if (rc != MTS_OK || S == 0) return rc;
  const RecArgs a = {gate, gate_stride, value, value_stride, offsets, h0, N, S, D, static_cast<int32_t*>(workspace)};
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    LaunchScope scope(K_RECURRENCE_BWD, s);
    recurrence_backward_serial<T><<<(unsigned)ceil_div(S * D, 128), 128, 0, s>>>(
        a, entry_states, static_cast<const T*>(grad_out), grad_out_stride, grad_final, static_cast<T*>(grad_gate), grad_gate_stride,
        static_cast<T*>(grad_value), grad_value_stride, grad_h0);
    return check_launch("recurrence_backward");
  });
}

extern "C" int mts_recurrence_status(const void* workspace, int32_t* host_status, void* stream) {
  if (!workspace || !host_status) return set_error(MTS_ERR_INVALID_ARG, "recurrence_status: null argument");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int rc = check_cuda(cudaMemcpyAsync(host_status, workspace, sizeof(int32_t), cudaMemcpyDeviceToHost, s), "cudaMemcpyAsync(status)");
  if (rc == MTS_OK) rc = check_cuda(cudaStreamSynchronize(s), "cudaStreamSynchronize(status)");
  if (rc == MTS_OK && (*host_status & REC_STATUS_TIMEOUT))
    rc = set_error(MTS_ERR_TIMEOUT, "recurrence: a bounded wait ran out, the results of the last call are incomplete");
  return rc;
}
