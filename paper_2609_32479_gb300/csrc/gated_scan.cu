// The gated recurrence over packed sequences: forward, backward, one row a sequence.
//
//   z = 1 / (1 + e^-p),  h_t = h_{t-1} + z_t (n_t - h_{t-1}), as (1 - z) h + z n
//   backward, from the last row of the direction to the first, with g the gradient of h:
//   D_t = g_t + (1 - z_{t+1}) D_{t+1},  dn = z D,  dp = z (1 - z) (n - h_{t-1}) D
//
// One thread a sequence and channel, a row after the other.
#include "seq_ops.cuh"

namespace {
using namespace seqops;

constexpr int SAVED = 128;                 // rows from one saved state to the next
constexpr int MAX_CHANNELS = 1 << 16;
constexpr int NT = 128;

struct GsArgs {
  const void *p, *n, *g;
  void *out, *dp, *dn;
  int64_t ps, ns, gs, os, dps, dns;        // row strides in elements
  const int64_t* offs;
  int64_t n_rows, n_seq;
  int C, reverse;
  const float *state_in, *d_state_out;
  float *state_out, *d_state_in;
  float* saved;                            // [(n_rows + 127) / 128][C]: the state before rows 0, 128, .. of the direction
};

__device__ __forceinline__ float gate(float p) { return 1.0f / (1.0f + expf(-p)); }

template <class T>
__global__ void __launch_bounds__(NT) scan_kernel(const GsArgs a) {
  const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x, b = i / a.C;
  const int c = (int)(i % a.C);
  if (b >= a.n_seq) return;
  const int64_t lo = clamp64(a.offs[b], 0, a.n_rows), hi = clamp64(a.offs[b + 1], lo, a.n_rows);
  float h = a.state_in ? a.state_in[i] : 0.0f;
  for (int64_t t = lo; t < hi; ++t) {
    const int64_t row = a.reverse ? lo + hi - 1 - t : t, pos = a.reverse ? a.n_rows - 1 - row : row;
    if (a.saved && pos % SAVED == 0) a.saved[pos / SAVED * a.C + c] = h;
    const float p = to_float(((const T*)a.p)[row * a.ps + c]);
    h = fmaf(gate(-p), h, gate(p) * to_float(((const T*)a.n)[row * a.ns + c]));
    put((T*)a.out + row * a.os + c, h);
  }
  if (a.state_out) a.state_out[i] = h;
}

template <class T>
__global__ void __launch_bounds__(NT) backward_kernel(const GsArgs a) {
  const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x, b = i / a.C;
  const int c = (int)(i % a.C);
  if (b >= a.n_seq) return;
  const int64_t lo = clamp64(a.offs[b], 0, a.n_rows), hi = clamp64(a.offs[b + 1], lo, a.n_rows);
  float d = a.d_state_out ? a.d_state_out[i] : 0.0f;
  // positions of the direction; the states of a run between two saved ones are formed again for each row
  const int64_t first = a.reverse ? a.n_rows - hi : lo, last = a.reverse ? a.n_rows - lo : hi;
  for (int64_t t = last - 1; t >= first; --t) {
    int64_t s = t / SAVED * SAVED;
    float h;
    if (s > first) h = a.saved[s / SAVED * a.C + c];
    else s = first, h = a.state_in ? a.state_in[i] : 0.0f;
    for (; s < t; ++s) {
      const int64_t row = a.reverse ? a.n_rows - 1 - s : s;
      const float p = to_float(((const T*)a.p)[row * a.ps + c]);
      h = fmaf(gate(-p), h, gate(p) * to_float(((const T*)a.n)[row * a.ns + c]));
    }
    const int64_t row = a.reverse ? a.n_rows - 1 - t : t;
    const float p = to_float(((const T*)a.p)[row * a.ps + c]), z = gate(p), w = gate(-p);
    d += to_float(((const T*)a.g)[row * a.gs + c]);
    put((T*)a.dn + row * a.dns + c, z * d);
    put((T*)a.dp + row * a.dps + c, z * w * (to_float(((const T*)a.n)[row * a.ns + c]) - h) * d);
    d *= w;
  }
  if (a.d_state_in) a.d_state_in[i] = d;
}

struct StepArgs {
  const void *p, *n;
  void* out;
  int64_t ps, ns, os;
  const int32_t* slots;
  const float* state_in;
  float* state_out;
  int64_t n_seq, n_slots;
  int C;
};

template <class T>
__global__ void __launch_bounds__(NT) step_kernel(const StepArgs a) {
  const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x, b = i / a.C;
  const int c = (int)(i % a.C);
  if (b >= a.n_seq) return;
  T* out = (T*)a.out + b * a.os + c;
  const int64_t slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    put(out, __uint_as_float(0x7fffffffu));
    return;
  }
  float h = a.state_in[slot * a.C + c];
  const float p = to_float(((const T*)a.p)[b * a.ps + c]);
  h = fmaf(gate(-p), h, gate(p) * to_float(((const T*)a.n)[b * a.ns + c]));
  a.state_out[slot * a.C + c] = h;
  put(out, h);
}

bool channels_ok(int32_t c) { return c >= 8 && c <= MAX_CHANNELS && c % 8 == 0; }

// The checks that forward and backward share; OK with *nothing set where there is no sequence.
int check(int32_t dtype, const GsArgs& a) {
  if (!type_ok(dtype) || a.n_rows < 0 || a.n_rows > (int64_t)1 << 40 || a.n_seq < 0 || a.n_seq > 0x7fffffff)
    return TRACKFIT_ERR_INVALID_ARG;
  if (!channels_ok(a.C)) return TRACKFIT_ERR_UNSUPPORTED;
  if (a.reverse != 0 && a.reverse != 1) return TRACKFIT_ERR_INVALID_ARG;
  if (a.n_seq == 0) return TRACKFIT_OK;
  if (!a.offs || (reinterpret_cast<uintptr_t>(a.offs) & 7u)) return TRACKFIT_ERR_INVALID_ARG;
  if (mis16(a.state_in) || mis16(a.state_out) || mis16(a.d_state_in) || mis16(a.d_state_out) || mis16(a.saved))
    return TRACKFIT_ERR_INVALID_ARG;
  const int sz = type_size(dtype);
  if (a.n_rows > 0 && (!rows_ok(a.p, a.ps, a.C, sz) || !rows_ok(a.n, a.ns, a.C, sz))) return TRACKFIT_ERR_INVALID_ARG;
  if ((a.n_seq * a.C + NT - 1) / NT > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  return TRACKFIT_OK;
}

}  // namespace

extern "C" size_t trackfit_gated_scan_saved(int64_t n_rows, int32_t channels) {
  if (n_rows < 0 || n_rows > (int64_t)1 << 40 || !channels_ok(channels)) return 0;
  return (size_t)((n_rows + SAVED - 1) / SAVED) * channels * 4;
}

extern "C" size_t trackfit_gated_scan_workspace(int32_t, int64_t, int64_t, int32_t) { return 0; }

extern "C" int trackfit_gated_scan(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                   int64_t cand_stride, int64_t n_rows, const int64_t* offsets, int64_t n_seq,
                                   int32_t channels, int32_t reverse, const float* state_in, float* state_out,
                                   float* saved, void* out, int64_t out_stride, void* workspace, size_t,
                                   void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan");
  GsArgs a = {};
  a.p = gate, a.ps = gate_stride, a.n = cand, a.ns = cand_stride, a.out = out, a.os = out_stride;
  a.offs = offsets, a.n_rows = n_rows, a.n_seq = n_seq, a.C = channels, a.reverse = reverse;
  a.state_in = state_in, a.state_out = state_out, a.saved = saved;
  if (mis16(workspace)) return TRACKFIT_ERR_INVALID_ARG;
  const int rc = check(dtype, a);
  if (rc != TRACKFIT_OK || n_seq == 0) return rc;
  if (n_rows > 0 && !rows_ok(out, out_stride, channels, type_size(dtype))) return TRACKFIT_ERR_INVALID_ARG;
  const unsigned grid = (unsigned)((n_seq * channels + NT - 1) / NT);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) scan_kernel<float><<<grid, NT, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) scan_kernel<__nv_bfloat16><<<grid, NT, 0, st>>>(a);
  else scan_kernel<__half><<<grid, NT, 0, st>>>(a);
  return launched();
}

extern "C" int trackfit_gated_scan_backward(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                            int64_t cand_stride, int64_t n_rows, const int64_t* offsets,
                                            int64_t n_seq, int32_t channels, int32_t reverse, const float* state_in,
                                            const float* saved, const void* d_out, int64_t d_out_stride,
                                            const float* d_state_out, float* d_state_in, void* d_gate,
                                            int64_t d_gate_stride, void* d_cand, int64_t d_cand_stride, void* workspace,
                                            size_t, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan_backward");
  GsArgs a = {};
  a.p = gate, a.ps = gate_stride, a.n = cand, a.ns = cand_stride, a.g = d_out, a.gs = d_out_stride;
  a.dp = d_gate, a.dps = d_gate_stride, a.dn = d_cand, a.dns = d_cand_stride;
  a.offs = offsets, a.n_rows = n_rows, a.n_seq = n_seq, a.C = channels, a.reverse = reverse;
  a.state_in = state_in, a.saved = const_cast<float*>(saved), a.d_state_out = d_state_out, a.d_state_in = d_state_in;
  if (mis16(workspace)) return TRACKFIT_ERR_INVALID_ARG;
  const int rc = check(dtype, a);
  if (rc != TRACKFIT_OK || n_seq == 0) return rc;
  const int sz = type_size(dtype);
  if (n_rows > 0 && (!saved || !rows_ok(d_out, d_out_stride, channels, sz) || !rows_ok(d_gate, d_gate_stride, channels, sz) ||
                     !rows_ok(d_cand, d_cand_stride, channels, sz)))
    return TRACKFIT_ERR_INVALID_ARG;
  const unsigned grid = (unsigned)((n_seq * channels + NT - 1) / NT);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) backward_kernel<float><<<grid, NT, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) backward_kernel<__nv_bfloat16><<<grid, NT, 0, st>>>(a);
  else backward_kernel<__half><<<grid, NT, 0, st>>>(a);
  return launched();
}

extern "C" int trackfit_gated_scan_step(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                        int64_t cand_stride, int64_t n_seq, int32_t channels, const int32_t* slots,
                                        int64_t n_slots, const float* state_in, float* state_out, void* out,
                                        int64_t out_stride, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan_step");
  if (!type_ok(dtype) || n_seq < 0 || n_seq > 0x7fffffff || n_slots < 0) return TRACKFIT_ERR_INVALID_ARG;
  if (!channels_ok(channels)) return TRACKFIT_ERR_UNSUPPORTED;
  if (!slots && n_slots < n_seq) return TRACKFIT_ERR_INVALID_ARG;
  if (n_seq == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!rows_ok(gate, gate_stride, channels, sz) || !rows_ok(cand, cand_stride, channels, sz) ||
      !rows_ok(out, out_stride, channels, sz))
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(slots) || !state_in || !state_out || mis16(state_in) || mis16(state_out)) return TRACKFIT_ERR_INVALID_ARG;
  StepArgs a;
  a.p = gate, a.ps = gate_stride, a.n = cand, a.ns = cand_stride, a.out = out, a.os = out_stride;
  a.slots = slots, a.state_in = state_in, a.state_out = state_out, a.n_seq = n_seq, a.n_slots = n_slots, a.C = channels;
  if ((n_seq * channels + NT - 1) / NT > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((n_seq * channels + NT - 1) / NT);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) step_kernel<float><<<grid, NT, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) step_kernel<__nv_bfloat16><<<grid, NT, 0, st>>>(a);
  else step_kernel<__half><<<grid, NT, 0, st>>>(a);
  return launched();
}
