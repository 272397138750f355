// Root-mean-square norm of rows, with the addition of a branch's output in the same pass and an
// output of the rows' type or in e4m3 with a scale a row.
//
//   s = x + delta,  y = s / sqrt(mean(s^2) + eps) * gain
//   8 bits: scale = max(max|y| / 448, 2^-100), q = e4m3(y / scale)
//
// A warp takes a row; the sum s, in fp32 and not rounded, is formed again in each of the passes.
#include "seq_ops.cuh"

#include <cuda_fp8.h>

namespace {
using namespace seqops;

constexpr int WARPS = 4;
constexpr int MAX_CHANNELS = 1 << 14;
constexpr float LARGEST = 448.0f;          // of e4m3
constexpr float LEAST_SCALE = 0x1p-100f;   // of a row, so that its inverse is finite

struct NormArgs {
  const void *x, *delta;
  void *sum, *out;
  int64_t xs, ds, ss, os;
  int64_t n;
  int C;
  float eps;
  const float* gain;
  float* scales;
};

template <class T, bool EIGHT>
__global__ void __launch_bounds__(WARPS * 32) norm_kernel(const NormArgs a) {
  const int64_t r = (int64_t)blockIdx.x * WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  if (r >= a.n) return;
  const T *x = (const T*)a.x + r * a.xs, *d = a.delta ? (const T*)a.delta + r * a.ds : nullptr;
  auto value = [&](int c) { return d ? to_float(x[c]) + to_float(d[c]) : to_float(x[c]); };
  float ss = 0.0f;
  for (int c = lane; c < a.C; c += 32) ss = fmaf(value(c), value(c), ss);
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(FULL, ss, o);
  const float inv = rsqrtf(ss / (float)a.C + a.eps);
  float scale = 1.0f;
  if constexpr (EIGHT) {
    float m = 0.0f;
    for (int c = lane; c < a.C; c += 32) m = fmaxf(m, fabsf(value(c) * inv * (a.gain ? a.gain[c] : 1.0f)));
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, o));
    scale = fmaxf(m / LARGEST, LEAST_SCALE);
    if (lane == 0) a.scales[r] = scale;
  }
  for (int c = lane; c < a.C; c += 32) {
    const float s = value(c), y = s * inv * (a.gain ? a.gain[c] : 1.0f);
    if constexpr (EIGHT)
      ((__nv_fp8_storage_t*)a.out)[r * a.os + c] = __nv_cvt_float_to_fp8(y / scale, __NV_SATFINITE, __NV_E4M3);
    else
      put((T*)a.out + r * a.os + c, y);
    if (a.sum) put((T*)a.sum + r * a.ss + c, s);
  }
}

template <class T>
void launch(const NormArgs& a, bool eight, cudaStream_t st) {
  const unsigned grid = (unsigned)((a.n + WARPS - 1) / WARPS);
  if (eight) norm_kernel<T, true><<<grid, WARPS * 32, 0, st>>>(a);
  else norm_kernel<T, false><<<grid, WARPS * 32, 0, st>>>(a);
}

}  // namespace

extern "C" int trackfit_add_norm(int32_t dtype, const void* x, int64_t x_stride, const void* delta,
                                 int64_t delta_stride, int64_t n_rows, int32_t channels, const float* gain, float eps,
                                 void* sum_out, int64_t sum_stride, int32_t out_type, void* out, int64_t out_stride,
                                 float* scales, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_add_norm");
  const bool eight = out_type == TRACKFIT_E4M3;
  if (!type_ok(dtype) || (out_type != dtype && !eight) || n_rows < 0 || n_rows > (int64_t)1 << 40)
    return TRACKFIT_ERR_INVALID_ARG;
  if (channels < 8 || channels > MAX_CHANNELS || channels % (eight ? 16 : 8) != 0) return TRACKFIT_ERR_UNSUPPORTED;
  if (!(eps > 0.0f) || !isfinite(eps)) return TRACKFIT_ERR_INVALID_ARG;
  if (n_rows == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!rows_ok(x, x_stride, channels, sz) || (delta && !rows_ok(delta, delta_stride, channels, sz)) ||
      (sum_out && !rows_ok(sum_out, sum_stride, channels, sz)) || !rows_ok(out, out_stride, channels, eight ? 1 : sz))
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(gain) || mis4(scales) || (eight != (scales != nullptr))) return TRACKFIT_ERR_INVALID_ARG;
  if ((n_rows + WARPS - 1) / WARPS > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  NormArgs a;
  a.x = x, a.xs = x_stride, a.delta = delta, a.ds = delta_stride, a.sum = sum_out, a.ss = sum_stride;
  a.out = out, a.os = out_stride, a.n = n_rows, a.C = channels, a.eps = eps, a.gain = gain, a.scales = scales;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) launch<float>(a, eight, st);
  else if (dtype == TRACKFIT_BF16_PROJ) launch<__nv_bfloat16>(a, eight, st);
  else launch<__half>(a, eight, st);
  return launched();
}
