// A product of rows with a weight matrix and its epilogue:
//   out = residual + act(x W^T [* x_scales w_scales] + bias) * sigma(gate)
//
// Tiles of 64 x 64 outputs on the CUDA cores, 16 channels at a time through shared memory.
#include "seq_ops.cuh"

#include <cuda_fp8.h>

namespace {
using namespace seqops;

constexpr int MAX_INNER = 1 << 14, MAX_OUTER = 1 << 16;
constexpr int TM = 64, TN = 64, TK = 16;

struct PrArgs {
  const void *x, *w, *gate, *res;
  void* out;
  int64_t xs, ws, gs, rs, os;
  const float *x_scales, *w_scales, *bias;
  int64_t n;
  int K, M, act;
};

template <class T>
__device__ __forceinline__ float operand(T x) { return to_float(x); }
__device__ __forceinline__ float operand(__nv_fp8_e4m3 x) { return (float)x; }
__device__ __forceinline__ float sigma(float x) { return 1.0f / (1.0f + expf(-x)); }
__device__ __forceinline__ float activate(float y, int act) {
  switch (act) {
    case TRACKFIT_ACT_RELU: return y < 0.0f ? 0.0f : y;
    case TRACKFIT_ACT_SILU: return y * sigma(y);
    case TRACKFIT_ACT_GELU: return 0.5f * y * erfcf(y * -0.70710678118654752f);
    default: return y;
  }
}

template <class T, class O>
__global__ void __launch_bounds__(256) product_kernel(const PrArgs a) {
  __shared__ float xs[TK][TM + 1], ws[TK][TN + 1];
  const int64_t r0 = (int64_t)blockIdx.x * TM;
  const int c0 = blockIdx.y * TN, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < a.K; k0 += TK) {
    for (int i = threadIdx.x; i < TM * TK; i += 256) {
      const int r = i / TK, k = i % TK;
      xs[k][r] = r0 + r < a.n && k0 + k < a.K ? operand(((const O*)a.x)[(r0 + r) * a.xs + k0 + k]) : 0.0f;
      ws[k][r] = c0 + r < a.M && k0 + k < a.K ? operand(((const O*)a.w)[(int64_t)(c0 + r) * a.ws + k0 + k]) : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < TK; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[k][ty * 4 + i], ws[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + ty * 4 + i;
      const int c = c0 + tx * 4 + j;
      if (r >= a.n || c >= a.M) continue;
      float y = acc[i][j];
      if (a.x_scales) y *= a.x_scales[r] * a.w_scales[c];
      if (a.bias) y += a.bias[c];
      y = activate(y, a.act);
      if (a.gate) y *= sigma(to_float(((const T*)a.gate)[r * a.gs + c]));
      if (a.res) y += to_float(((const T*)a.res)[r * a.rs + c]);
      put((T*)a.out + r * a.os + c, y);
    }
}

template <class T>
void launch(const PrArgs& a, bool eight, dim3 grid, cudaStream_t st) {
  if (eight) product_kernel<T, __nv_fp8_e4m3><<<grid, 256, 0, st>>>(a);
  else product_kernel<T, T><<<grid, 256, 0, st>>>(a);
}

}  // namespace

extern "C" int trackfit_product(int32_t dtype, int32_t operand_type, const void* x, int64_t x_stride,
                                const float* x_scales, const void* weight, int64_t weight_stride,
                                const float* weight_scales, int64_t n_rows, int32_t in_dim, int32_t out_dim,
                                const float* bias, int32_t activation, const void* gate, int64_t gate_stride,
                                const void* residual, int64_t residual_stride, void* out, int64_t out_stride,
                                void* stream) {
  tf_nvtx_range nvtx_range("trackfit_product");
  const bool eight = operand_type == TRACKFIT_E4M3;
  if (!type_ok(dtype) || (operand_type != dtype && !eight) || n_rows < 0 || n_rows > (int64_t)1 << 40)
    return TRACKFIT_ERR_INVALID_ARG;
  if (in_dim < 8 || in_dim > MAX_INNER || in_dim % (eight ? 16 : 8) != 0 || out_dim < 8 || out_dim > MAX_OUTER || out_dim % 8 != 0)
    return TRACKFIT_ERR_UNSUPPORTED;
  if (activation < TRACKFIT_ACT_NONE || activation > TRACKFIT_ACT_GELU) return TRACKFIT_ERR_INVALID_ARG;
  if (n_rows == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype), osz = eight ? 1 : sz;
  if (!rows_ok(x, x_stride, in_dim, osz) || !rows_ok(weight, weight_stride, in_dim, osz) ||
      !rows_ok(out, out_stride, out_dim, sz) || (gate && !rows_ok(gate, gate_stride, out_dim, sz)) ||
      (residual && !rows_ok(residual, residual_stride, out_dim, sz)))
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(bias) || mis4(x_scales) || mis4(weight_scales) || (eight != (x_scales != nullptr)) || (eight != (weight_scales != nullptr)))
    return TRACKFIT_ERR_INVALID_ARG;
  PrArgs a;
  a.x = x, a.xs = x_stride, a.w = weight, a.ws = weight_stride, a.gate = gate, a.gs = gate_stride;
  a.res = residual, a.rs = residual_stride, a.out = out, a.os = out_stride;
  a.x_scales = x_scales, a.w_scales = weight_scales, a.bias = bias;
  a.n = n_rows, a.K = in_dim, a.M = out_dim, a.act = activation;
  const int64_t tiles = (n_rows + TM - 1) / TM;
  const int cols = (out_dim + TN - 1) / TN;
  if (tiles > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)tiles, (unsigned)cols);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) launch<float>(a, eight, grid, st);
  else if (dtype == TRACKFIT_BF16_PROJ) launch<__nv_bfloat16>(a, eight, grid, st);
  else launch<__half>(a, eight, grid, st);
  return launched();
}
