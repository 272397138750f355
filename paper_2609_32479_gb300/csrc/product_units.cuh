// Rows times a weight matrix with its epilogue: arguments, and what a sum goes through.
#pragma once

#include "seq_ops.cuh"

#include <cuda_fp8.h>

namespace seqops {

struct ProductArgs {
  const void *x, *w, *gate, *res;
  void* out;
  int64_t xs, ws, gs, rs, os;                  // row strides in elements
  const float *x_scales, *w_scales, *bias;
  int64_t n;
  int K, M, act;
};

// sigma(x) by the hardware's 2^x and division: a few units in fp32's last place, (2 |x| + 10) 2^-24 in all
// (the product with log2 e is rounded once).  2^x = inf gives 0.
__device__ __forceinline__ float sigma(float x) { return __fdividef(1.0f, 1.0f + ex2(-LOG2E * x)); }

// Half of erfc, not of 1 + erf, which below -3 would leave few bits.
__device__ __forceinline__ float gelu(float y) { return 0.5f * y * erfcf(y * -0.70710678118654752f); }

// VE sums of a row, from output `col` on: scaled, with the bias, activated, gated and added to the
// residual; gate and residual 16 bytes each.
template <class T, bool EIGHT, int VE>
__device__ __forceinline__ void finish(const ProductArgs& a, float (&y)[VE], float x_scale, int col, const uint4& g,
                                       const uint4& x) {
  static_assert(VE * sizeof(T) == 16, "16 bytes of outputs");
#pragma unroll
  for (int i = 0; i < VE; i += 4) {
    if constexpr (EIGHT) {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[i + e] *= x_scale * __ldg(a.w_scales + col + i + e);
    }
    if (a.bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[i + e] += __ldg(a.bias + col + i + e);
    }
  }
  switch (a.act) {
    case TRACKFIT_ACT_RELU:
#pragma unroll
      for (int i = 0; i < VE; ++i) y[i] = y[i] < 0.0f ? 0.0f : y[i];
      break;
    case TRACKFIT_ACT_SILU:
#pragma unroll
      for (int i = 0; i < VE; ++i) y[i] *= sigma(y[i]);
      break;
    case TRACKFIT_ACT_GELU:
#pragma unroll
      for (int i = 0; i < VE; ++i) y[i] = gelu(y[i]);
      break;
    default: break;
  }
  float v[VE];
  if (a.gate) {
    unpack(g, v, T());
#pragma unroll
    for (int i = 0; i < VE; ++i) y[i] *= sigma(v[i]);
  }
  if (a.res) {
    unpack(x, v, T());
#pragma unroll
    for (int i = 0; i < VE; ++i) y[i] += v[i];
  }
}

// product_tc.cu: 16-bit and 8-bit operands by the tensor cores, many rows.
int product_tc(int32_t dtype, const ProductArgs& a, cudaStream_t st);
// product_few.cu: few rows, where the weights are what is read.
constexpr int PRODUCT_FEW = 16;
int product_few(int32_t dtype, const ProductArgs& a, cudaStream_t st);

}  // namespace seqops
