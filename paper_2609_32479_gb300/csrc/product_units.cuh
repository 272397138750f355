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

// sigma(x) by the hardware's 2^x and reciprocal: a few units in fp32's last place, (2 |x| + 10) 2^-24 in all
// (the product with log2 e is rounded once).  2^x = inf gives 0.
__device__ __forceinline__ float sigma(float x) { return rcp(1.0f + ex2(-LOG2E * x)); }

// y Phi(y).  Of the normal distribution's smaller tail, erfc(x) / 2 with x = |y| / sqrt 2, not of
// 1 + erf, which below -3 would leave few bits: erfc(x) = t 2^(-x^2 log2 e + P(t)) with t = 1 / (1 + x / 2),
// the form of Press et al., Numerical Recipes; P, of degree 9, is a least-squares fit of
// log2(exp(x^2) erfc(x) / 2 t) over y in [0, 14] with weights moved to where it was off most: by 7e-8.
// In fp32 the tail is off by (8 + 2 y^2) 2^-24 of itself at most (y^2 for the exponent's rounding).
__device__ __forceinline__ float gelu(float y) {
  const float t = rcp(fmaf(fabsf(y), 0.35355339f, 1.0f));
  float p = 0.204026341f;
  p = fmaf(p, t, -0.954790890f);
  p = fmaf(p, t, 1.60470486f);
  p = fmaf(p, t, -0.919945478f);
  p = fmaf(p, t, -0.184892729f);
  p = fmaf(p, t, 0.0379605107f);
  p = fmaf(p, t, 0.0378692932f);
  p = fmaf(p, t, 0.560266495f);
  p = fmaf(p, t, 1.44044387f);
  p = fmaf(p, t, -2.82564235f);
  const float tail = t * ex2(fmaf(y * y, -0.5f * LOG2E, p));
  return y * (y < 0.0f ? tail : 1.0f - tail);
}

// fp32 vectors of a value an output, four at a time where their alignment lets them (a multiple of 4
// outputs from the first).
__device__ __forceinline__ float4 four(const float* p, bool aligned) {
  if (aligned) return __ldg(reinterpret_cast<const float4*>(p));
  return make_float4(__ldg(p), __ldg(p + 1), __ldg(p + 2), __ldg(p + 3));
}
__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// N sums of a row, from output `col` on (all of them outputs): scaled, with the bias, activated.
template <bool EIGHT, int N>
__device__ __forceinline__ void activated(const ProductArgs& a, float (&y)[N], float x_scale, int col) {
  if constexpr (EIGHT) {
    const bool al = aligned16(a.w_scales);
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 w = four(a.w_scales + col + i, al);
      y[i] *= x_scale * w.x, y[i + 1] *= x_scale * w.y, y[i + 2] *= x_scale * w.z, y[i + 3] *= x_scale * w.w;
    }
  }
  if (a.bias) {
    const bool al = aligned16(a.bias);
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 b = four(a.bias + col + i, al);
      y[i] += b.x, y[i + 1] += b.y, y[i + 2] += b.z, y[i + 3] += b.w;
    }
  }
  switch (a.act) {
    case TRACKFIT_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = y[i] < 0.0f ? 0.0f : y[i];
      break;
    case TRACKFIT_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] *= sigma(y[i]);
      break;
    case TRACKFIT_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = gelu(y[i]);
      break;
    default: break;
  }
}
// VE activated values times sigma(gate), onto the residual, 16 bytes of each.
template <class T, int VE>
__device__ __forceinline__ void gated(const ProductArgs& a, float (&y)[VE], const uint4& g, const uint4& x) {
  static_assert(VE * sizeof(T) == 16, "16 bytes of outputs");
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
template <class T, bool EIGHT, int VE>
__device__ __forceinline__ void finish(const ProductArgs& a, float (&y)[VE], float x_scale, int col, const uint4& g,
                                       const uint4& x) {
  activated<EIGHT>(a, y, x_scale, col);
  gated<T>(a, y, g, x);
}

// product_tc.cu: 16-bit and 8-bit operands by the tensor cores, many rows.
int product_tc(int32_t dtype, const ProductArgs& a, cudaStream_t st);
// product_few.cu: few rows, where the weights are what is read (24 rows through 4096 x 4096 in bf16: 25 us
// there, 19 by the tiles; 16: 21 and 19, but 9.0 and 10.9 through 1024 x 1024, 6.8 and 10.9 from 128 to 768).
constexpr int PRODUCT_FEW = 16;
int product_few(int32_t dtype, const ProductArgs& a, cudaStream_t st);

}  // namespace seqops
