// Root-mean-square norm of rows, with the addition of a branch's output in the same pass and an
// output of the rows' type or in e4m3 with a scale a row.
//
//   s = x + delta,  y = s / sqrt(mean(s^2) + eps) * gain
//   8 bits: scale = max(max|y| / 448, 2^-100), q = e4m3(y / scale)
//
// A pass over memory, which bounds it: each value is read once and written once.  G threads hold a
// row, V pieces of 16 bytes each, s in fp32 as it was added up; the sum of squares and the largest
// |y| go through the G threads (a part of a warp, or two to eight warps through shared memory).  Narrow
// rows: a few rows' loads are under way together.
//
// Measured: 1,835,003 rows of 256 in bf16, with the sum, into 8 bits: 520 us, 6.3 TB/s of the 6.8 that a
// copy moves; 100,000 rows of 2,048 in fp32 488 us, 6.7; rows of 1,104 into 8 bits 2.9 TB/s (two warps a row
// with 138 pieces for 256 places).
#include "seq_ops.cuh"

#include <cuda_fp8.h>

namespace {
using namespace seqops;

constexpr int NT = 256;
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

__device__ __forceinline__ uint16_t eight2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
// y as 8-bit values, nearest, ties to even (they are within 448 but for a rounding).
__device__ __forceinline__ void put8(uint8_t* p, const float (&y)[8]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(eight2(y[0], y[1]) | (uint32_t)eight2(y[2], y[3]) << 16,
                                            eight2(y[4], y[5]) | (uint32_t)eight2(y[6], y[7]) << 16);
}
__device__ __forceinline__ void put8(uint8_t* p, const float (&y)[4]) {
  *reinterpret_cast<uint32_t*>(p) = eight2(y[0], y[1]) | (uint32_t)eight2(y[2], y[3]) << 16;
}

// Over the G threads of a row; `at` is a place in shared memory of this row's own (eight warps).
template <int G, bool MAX>
__device__ __forceinline__ float over_row(float v, float* at) {
#pragma unroll
  for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(FULL, v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  if constexpr (G > 32) {
    if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int i = 1; i < G / 32; ++i) v = MAX ? fmaxf(v, at[i]) : v + at[i];
  }
  return v;
}

// (rows that a part of a warp holds: CTAs of 256 threads; wider ones: a CTA a row)
__host__ __device__ constexpr int threads_of(int G) { return G > 32 ? G : NT; }

template <class T, bool EIGHT, int G, int V, int ROWS>
__global__ void __launch_bounds__(threads_of(G)) norm_kernel(const NormArgs a) {
  constexpr int VE = 16 / sizeof(T), GROUPS = threads_of(G) / G;
  static_assert(G <= 32 || ROWS == 1, "the warps of a CTA take one row at a time");
  __shared__ float part[2][2][NT / 32];
  const int e = threadIdx.x % G;
  const float inv_c = 1.0f / (float)a.C;
  const bool wide_gain = (reinterpret_cast<uintptr_t>(a.gain) & 15u) == 0;
  auto gains = [&](int c, float (&g)[VE]) {
#pragma unroll
    for (int i = 0; i < VE; i += 4)
      if (!a.gain) {
        g[i] = g[i + 1] = g[i + 2] = g[i + 3] = 1.0f;
      } else if (wide_gain) {
        *reinterpret_cast<float4*>(&g[i]) = __ldg(reinterpret_cast<const float4*>(a.gain + c + i));
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) g[i + k] = __ldg(a.gain + c + i + k);
      }
  };
  // one piece a thread: its gains stay in registers
  float kept[V == 1 ? VE : 1];
  if constexpr (V == 1) {
#pragma unroll
    for (int i = 0; i < VE; ++i) kept[i] = 1.0f;
    if (e * VE < a.C) gains(e * VE, kept);
  }
  int turn = 0;
  const int64_t step = (int64_t)gridDim.x * GROUPS * ROWS;
  // (every thread of a warp makes every round: the sums go through whole warps)
  for (int64_t base = (int64_t)blockIdx.x * GROUPS * ROWS; base < a.n; base += step, turn ^= 1) {
    const int64_t r0 = base + threadIdx.x / G * ROWS;
    uint4 xu[ROWS][V], du[ROWS][V];
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (e + v * G) * VE;
        const bool in = r0 + j < a.n && c < a.C;
        xu[j][v] = in ? *reinterpret_cast<const uint4*>((const T*)a.x + (r0 + j) * a.xs + c) : make_uint4(0, 0, 0, 0);
        if (a.delta) du[j][v] = in ? *reinterpret_cast<const uint4*>((const T*)a.delta + (r0 + j) * a.ds + c) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      const int64_t r = r0 + j;
      float s[V][VE];
      float ss = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        unpack(xu[j][v], s[v], T());
        if (a.delta) {
          float d[VE];
          unpack(du[j][v], d, T());
#pragma unroll
          for (int i = 0; i < VE; ++i) s[v][i] += d[i];
        }
#pragma unroll
        for (int i = 0; i < VE; ++i) ss = fmaf(s[v][i], s[v][i], ss);
      }
      const float inv = rsqrtf(over_row<G, false>(ss, part[turn][0]) * inv_c + a.eps);
      if (a.sum) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int c = (e + v * G) * VE;
          if (r < a.n && c < a.C) *reinterpret_cast<uint4*>((T*)a.sum + r * a.ss + c) = pack(s[v], T());
        }
      }
      float most = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (e + v * G) * VE;
        if constexpr (V == 1) {
#pragma unroll
          for (int i = 0; i < VE; ++i) s[v][i] *= inv * kept[i];
        } else if (c < a.C) {
          float g[VE];
          gains(c, g);
#pragma unroll
          for (int i = 0; i < VE; ++i) s[v][i] *= inv * g[i];
        }
        if constexpr (EIGHT) {
#pragma unroll
          for (int i = 0; i < VE; ++i) most = fmaxf(most, fabsf(s[v][i]));
        }
      }
      float back = 1.0f, scale = 1.0f;
      if constexpr (EIGHT) {
        scale = fmaxf(over_row<G, true>(most, part[turn][1]) / LARGEST, LEAST_SCALE);
        back = 1.0f / scale;
        if (e == 0 && r < a.n) a.scales[r] = scale;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int c = (e + v * G) * VE;
        if (r >= a.n || c >= a.C) continue;
        if constexpr (EIGHT) {
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            // the quotient, by its remainder as good as rounded once: a value near a border of two 8-bit
            // values goes the way that it should
            const float q = s[v][i] * back;
            s[v][i] = fmaf(fmaf(-q, scale, s[v][i]), back, q);
          }
          put8((uint8_t*)a.out + r * a.os + c, s[v]);
        } else {
          *reinterpret_cast<uint4*>((T*)a.out + r * a.os + c) = pack(s[v], T());
        }
      }
    }
  }
}

template <class T, bool EIGHT, int G, int V, int ROWS>
int launch(const NormArgs& a, cudaStream_t st) {
  // as many CTAs as an SM holds at most; few rows are spread over more of them
  constexpr int threads = threads_of(G), rows = threads / G * ROWS;
  const int64_t need = (a.n + rows - 1) / rows, most = 152 * 8 * (NT / threads);
  norm_kernel<T, EIGHT, G, V, ROWS><<<(unsigned)(need < most ? need : most), threads, 0, st>>>(a);
  return launched();
}

template <class T, bool EIGHT>
int by_width(const NormArgs& a, cudaStream_t st) {
  const int v = a.C * (int)sizeof(T) / 16;   // 16-byte pieces of a row
  // a row at a time while the rows are too few to fill the GPU
  const bool few = a.n <= 152 * 32;
  if (v <= 2) return few ? launch<T, EIGHT, 2, 1, 1>(a, st) : launch<T, EIGHT, 2, 1, 4>(a, st);
  if (v <= 8) return few ? launch<T, EIGHT, 8, 1, 1>(a, st) : launch<T, EIGHT, 8, 1, 4>(a, st);
  if (v <= 16) return few ? launch<T, EIGHT, 16, 1, 1>(a, st) : launch<T, EIGHT, 16, 1, 4>(a, st);
  if (v <= 32) return few ? launch<T, EIGHT, 32, 1, 1>(a, st) : launch<T, EIGHT, 32, 1, 4>(a, st);
  if (v <= 64) return few ? launch<T, EIGHT, 32, 2, 1>(a, st) : launch<T, EIGHT, 32, 2, 2>(a, st);
  if (v <= 128) return launch<T, EIGHT, 32, 4, 1>(a, st);
  if (v <= 256) return launch<T, EIGHT, 64, 4, 1>(a, st);
  if (v <= 512) return launch<T, EIGHT, 128, 4, 1>(a, st);
  if (v <= 1024) return launch<T, EIGHT, NT, 4, 1>(a, st);
  if (v <= 2048) return launch<T, EIGHT, NT, 8, 1>(a, st);
  if constexpr (sizeof(T) == 4) return launch<T, EIGHT, NT, 16, 1>(a, st);
  return TRACKFIT_ERR_UNSUPPORTED;
}

template <class T>
int by_output(const NormArgs& a, bool eight, cudaStream_t st) {
  return eight ? by_width<T, true>(a, st) : by_width<T, false>(a, st);
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
  NormArgs a;
  a.x = x, a.xs = x_stride, a.delta = delta, a.ds = delta_stride, a.sum = sum_out, a.ss = sum_stride;
  a.out = out, a.os = out_stride, a.n = n_rows, a.C = channels, a.eps = eps, a.gain = gain, a.scales = scales;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) return by_output<float>(a, eight, st);
  if (dtype == TRACKFIT_BF16_PROJ) return by_output<__nv_bfloat16>(a, eight, st);
  return by_output<__half>(a, eight, st);
}
