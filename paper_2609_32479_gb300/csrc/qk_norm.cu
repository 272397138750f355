// Norms of queries and keys per head, with the position rotation in the same pass.
//
// Per row and head, over its D channels (sums in fp32 whatever the type):
//   y = x / sqrt(mean(x^2) + eps) * gain
//   and, for i < r / 2, the pair (y_i, y_{i + r/2}) turned by the angle
//   position * base^(-2 i / r); channels from r on are not turned.
//
// A pass over memory: each value is read once and written once, and that traffic bounds
// it.  A warp takes a few rows; G lanes hold a head, 16 bytes each, so that the norm is a
// sum over G lanes and a pair's other half is r/2 channels, hence whole lanes, away.
//
// The angle in turns is a product modulo 1: position times the frequency as a 64-bit
// fixed-point fraction of a turn, whose low 64 bits are exactly the fraction, however far the
// position.  What is lost: the frequency comes from fp64 operations, 2^-51 of it at most (at
// position 2^31 2^-22 of a turn), and the fraction's 32 upper bits are rounded to fp32, 2^-26 of a
// turn.  Every angle of a row is formed by one lane and shared through shared memory: all heads of a
// row turn alike.
//
// Measured: 1,310,003 rows of 4 + 4 heads of 32, bf16: 261 us, 5.2 TB/s of the 6.8 that a copy
// moves; 404 with two rows' loads under way instead of four and the frequencies read from the
// kernel's arguments, where lanes that ask for different ones wait for one another.
#include "seq_ops.cuh"

namespace {
using namespace seqops;

constexpr int WARPS = 8;
constexpr int CTAS = 4;          // of an SM
constexpr int MAX_ROWS = 4;      // rows that a warp takes at a time

struct QkArgs {
  const void *q, *k;
  void *qo, *ko;
  int64_t qs, ks, qos, kos;      // row strides in elements
  int64_t n;
  int hq, hk, D, half;           // half = r / 2
  int rows;                      // rows that a warp takes at a time, <= MAX_ROWS
  float eps;
  const float *qg, *kg;
  const int32_t* pos;
  uint64_t freq[MAX_DIM / 2];    // turns per position, in 2^-64 turns
};

template <class T, int G>
__global__ void __launch_bounds__(WARPS * 32, CTAS) qk_norm_kernel(const __grid_constant__ QkArgs a) {
  constexpr int VE = 16 / sizeof(T);
  constexpr int HPP = 32 / G;                       // heads of a pass
  // cosines, sines and sines with the other sign of a row's angles
  __shared__ __align__(16) float tab[WARPS][MAX_ROWS][3][MAX_DIM / 2];
  __shared__ uint64_t freq[MAX_DIM / 2];            // (lanes ask for different ones at once)
  for (int i = threadIdx.x; i < a.half; i += WARPS * 32) freq[i] = a.freq[i];
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int vi = lane % G, e0 = vi * VE;            // this lane's channels of a head
  const bool in_head = e0 < a.D;
  const int half = a.half, hl = half / VE;          // lanes between the halves of a pair
  const bool lower = e0 < half, turned = e0 < 2 * half;
  const int mate = turned ? (lower ? lane + hl : lane - hl) : lane;
  // the lower half of a pair is a cos - b sin, the upper b cos + a sin
  const float* tc = &tab[warp][0][0][turned ? (lower ? e0 : e0 - half) : 0];
  const float* ts = tc + (lower ? 2 : 1) * (MAX_DIM / 2);
  const float inv_d = 1.0f / (float)a.D;
  const int heads = a.hq + a.hk;
  const int passes = (heads + HPP - 1) / HPP;
  int lh = 0;                                       // angles of a row, to a power of two: 2^lh
  while ((1 << lh) < half) ++lh;
  const int64_t step = (int64_t)gridDim.x * WARPS * a.rows;
  for (int64_t r0 = ((int64_t)blockIdx.x * WARPS + warp) * a.rows; r0 < a.n; r0 += step) {
    const int nr = a.n - r0 < a.rows ? (int)(a.n - r0) : a.rows;
    for (int p = 0; p < passes; ++p) {
      const int head = p * HPP + lane / G;
      const bool on = head < heads && in_head, isq = head < a.hq;
      const T* src = isq ? (const T*)a.q + r0 * a.qs + head * a.D : (const T*)a.k + r0 * a.ks + (head - a.hq) * a.D;
      T* dst = isq ? (T*)a.qo + r0 * a.qos + head * a.D : (T*)a.ko + r0 * a.kos + (head - a.hq) * a.D;
      const int64_t from = isq ? a.qs : a.ks, to = isq ? a.qos : a.kos;
      uint4 u[MAX_ROWS];                            // the rows' loads under way together
#pragma unroll
      for (int j = 0; j < MAX_ROWS; ++j)
        u[j] = on && j < nr ? *reinterpret_cast<const uint4*>(src + j * from + e0) : make_uint4(0, 0, 0, 0);
      if (p == 0 && half > 0) {                     // the angles, while the rows come
        __syncwarp();
        for (int i = lane; i < nr << lh; i += 32) {
          const int f = i & ((1 << lh) - 1), rr = i >> lh;
          if (f >= half) continue;
          const uint64_t turn = (uint64_t)(int64_t)a.pos[r0 + rr] * freq[f];
          float s, c;
          sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &c);   // half turns in [-1, 1)
          tab[warp][rr][0][f] = c, tab[warp][rr][1][f] = s, tab[warp][rr][2][f] = -s;
        }
        __syncwarp();
      }
      const float* gain = isq ? a.qg : a.kg;
      float gn[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) gn[i] = gain && on ? gain[e0 + i] : 1.0f;
#pragma unroll
      for (int j = 0; j < MAX_ROWS; ++j) {
        if (j >= nr) break;
        float x[VE];
        unpack(u[j], x, T());
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < VE; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(FULL, ss, o);
        const float inv = rsqrtf(ss * inv_d + a.eps);
#pragma unroll
        for (int i = 0; i < VE; ++i) x[i] *= inv * gn[i];
        if (half > 0) {
          float c[VE], s[VE];
#pragma unroll
          for (int i = 0; i < VE; i += 4) {
            *reinterpret_cast<float4*>(&c[i]) = *reinterpret_cast<const float4*>(tc + j * 3 * (MAX_DIM / 2) + i);
            *reinterpret_cast<float4*>(&s[i]) = *reinterpret_cast<const float4*>(ts + j * 3 * (MAX_DIM / 2) + i);
          }
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            const float y = __shfl_sync(FULL, x[i], mate);
            if (turned) x[i] = fmaf(x[i], c[i], y * s[i]);
          }
        }
        if (on) *reinterpret_cast<uint4*>(dst + j * to + e0) = pack(x, T());
      }
    }
  }
}

template <class T, int G>
int launch(const QkArgs& a, unsigned grid, cudaStream_t st) {
  qk_norm_kernel<T, G><<<grid, WARPS * 32, 0, st>>>(a);
  return launched();
}

template <class T>
int by_width(const QkArgs& a, unsigned grid, cudaStream_t st) {
  const int v = a.D * (int)sizeof(T) / 16;   // 16-byte pieces of a head
  if constexpr (sizeof(T) == 2) {
    if (v <= 1) return launch<T, 1>(a, grid, st);
  }
  if (v <= 2) return launch<T, 2>(a, grid, st);
  if (v <= 4) return launch<T, 4>(a, grid, st);
  if (v <= 8) return launch<T, 8>(a, grid, st);
  if constexpr (sizeof(T) == 4) {
    if (v > 16) return launch<T, 32>(a, grid, st);
  }
  return launch<T, 16>(a, grid, st);
}

}  // namespace

extern "C" int trackfit_qk_norm(int32_t dtype, const void* q, int64_t q_stride, int32_t q_heads, const void* k,
                                int64_t k_stride, int32_t k_heads, int32_t head_dim, int64_t n_rows,
                                const float* q_gain, const float* k_gain, float eps, const int32_t* positions,
                                int32_t rot_dim, double rot_base, void* q_out, int64_t q_out_stride, void* k_out,
                                int64_t k_out_stride, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_qk_norm");
  if (!type_ok(dtype) || n_rows < 0 || n_rows > (int64_t)1 << 40) return TRACKFIT_ERR_INVALID_ARG;
  if (!dim_ok(head_dim) || !heads_ok(q_heads) || k_heads < 0 || k_heads > MAX_HEADS) return TRACKFIT_ERR_UNSUPPORTED;
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16 != 0) return TRACKFIT_ERR_UNSUPPORTED;
  if (!(eps > 0.0f) || !isfinite(eps)) return TRACKFIT_ERR_INVALID_ARG;
  if (rot_dim > 0 && (!(rot_base >= 1.0) || !isfinite(rot_base))) return TRACKFIT_ERR_INVALID_ARG;
  if (n_rows == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!rows_ok(q, q_stride, (int64_t)q_heads * head_dim, sz) ||
      !rows_ok(q_out, q_out_stride, (int64_t)q_heads * head_dim, sz))
    return TRACKFIT_ERR_INVALID_ARG;
  if (k_heads > 0 && (!rows_ok(k, k_stride, (int64_t)k_heads * head_dim, sz) ||
                      !rows_ok(k_out, k_out_stride, (int64_t)k_heads * head_dim, sz)))
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(q_gain) || mis4(k_gain) || mis4(positions) || (rot_dim > 0 && !positions)) return TRACKFIT_ERR_INVALID_ARG;
  QkArgs a;
  a.q = q, a.k = k, a.qo = q_out, a.ko = k_out;
  a.qs = q_stride, a.ks = k_stride, a.qos = q_out_stride, a.kos = k_out_stride;
  a.n = n_rows, a.hq = q_heads, a.hk = k_heads, a.D = head_dim, a.half = rot_dim / 2;
  a.eps = eps, a.qg = q_gain, a.kg = k_gain, a.pos = positions;
  for (int i = 0; i < rot_dim / 2; ++i)
    a.freq[i] = (uint64_t)ldexp(pow(rot_base, -2.0 * i / rot_dim) / (2.0 * 3.14159265358979323846), 64);
  // a row a warp while the rows are too few to fill the GPU, else four, whose loads are under way
  // together and whose angles (r / 2 a row) keep the lanes busy
  const int64_t fill = 152 * CTAS;
  a.rows = n_rows >= fill * WARPS * MAX_ROWS ? MAX_ROWS : 1;
  const int64_t need = (n_rows + (int64_t)WARPS * a.rows - 1) / ((int64_t)WARPS * a.rows);
  const unsigned grid = (unsigned)(need < fill ? need : fill);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) return by_width<float>(a, grid, st);
  if (dtype == TRACKFIT_BF16_PROJ) return by_width<__nv_bfloat16>(a, grid, st);
  return by_width<__half>(a, grid, st);
}
