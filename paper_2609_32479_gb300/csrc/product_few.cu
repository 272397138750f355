// Rows times a weight matrix for up to 16 rows of 16 or 8 bits: the weights are read once, and that
// bounds it.
//
// A warp takes 16 outputs and a part of K with the weights as the product's A (16 x 16) and the rows
// as its B (16 x 8).  Which channel stands where in a product does not matter as long as it is the
// same in both, so a lane's 16 bytes of a weight row, as they come from memory, are its part of two
// products (four of 8 bits, turned to fp16, exactly).  No shared memory on the way; the warps' sums
// are added in their order through it, then a thread finishes 16 bytes of outputs.
//
// Measured: 7 rows through 4096 x 4096 in bf16: 6.0 us among others in a graph, 5.6 TB/s of the 6.8 that a
// copy moves (weights in L2 from call to call would go faster, new ones take 13).
#include "product_units.cuh"

namespace {
using namespace seqops;

constexpr int WARPS = 8;

template <class T>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1) {
  if constexpr (__is_same(T, __half))
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Four values of 8 bits as two words of fp16 pairs.
__device__ __forceinline__ void widen(uint32_t u, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(u));
}

__device__ __forceinline__ uint4 load16(const uint8_t* p, bool there) {
  return there ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
}

template <class T, bool EIGHT, int NT>
__global__ void __launch_bounds__(WARPS * 32) product_few_kernel(const ProductArgs a) {
  constexpr int SZ = EIGHT ? 1 : 2, KS = 64 / SZ;     // channels that four lanes' 16 bytes hold
  constexpr int ROWS = 8 * NT, AHEAD = 4;
  __shared__ float sums[WARPS][ROWS][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int m0 = blockIdx.x * 16;
  const int steps = (a.K + KS - 1) / KS, per = (steps + WARPS - 1) / WARPS;
  const int s0 = warp * per, s1 = s0 + per < steps ? s0 + per : steps;
  const uint8_t* w0 = (const uint8_t*)a.w + (int64_t)(m0 + g) * a.ws * SZ + 16 * t;
  const uint8_t* w1 = w0 + 8 * a.ws * SZ;
  const uint8_t* x0 = (const uint8_t*)a.x + (int64_t)g * a.xs * SZ + 16 * t;
  const bool in1 = m0 + g + 8 < a.M;
  float acc[NT][4] = {};
  for (int s = s0; s < s1; s += AHEAD) {
    uint4 u0[AHEAD], u1[AHEAD], v[AHEAD][NT];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const bool in = s + i < s1 && (s + i) * KS + 16 / SZ * t < a.K;
      const int64_t at = (int64_t)(s + i) * 64;
      u0[i] = load16(w0 + at, in);
      u1[i] = load16(w1 + at, in && in1);
#pragma unroll
      for (int n = 0; n < NT; ++n) v[i][n] = load16(x0 + 8 * n * a.xs * SZ + at, in && g + 8 * n < a.n);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const uint32_t p[4] = {u0[i].x, u0[i].y, u0[i].z, u0[i].w}, q[4] = {u1[i].x, u1[i].y, u1[i].z, u1[i].w};
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint32_t r[4] = {v[i][n].x, v[i][n].y, v[i][n].z, v[i][n].w};
        if constexpr (EIGHT) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t a0, a1, a2, a3, b0, b1;
            widen(p[j], a0, a2), widen(q[j], a1, a3), widen(r[j], b0, b1);
            mma16<__half>(acc[n], a0, a1, a2, a3, b0, b1);
          }
        } else {
          mma16<T>(acc[n], p[0], q[0], p[1], q[1], r[0], r[1]);
          mma16<T>(acc[n], p[2], q[2], p[3], q[3], r[2], r[3]);
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    sums[warp][8 * n + 2 * t][g] = acc[n][0], sums[warp][8 * n + 2 * t + 1][g] = acc[n][1];
    sums[warp][8 * n + 2 * t][g + 8] = acc[n][2], sums[warp][8 * n + 2 * t + 1][g + 8] = acc[n][3];
  }
  __syncthreads();
  constexpr int VE = 16 / sizeof(T), PER = 16 / VE;   // threads of a row
  const int c = threadIdx.x % PER * VE;
  for (int r = threadIdx.x / PER; r < ROWS; r += WARPS * 32 / PER) {
    if (r >= a.n || m0 + c >= a.M) return;
    float y[VE] = {};
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
#pragma unroll
      for (int i = 0; i < VE; ++i) y[i] += sums[w][r][c + i];
    const int64_t col = m0 + c;
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 gate = a.gate ? *reinterpret_cast<const uint4*>((const T*)a.gate + r * a.gs + col) : none;
    const uint4 res = a.res ? *reinterpret_cast<const uint4*>((const T*)a.res + r * a.rs + col) : none;
    finish<T, EIGHT>(a, y, EIGHT ? a.x_scales[r] : 1.0f, (int)col, gate, res);
    *reinterpret_cast<uint4*>((T*)a.out + r * a.os + col) = pack(y, T());
  }
}

template <class T, bool EIGHT>
int launch(const ProductArgs& a, cudaStream_t st) {
  const unsigned grid = (unsigned)((a.M + 15) / 16);
  if (a.n <= 8) product_few_kernel<T, EIGHT, 1><<<grid, WARPS * 32, 0, st>>>(a);
  else product_few_kernel<T, EIGHT, 2><<<grid, WARPS * 32, 0, st>>>(a);
  return launched();
}

}  // namespace

int seqops::product_few(int32_t dtype, const ProductArgs& a, cudaStream_t st) {
  if (a.x_scales)
    return dtype == TRACKFIT_FP32 ? launch<float, true>(a, st)
           : dtype == TRACKFIT_BF16_PROJ ? launch<__nv_bfloat16, true>(a, st) : launch<__half, true>(a, st);
  return dtype == TRACKFIT_BF16_PROJ ? launch<__nv_bfloat16, false>(a, st) : launch<__half, false>(a, st);
}
