// Rows times a weight matrix and the product's epilogue:
//   out = residual + act(x W^T [* x_scales w_scales] + bias) * sigma(gate)
//
// Up to 16 rows of 16 or 8 bits go to product_few.cu, more to product_tc.cu, fp32 to the kernel here:
// tiles on the CUDA cores, 16 channels at a time through two buffers in shared memory, the next one's
// loads under way while one is used.  A thread adds up RM x RN sums, two neighbouring ones in an
// instruction, in fp32 and in the order of the channels.  Where tiles are few, a cluster of CTAs has a
// tile, each a part of the channels; each adds up some of the tile's sums out of all parts, in their
// order.  4000 x 2048 x 4096: 1265 us, 53 TFLOP/s of about 75 that the multipliers could.
#include "product_units.cuh"

namespace {
using namespace seqops;

constexpr int MAX_INNER = 1 << 14, MAX_OUTER = 1 << 16;
constexpr int TK = 16, NT = 256;

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Four floats at the same place in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ float4 from_cta(uint32_t at, int rank) {
  uint32_t u;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(u) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(u) : "memory");
  return v;
}

// Tiles of TM x TN sums with 256 / TX x TX threads; `split` CTAs, a cluster, of a tile.  FEW: the tile's
// rows are outputs and its columns rows of x (up to 16 of them), else the other way round.
template <int RM, int RN, int TX, bool FEW>
__global__ void __launch_bounds__(NT) product_fp32_kernel(const ProductArgs a, int tiles_n, int split) {
  constexpr int TY = NT / TX, TM = TY * RM, TN = TX * RN, LX = TM * 4 / NT, LW = (TN * 4 + NT - 1) / NT;
  static_assert(RM % 4 == 0 && RN % 4 == 0, "16 bytes of rows and outputs");
  constexpr int SX = TM + 4, SW = TN + 4, HALF = TK * (SX + SW), SUMS = RM == 4 ? TM * TN : 0;
  __shared__ __align__(16) float buf[2 * HALF > SUMS ? 2 * HALF : SUMS];
  const int part = blockIdx.x % split, tile = blockIdx.x / split;
  // this CTA's channels: whole steps
  const int steps = (a.K + TK - 1) / TK, k_lo = (int)((int64_t)steps * part / split) * TK;
  const int k_hi = min(a.K, (int)((int64_t)steps * (part + 1) / split) * TK);
  const int64_t r0 = (int64_t)(tile / tiles_n) * TM;
  const int c0 = tile % tiles_n * TN, tx = threadIdx.x % TX, ty = threadIdx.x / TX;
  const float *px = (const float*)(FEW ? a.w : a.x), *pw = (const float*)(FEW ? a.x : a.w);
  const int64_t nx = FEW ? a.M : a.n, nw = FEW ? a.n : a.M, sx = FEW ? a.ws : a.xs, sw = FEW ? a.xs : a.ws;
  const int lr = threadIdx.x / 4, lk = threadIdx.x % 4 * 4;       // this thread's row and channels of a load
  const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float4 u[LX], v[LW];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      const int64_t r = r0 + lr + i * (NT / 4);
      u[i] = r < nx && k0 + lk < a.K ? __ldg(reinterpret_cast<const float4*>(px + r * sx + k0 + lk)) : none;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      const int64_t c = c0 + lr + i * (NT / 4);
      v[i] = lr + i * (NT / 4) < TN && c < nw && k0 + lk < a.K ? __ldg(reinterpret_cast<const float4*>(pw + c * sw + k0 + lk)) : none;
    }
  };
  auto put_down = [&](int b) {
    float *xs = buf + b * HALF, *ws = xs + TK * SX;
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      float* d = xs + lk * SX + lr + i * (NT / 4);
      d[0] = u[i].x, d[SX] = u[i].y, d[2 * SX] = u[i].z, d[3 * SX] = u[i].w;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      if (lr + i * (NT / 4) >= TN) continue;
      float* d = ws + lk * SW + lr + i * (NT / 4);
      d[0] = v[i].x, d[SW] = v[i].y, d[2 * SW] = v[i].z, d[3 * SW] = v[i].w;
    }
  };
  uint64_t acc[RM][RN / 2];
#pragma unroll
  for (int i = 0; i < RM; ++i)
#pragma unroll
    for (int j = 0; j < RN / 2; ++j) acc[i][j] = 0;
  if (k_lo < k_hi) load(k_lo), put_down(0);
  __syncthreads();
  for (int k0 = k_lo, b = 0; k0 < k_hi; k0 += TK, b ^= 1) {
    if (k0 + TK < k_hi) load(k0 + TK);
    const float *xs = buf + b * HALF + 4 * ty, *ws = buf + b * HALF + TK * SX + 4 * tx;
#pragma unroll
    for (int k = 0; k < TK; ++k) {
      float x[RM];
      uint64_t w[RN / 2];
#pragma unroll
      for (int i = 0; i < RM; i += 4) *reinterpret_cast<float4*>(&x[i]) = *reinterpret_cast<const float4*>(xs + k * SX + TY * i);
#pragma unroll
      for (int j = 0; j < RN; j += 4) {
        const ulonglong2 t = *reinterpret_cast<const ulonglong2*>(ws + k * SW + TX * j);
        w[j / 2] = t.x, w[j / 2 + 1] = t.y;
      }
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const uint64_t xx = both(x[i], x[i]);
#pragma unroll
        for (int j = 0; j < RN / 2; ++j) acc[i][j] = fma2(xx, w[j], acc[i][j]);
      }
    }
    if (k0 + TK < k_hi) put_down(b ^ 1);
    __syncthreads();
  }
  auto put = [&](int64_t r, int64_t c, float (&y)[4]) {
    if (r >= a.n || c >= a.M) return;
    const uint4 z = make_uint4(0, 0, 0, 0);
    const uint4 gate = a.gate ? *reinterpret_cast<const uint4*>((const float*)a.gate + r * a.gs + c) : z;
    const uint4 res = a.res ? *reinterpret_cast<const uint4*>((const float*)a.res + r * a.rs + c) : z;
    finish<float, false>(a, y, 1.0f, (int)c, gate, res);
    *reinterpret_cast<uint4*>((float*)a.out + r * a.os + c) = pack(y, 0.0f);
  };
  if constexpr (RM == 4 && RN == 4) {
    float s[4][4];                          // rows of the tile, columns
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 lo = parts(acc[i][0]), hi = parts(acc[i][1]);
      s[i][0] = lo.x, s[i][1] = lo.y, s[i][2] = hi.x, s[i][3] = hi.y;
    }
    // of four numbers a thread, in FEW the transposed: four outputs of a row of x
    if (split == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = FEW ? s[e][i] : s[i][e];
        if (FEW) put(c0 + 4 * tx + i, r0 + 4 * ty, y);
        else put(r0 + 4 * ty + i, c0 + 4 * tx, y);
      }
      return;
    }
    // the parts' sums in the buffers' place, four outputs side by side; then each CTA takes every
    // split-th group of four out of all parts
    constexpr int ACROSS = FEW ? TM / 4 : TN / 4;      // groups of a row of x
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int group = FEW ? (4 * tx + i) * ACROSS + ty : (4 * ty + i) * ACROSS + tx;
      *reinterpret_cast<float4*>(buf + 4 * group) =
          FEW ? make_float4(s[0][i], s[1][i], s[2][i], s[3][i]) : make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
    }
    cluster_sync();
    for (int g = part * NT + threadIdx.x; g < TM * TN / 4; g += split * NT) {
      const int64_t r = (FEW ? c0 : r0) + g / ACROSS, c = (FEW ? r0 : c0) + g % ACROSS * 4;
      if (r >= a.n || c >= a.M) continue;
      float y[4] = {};
      for (int p = 0; p < split; ++p) {
        const float4 t = from_cta(smem_addr(buf + 4 * g), p);
        y[0] += t.x, y[1] += t.y, y[2] += t.z, y[3] += t.w;
      }
      put(r, c, y);
    }
    cluster_sync();      // no CTA goes while another reads its sums
  } else {
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int j = 0; j < RN; j += 4) {
        const float2 lo = parts(acc[i][j / 2]), hi = parts(acc[i][j / 2 + 1]);
        float y[4] = {lo.x, lo.y, hi.x, hi.y};
        put(r0 + TY * (i / 4 * 4) + 4 * ty + i % 4, c0 + TX * j + 4 * tx, y);
      }
  }
}

template <int RM, int RN, int TX, bool FEW>
int launch(const ProductArgs& a, cudaStream_t st) {
  constexpr int TM = NT / TX * RM, TN = TX * RN;
  const int64_t rows = FEW ? a.M : a.n, cols = FEW ? a.n : a.M;
  const int tiles_n = (int)((cols + TN - 1) / TN);
  const int64_t tiles = (rows + TM - 1) / TM * tiles_n;
  // as many parts as fill the SMs twice, of 128 channels at least
  int split = 1;
  if (RM == 4)
    while (split < 8 && tiles * split < 2 * 152 && a.K / (2 * split) >= 128) split *= 2;
  if (tiles * split > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  if (split == 1) {
    product_fp32_kernel<RM, RN, TX, FEW><<<(unsigned)tiles, NT, 0, st>>>(a, tiles_n, 1);
  } else {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(tiles * split)), cfg.blockDim = dim3(NT), cfg.stream = st, cfg.attrs = &at, cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, product_fp32_kernel<RM, RN, TX, FEW>, a, tiles_n, split);
    if (e != cudaSuccess) return tf_status_from_cuda(e);
  }
  return launched();
}

// fp32: the tile whose work, with what of it lies beyond the array, is least; a thread's 8 x 8 sums take
// two thirds of the time of 4 x 4 ones for an output (51 against 34 TFLOP/s), where they fill the SMs.
int product_fp32(const ProductArgs& a, cudaStream_t st) {
  if (a.n <= 16) return launch<4, 4, 4, true>(a, st);
  auto padded = [&](int64_t tm, int64_t tn) { return (double)((a.n + tm - 1) / tm * tm) * (double)((a.M + tn - 1) / tn * tn); };
  const double large = padded(128, 128), square = 1.5 * padded(64, 64), narrow = 1.5 * padded(128, 32), thin = 1.5 * padded(256, 16);
  const bool fills = (a.n + 127) / 128 * ((a.M + 127) / 128) >= 152;
  if (fills && large <= square && large <= narrow && large <= thin) return launch<8, 8, 16, false>(a, st);
  if (thin < narrow && thin < square) return launch<4, 4, 4, false>(a, st);
  return narrow < square ? launch<4, 4, 8, false>(a, st) : launch<4, 4, 16, false>(a, st);
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
  if (n_rows > 0x7fffff00) return TRACKFIT_ERR_UNSUPPORTED;   // a tile's coordinates have 32 bits
  ProductArgs a;
  a.x = x, a.xs = x_stride, a.w = weight, a.ws = weight_stride, a.gate = gate, a.gs = gate_stride;
  a.res = residual, a.rs = residual_stride, a.out = out, a.os = out_stride;
  a.x_scales = x_scales, a.w_scales = weight_scales, a.bias = bias;
  a.n = n_rows, a.K = in_dim, a.M = out_dim, a.act = activation;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (!eight && dtype == TRACKFIT_FP32) return product_fp32(a, st);
  return n_rows <= PRODUCT_FEW ? product_few(dtype, a, st) : product_tc(dtype, a, st);
}
