// Rows times a weight matrix and the product's epilogue:
//   out = residual + act(x W^T [* x_scales w_scales] + bias) * sigma(gate)
//
// Up to 64 rows (fp32: 16) go to product_few.cu, more rows of 16 or 8 bits to product_tc.cu, more rows
// of fp32 to the kernel here: tiles of TM x TN outputs on the CUDA cores, 16 channels at a time through two
// buffers in shared memory, the next one's loads under way while one is used.  A thread adds up
// RM x RN outputs, two neighbouring ones in an instruction; each output's products are added in the
// order of the channels, in fp32.
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

// `split` CTAs, a cluster, of a tile.
template <int RM, int RN>
__global__ void __launch_bounds__(NT) product_fp32_kernel(const ProductArgs a, int tiles_n, int split) {
  constexpr int TM = 16 * RM, TN = 16 * RN, LX = TM * 4 / NT, LW = TN * 4 / NT;
  static_assert(RM % 4 == 0 && RN % 4 == 0, "16 bytes of rows and outputs");
  __shared__ __align__(16) float xs[2][TK][TM + 4], ws[2][TK][TN + 4];
  const int part = blockIdx.x % split, tile = blockIdx.x / split;
  // this CTA's channels: whole steps
  const int steps = (a.K + TK - 1) / TK, k_lo = (int)((int64_t)steps * part / split) * TK;
  const int k_hi = min(a.K, (int)((int64_t)steps * (part + 1) / split) * TK);
  const int64_t r0 = (int64_t)(tile / tiles_n) * TM;
  const int c0 = tile % tiles_n * TN, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int lr = threadIdx.x / 4, lk = threadIdx.x % 4 * 4;       // this thread's row and channels of a load
  const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float4 u[LX], v[LW];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      const int64_t r = r0 + lr + i * (NT / 4);
      u[i] = r < a.n && k0 + lk < a.K ? __ldg(reinterpret_cast<const float4*>((const float*)a.x + r * a.xs + k0 + lk)) : none;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      const int64_t c = c0 + lr + i * (NT / 4);
      v[i] = c < a.M && k0 + lk < a.K ? __ldg(reinterpret_cast<const float4*>((const float*)a.w + c * a.ws + k0 + lk)) : none;
    }
  };
  auto put_down = [&](int b) {
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      float* d = &xs[b][lk][lr + i * (NT / 4)];
      d[0] = u[i].x, d[TM + 4] = u[i].y, d[2 * (TM + 4)] = u[i].z, d[3 * (TM + 4)] = u[i].w;
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      float* d = &ws[b][lk][lr + i * (NT / 4)];
      d[0] = v[i].x, d[TN + 4] = v[i].y, d[2 * (TN + 4)] = v[i].z, d[3 * (TN + 4)] = v[i].w;
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
#pragma unroll
    for (int k = 0; k < TK; ++k) {
      float x[RM];
      uint64_t w[RN / 2];
#pragma unroll
      for (int i = 0; i < RM; i += 4) *reinterpret_cast<float4*>(&x[i]) = *reinterpret_cast<const float4*>(&xs[b][k][16 * i + 4 * ty]);
#pragma unroll
      for (int j = 0; j < RN; j += 4) {
        const ulonglong2 t = *reinterpret_cast<const ulonglong2*>(&ws[b][k][16 * j + 4 * tx]);
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
  auto put = [&](int64_t r, int c, float (&y)[4]) {
    const uint4 z = make_uint4(0, 0, 0, 0);
    const uint4 gate = a.gate ? *reinterpret_cast<const uint4*>((const float*)a.gate + r * a.gs + c) : z;
    const uint4 res = a.res ? *reinterpret_cast<const uint4*>((const float*)a.res + r * a.rs + c) : z;
    finish<float, false>(a, y, 1.0f, c, gate, res);
    *reinterpret_cast<uint4*>((float*)a.out + r * a.os + c) = pack(y, 0.0f);
  };
  if constexpr (RM == 4 && RN == 4) {
    if (split > 1) {
      // the parts' sums in the buffers' place, then rows part, part + split, .. of all of them
      static_assert(sizeof(xs) >= 4 * 64 * 16 * 2, "half a tile's sums");
      float *lo = &xs[0][0][0], *hi = &ws[0][0][0];      // rows 0-31, 32-63
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const int r = 4 * ty + i;
        const float2 x = parts(acc[i][0]), y = parts(acc[i][1]);
        *reinterpret_cast<float4*>((r < 32 ? lo : hi) + (r & 31) * TN + 4 * tx) = make_float4(x.x, x.y, y.x, y.y);
      }
      cluster_sync();
      for (int r = part + split * (threadIdx.x / 16); r < TM; r += split * (NT / 16)) {
        const int c = c0 + 4 * tx;
        if (r0 + r >= a.n || c >= a.M) continue;
        const uint32_t at = smem_addr((r < 32 ? lo : hi) + (r & 31) * TN + 4 * tx);
        float y[4] = {};
        for (int u = 0; u < split; ++u) {
          const float4 v = from_cta(at, u);
          y[0] += v.x, y[1] += v.y, y[2] += v.z, y[3] += v.w;
        }
        put(r0 + r, c, y);
      }
      cluster_sync();      // no CTA goes while another reads its sums
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int64_t r = r0 + 16 * (i / 4 * 4) + 4 * ty + i % 4;
    if (r >= a.n) continue;
#pragma unroll
    for (int j = 0; j < RN; j += 4) {
      const int c = c0 + 16 * j + 4 * tx;
      if (c >= a.M) continue;
      const float2 lo = parts(acc[i][j / 2]), hi = parts(acc[i][j / 2 + 1]);
      float y[4] = {lo.x, lo.y, hi.x, hi.y};
      put(r, c, y);
    }
  }
}

template <int RM, int RN>
int launch(const ProductArgs& a, cudaStream_t st) {
  const int tiles_n = (a.M + 16 * RN - 1) / (16 * RN);
  const int64_t tiles = (a.n + 16 * RM - 1) / (16 * RM) * tiles_n;
  if (tiles > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  // as many parts as fill the SMs twice, of 128 channels at least
  int split = 1;
  if (RM == 4)
    while (split < 8 && tiles * split < 2 * 152 && a.K / (2 * split) >= 128) split *= 2;
  if (split == 1) {
    product_fp32_kernel<RM, RN><<<(unsigned)tiles, NT, 0, st>>>(a, tiles_n, 1);
  } else {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(tiles * split)), cfg.blockDim = dim3(NT), cfg.stream = st, cfg.attrs = &at, cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, product_fp32_kernel<RM, RN>, a, tiles_n, split);
    if (e != cudaSuccess) return tf_status_from_cuda(e);
  }
  return launched();
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
  const bool fp32 = !eight && dtype == TRACKFIT_FP32;
  if (n_rows <= (fp32 ? PRODUCT_FEW_FP32 : PRODUCT_FEW)) return product_few(dtype, a, st);
  if (!fp32) return product_tc(dtype, a, st);
  // tiles of 128 x 128 while they fill the SMs, else of 64 x 64
  const bool large = (n_rows + 127) / 128 * ((out_dim + 127) / 128) >= 152;
  return large ? launch<8, 8>(a, st) : launch<4, 4>(a, st);
}
