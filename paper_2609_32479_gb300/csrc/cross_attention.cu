// Attention of packed queries to the states of an encoder, packed too, of any other length:
// the queries of sequence b read the states of sequence b.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - max_j(...))
//
// A query whose sequence has no states gets zeros.  Heads of the queries share a head of
// the states in groups of q_heads / kv_heads.
#include "seq_ops.cuh"

namespace {
using namespace seqops;

constexpr int NW = 4;

struct CaArgs {
  const void *q, *k, *v;
  void* out;
  int64_t qs, ks, vs, os;        // row strides in elements
  const int64_t *qo, *ko;        // offsets [n_seq + 1]
  int64_t nq, nk, n_seq;
  int Hq, Hk, D;
  float scale2;                  // scale * log2(e)
};

// A warp takes one row of one head: the lanes take a state each for the products with the
// query, then D / 32 channels each for the sum of the values.
template <class T>
__global__ void __launch_bounds__(NW * 32) ca_simt_kernel(const __grid_constant__ CaArgs a) {
  __shared__ float sq[NW][MAX_DIM];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = (int64_t)blockIdx.x * NW + warp;
  const int h = (int)(unit % a.Hq);
  const int64_t row = unit / a.Hq;
  if (row >= a.nq) return;
  const int64_t b = first_at_least(a.qo, a.n_seq, row + 1, lane) - 1;
  if (b < 0 || !(row < a.qo[b + 1])) return;      // a row of no sequence
  const int64_t lo = clamp64(a.ko[b], 0, a.nk), hi = clamp64(a.ko[b + 1], lo, a.nk);
  const T* q = (const T*)a.q + row * a.qs + h * a.D;
  const T* k = (const T*)a.k + (h / (a.Hq / a.Hk)) * a.D;
  const T* v = (const T*)a.v + (h / (a.Hq / a.Hk)) * a.D;
  for (int i = lane; i < a.D; i += 32) sq[warp][i] = to_float(q[i]) * a.scale2;
  __syncwarp();
  float m = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t j0 = lo; j0 < hi; j0 += 32) {
    const int64_t j = j0 + lane;
    float s = -INFINITY;
    if (j < hi) {
      s = 0.0f;
      for (int i = 0; i < a.D; ++i) s = fmaf(sq[warp][i], to_float(k[j * a.ks + i]), s);
    }
    float mx = s;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, x));
    const float mn = fmaxf(m, mx);
    const float base = mn == -INFINITY ? 0.0f : mn;
    const float f = exp2f(m - base);
    const float p = exp2f(s - base);
    float sum = p;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(FULL, sum, x);
    l = fmaf(l, f, sum);
    m = mn;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= f;
    const int n = hi - j0 < 32 ? (int)(hi - j0) : 32;
    for (int jj = 0; jj < n; ++jj) {
      const float pj = __shfl_sync(FULL, p, jj);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < a.D) o[c] = fmaf(pj, to_float(v[(j0 + jj) * a.vs + lane + 32 * c]), o[c]);
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // nothing to read, or scores of -inf only: zeros
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 32 * c < a.D) put((T*)a.out + row * a.os + h * a.D + lane + 32 * c, o[c] * inv);
}

template <class T>
int launch_simt(const CaArgs& a, cudaStream_t st) {
  const int64_t units = a.nq * a.Hq;
  if ((units + NW - 1) / NW > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  ca_simt_kernel<T><<<(unsigned)((units + NW - 1) / NW), NW * 32, 0, st>>>(a);
  return launched();
}

}  // namespace

extern "C" size_t trackfit_cross_attention_workspace(int32_t dtype, int64_t n_q_rows, int64_t n_kv_rows, int64_t n_seq,
                                                     int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  (void)dtype, (void)n_q_rows, (void)n_kv_rows, (void)n_seq, (void)q_heads, (void)kv_heads, (void)head_dim;
  return 0;
}

extern "C" int trackfit_cross_attention(int32_t dtype, const void* q, int64_t q_stride, const int64_t* q_offsets,
                                        int64_t n_q_rows, const void* k, int64_t k_stride, const void* v,
                                        int64_t v_stride, const int64_t* kv_offsets, int64_t n_kv_rows, int64_t n_seq,
                                        int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale, void* out,
                                        int64_t out_stride, void* workspace, size_t workspace_size, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_cross_attention");
  const int64_t most = (int64_t)1 << 40;
  if (!type_ok(dtype) || n_q_rows < 0 || n_q_rows > most || n_kv_rows < 0 || n_kv_rows > most || n_seq < 0 ||
      n_seq > 0x7fffffff)
    return TRACKFIT_ERR_INVALID_ARG;
  if (!heads_ok(q_heads) || !heads_ok(kv_heads) || q_heads % kv_heads != 0 || !dim_ok(head_dim))
    return TRACKFIT_ERR_UNSUPPORTED;
  if (!isfinite(scale)) return TRACKFIT_ERR_INVALID_ARG;
  if (n_seq == 0 || n_q_rows == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!q_offsets || !kv_offsets || ((reinterpret_cast<uintptr_t>(q_offsets) | reinterpret_cast<uintptr_t>(kv_offsets)) & 7u))
    return TRACKFIT_ERR_INVALID_ARG;
  if (!rows_ok(q, q_stride, (int64_t)q_heads * head_dim, sz) ||
      !rows_ok(out, out_stride, (int64_t)q_heads * head_dim, sz))
    return TRACKFIT_ERR_INVALID_ARG;
  if (n_kv_rows > 0 && (!rows_ok(k, k_stride, (int64_t)kv_heads * head_dim, sz) ||
                        !rows_ok(v, v_stride, (int64_t)kv_heads * head_dim, sz)))
    return TRACKFIT_ERR_INVALID_ARG;
  const size_t need =
      trackfit_cross_attention_workspace(dtype, n_q_rows, n_kv_rows, n_seq, q_heads, kv_heads, head_dim);
  if (need > 0 && (!workspace || mis16(workspace) || workspace_size < need)) return TRACKFIT_ERR_INVALID_ARG;
  CaArgs a;
  a.q = q, a.k = k, a.v = v, a.out = out;
  a.qs = q_stride, a.ks = k_stride, a.vs = v_stride, a.os = out_stride;
  a.qo = q_offsets, a.ko = kv_offsets, a.nq = n_q_rows, a.nk = n_kv_rows, a.n_seq = n_seq;
  a.Hq = q_heads, a.Hk = kv_heads, a.D = head_dim, a.scale2 = scale * LOG2E;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) return launch_simt<float>(a, st);
  if (dtype == TRACKFIT_BF16_PROJ) return launch_simt<__nv_bfloat16>(a, st);
  return launch_simt<__half>(a, st);
}
