// Attention of packed queries to the states of an encoder, packed too, of any other length:
// the queries of sequence b read the states of sequence b.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i . k_j - max_j(...))
//
// A query whose sequence has no states gets zeros.  Heads of the queries share a head of
// the states in groups of q_heads / kv_heads.
#include "cross_units.cuh"

namespace {
using namespace seqops;

constexpr int NW = 4;
constexpr int64_t MOST_ROWS = 0x7fffff00;   // of the products, and of states: counted in 32 bits

// The parts of each row's range joined: a warp a row and head of the states.
template <class T>
__global__ void __launch_bounds__(NW * 32) ca_join_kernel(const __grid_constant__ CaArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * NW + (threadIdx.x >> 5);
  const int64_t rows = a.nq * a.G, all = rows * a.Hk;
  if (unit >= all) return;
  const int hk = (int)(unit % a.Hk);
  const int64_t row = unit / a.Hk, q = row / a.G;
  const int64_t b = first_at_least(a.qo, a.n_seq, q + 1, lane) - 1;
  if (b < 0 || !(q < a.qo[b + 1])) return;      // a row of no sequence: no part has been written
  // a lane a part (splits <= 32)
  const float2 ml = lane < a.splits ? a.ws_ml[lane * all + unit] : make_float2(-INFINITY, 0.0f);
  float m = ml.x;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, x));
  const float f = ex2(ml.x - (m == -INFINITY ? 0.0f : m));
  float l = ml.y * f;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(FULL, l, x);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < a.splits; ++s) {
    const float fs = __shfl_sync(FULL, f, s);
    const float* p = a.ws_o + (s * all + unit) * a.D;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (lane + 32 * c < a.D) o[c] = fmaf(fs, p[lane + 32 * c], o[c]);
  }
  T* out = (T*)a.out + q * a.os + (hk * a.G + row % a.G) * a.D;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 32 * c < a.D) put(out + lane + 32 * c, average(o[c], inv));
}

// Whether the 128-row kernel runs: 16-bit types, sequences of at least 512 states and 64 rows of the
// products (queries by shared heads) on average, 128 where the 16-row kernel's heads are narrowest.
// Measured, the 16-row kernel against it, us (heads on heads of the states x width; sequences of
// rows and states):
//   8 on 8 x 64    64 of 64, 256: 26, 30 fp16 and 26, 27 bf16; 64 of 64, 512: 40, 39 and 40, 34; 64 of
//                  32, 2,048: 65, 108 and 65, 88; 64 of 64, 2,048: 125, 89 and 125, 74
//   4 on 4 x 128   64 of 64, 256: 28, 32 and 28, 28; 64 of 64, 512: 44, 42 and 44, 34; 64 of 32, 2,048:
//                  86, 110 and 85, 85; 256 of 100, 300: 158, 187 and 157, 160; of 100, 512: 236, 234
//                  and 235, 186
//   16 on 4 x 128  64 of 64, 512: 44, 42 fp16;  8 on 2 x 64  64 of 64, 512: 24, 32; of 64, 2,048: 55, 49
//   4 on 4 x 32    64 of 64, 512: 19, 32 and 19, 26; 64 of 64, 2,048: 55, 64 and 55, 55; 64 of 128, 512:
//                  26, 26 and 26, 24; 64 of 128, 2,048: 78, 51 and 79, 44
bool wide_tiles(int32_t dtype, int64_t nq, int64_t nk, int64_t n_seq, int G, int D) {
  return dtype != TRACKFIT_FP32 && nq * G >= (D <= 32 ? 128 : 64) * n_seq && nk >= 512 * n_seq;
}
// How a call is cut.  Parts of each row's range: as many as give every warp of the GPU something
// to do (152 x 12 of the 16-row kernels, 152 x 2 CTAs of the 128-row one, 152 for wide heads), not
// under 256 states each (512) on average, and at most the 32 that the joining warp has lanes
// for.  Where that leaves less than half of the warps busy, tiles of fewer rows, down to a
// sequence's (20 sequences of 1-2 queries, 4 heads: two tiles of 16 rows a head, each through ten
// sequences' states).
struct Cut {
  bool wide;
  int splits, tr;
};
Cut cut_of(int32_t dtype, int64_t nq, int64_t nk, int64_t n_seq, int Hq, int Hk, int D) {
  Cut c = {false, 1, 16};
  if (nq <= 0 || n_seq <= 0) return c;
  const int64_t G = Hq / Hk, rows = nq * G;
  c.wide = wide_tiles(dtype, nq, nk, n_seq, (int)G, D);
  const int64_t target = c.wide ? (D <= 64 ? 304 : 152) : 152 * 12, most = nk / n_seq / (c.wide ? 512 : 256);
  for (;; c.tr /= 2) {
    const int64_t units = (c.wide ? (rows + 127) / 128 : (rows + c.tr - 1) / c.tr) * Hk;
    int64_t s = target / units;
    if (s > most) s = most;
    c.splits = s < 1 ? 1 : s > 32 ? 32 : (int)s;
    if (c.wide || c.tr == 1 || units * c.splits * 2 >= target || c.tr / 2 < (rows + n_seq - 1) / n_seq) return c;
  }
}

}  // namespace

extern "C" size_t trackfit_cross_attention_workspace(int32_t dtype, int64_t n_q_rows, int64_t n_kv_rows, int64_t n_seq,
                                                     int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  if (!type_ok(dtype) || n_q_rows < 0 || n_kv_rows < 0 || n_seq < 0 || !heads_ok(q_heads) || !heads_ok(kv_heads) ||
      q_heads % kv_heads != 0 || !dim_ok(head_dim) || n_q_rows > MOST_ROWS / (q_heads / kv_heads) || n_kv_rows > MOST_ROWS)
    return 0;
  const int s = cut_of(dtype, n_q_rows, n_kv_rows, n_seq, q_heads, kv_heads, head_dim).splits;
  return s > 1 ? (size_t)s * n_q_rows * q_heads * (head_dim + 2) * 4 : 0;
}

extern "C" int trackfit_cross_attention(int32_t dtype, const void* q, int64_t q_stride, const int64_t* q_offsets,
                                        int64_t n_q_rows, const void* k, int64_t k_stride, const void* v,
                                        int64_t v_stride, const int64_t* kv_offsets, int64_t n_kv_rows, int64_t n_seq,
                                        int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale, void* out,
                                        int64_t out_stride, void* workspace, size_t workspace_size, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_cross_attention");
  if (!type_ok(dtype) || n_q_rows < 0 || n_kv_rows < 0 || n_seq < 0 || n_seq > 0x7fffffff) return TRACKFIT_ERR_INVALID_ARG;
  if (!heads_ok(q_heads) || !heads_ok(kv_heads) || q_heads % kv_heads != 0 || !dim_ok(head_dim))
    return TRACKFIT_ERR_UNSUPPORTED;
  if (n_q_rows > MOST_ROWS / (q_heads / kv_heads) || n_kv_rows > MOST_ROWS) return TRACKFIT_ERR_UNSUPPORTED;
  if (!isfinite(scale * LOG2E)) return TRACKFIT_ERR_INVALID_ARG;
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
  a.Hq = q_heads, a.Hk = kv_heads, a.G = q_heads / kv_heads, a.D = head_dim;
  a.scale2 = scale == 0.0f ? 1.0f : fabsf(scale) * LOG2E;
  a.q_and = scale == 0.0f ? 0u : ~0u, a.q_xor = scale < 0.0f ? (dtype == TRACKFIT_FP32 ? 0x80000000u : 0x80008000u) : 0u;
  const Cut cut = cut_of(dtype, n_q_rows, n_kv_rows, n_seq, q_heads, kv_heads, head_dim);
  a.splits = cut.splits, a.tr = cut.tr;
  // all heads of a tile by one warp where that leaves ten tiles for each of the 152 x 16 warps
  // (131,072 tracks of five queries, with one part a weight: 319 us, with a warp a head 451)
  a.each = (n_q_rows * a.G + 15) / 16 >= 10 * 152 * 16 ? kv_heads : 1;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = reinterpret_cast<float2*>(a.ws_o + (need > 0 ? (int64_t)a.splits * n_q_rows * q_heads * head_dim : 0));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  a.tc_from = 0;
  if (cut.wide) {
    // the 16-row kernel after it takes the sequences of few states, if there are any
    a.tc_from = CROSS_TC_FROM;
    const int rc = cross_tc(dtype, a, st);
    if (rc != TRACKFIT_OK) return rc;
  }
  const int rc = dtype == TRACKFIT_FP32 ? cross_tf32(a, st) : cross_mma(dtype, a, st);
  if (rc != TRACKFIT_OK || a.splits == 1) return rc;
  const unsigned grid = (unsigned)((n_q_rows * q_heads + NW - 1) / NW);   // (only few rows are split)
  if (dtype == TRACKFIT_FP32) ca_join_kernel<float><<<grid, NW * 32, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) ca_join_kernel<__nv_bfloat16><<<grid, NW * 32, 0, st>>>(a);
  else ca_join_kernel<__half><<<grid, NW * 32, 0, st>>>(a);
  return launched();
}
