// Attention of packed queries to packed states: arguments and how the work is cut.
//
// The G = q_heads / kv_heads heads of a query that share a head of the states are rows of the
// same products: row i G + j stands for query i, head (kv head) G + j.  A tile is 16 (fewer where
// tiles are few, 128 for many queries to many states) of these rows, counted from row 0 whatever the sequences; each
// row has the range of states of its own sequence.  Where tiles are few, each row's range is
// cut into `splits` parts, and the parts' sums are joined by a second kernel.
#pragma once

#include <float.h>

#include "seq_ops.cuh"

namespace seqops {

struct CaArgs {
  const void *q, *k, *v;
  void* out;
  int64_t qs, ks, vs, os;        // row strides in elements
  const int64_t *qo, *ko;        // offsets [n_seq + 1]
  int64_t nq, nk, n_seq;
  int Hq, Hk, G, D;
  float scale2;                  // |scale| * log2(e), or 1 with a scale of 0
  uint32_t q_and, q_xor;         // on queries (two of 16 bits): zeroed with a scale of 0, negated below it
  int splits;
  int tr;                        // rows of a tile of the 16-row kernels, 1 to 16
  int tc_from;                   // sequences of at least so many states are cross_tc.cu's (0: none)
  int each;                      // heads of the states that a warp takes one after the other
  float* ws_o;                   // [splits][rows][Hk][D], sums not yet divided
  float2* ws_ml;                 // [splits][rows][Hk]: the largest score (base 2), the sum of weights
};

constexpr int FARTHEST = 0x7fffffff;

// Weights are 2^(score - largest + up), and so are their sums and O, which the division takes out
// again.  Alike for all parts of a row.
// fp32, bf16: with as many weights of one as there are states, values next to the type's largest
// would leave fp32 in O where their average does not.  (Not further down than these need: values
// next to the smallest would be lost.)
// fp16: the weights as operands have its range, 2^-24 to 65504, of which 2^15 for the largest uses
// all: they keep their bits down to 2^-29 of it, and none is more than 2^-40 of it off.  (Taken
// against one, they were lost below 2^-25: many states 17 below one of theirs, together as heavy,
// counted in the sum but not in O.)  2^31 values of fp16 by 2^15 are far below fp32's largest.
template <class T>
__device__ __forceinline__ float weight_up(int states) {
  return __is_same(T, __half) ? 15.0f : -(float)(32 - __clz(states));
}

// o f, an average of finite values where o is finite: held at the largest fp32, which the roundings
// may pass.
__device__ __forceinline__ float average(float o, float f) {
  const float y = o * f;
  return fabsf(y) == INFINITY && fabsf(o) < INFINITY ? copysignf(FLT_MAX, y) : y;
}

// The states that row (lane & 15) of a tile reads, [lo, hi) of this part, whether it is a query of a
// sequence at all, and the most states that a row of the tile reads in all parts.
__device__ __forceinline__ void find_rows(const CaArgs& a, int tile, int split, int lane, bool& in, int& lo, int& hi, int& most) {
  const int first = tile * a.tr, row = first + (lane & 15);
  const bool there = (lane & 15) < a.tr && row < (int)(a.nq * a.G);
  const int64_t q = (there ? row : first) / a.G;
  int64_t b = first_at_least(a.qo, a.n_seq, (int64_t)first / a.G + 1, lane) - 1;   // the last that begins at or
  if (b < 0) b = 0;                                                                // before the first row
  // the offsets that follow, 32 at a time: how many are at or before the row's query
  for (int64_t at = b + 1;; at += 32) {
    const int64_t o = at + lane < a.n_seq ? a.qo[at + lane] : INT64_MAX;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) n += __shfl_sync(FULL, o, i) <= q;
    b += n;
    if (!__any_sync(FULL, n == 32)) break;
  }
  in = there && a.qo[b] <= q && q < a.qo[b + 1];
  lo = hi = most = 0;
  if (in) {
    const int64_t l = clamp64(a.ko[b], 0, a.nk), h = clamp64(a.ko[b + 1], l, a.nk);
    if (a.tc_from && h - l >= a.tc_from) {
      in = false;
    } else {
      lo = (int)(l + (h - l) * split / a.splits), hi = (int)(l + (h - l) * (split + 1) / a.splits);
      most = (int)(h - l);
    }
  }
  most = __reduce_max_sync(FULL, most);
}

// The first state from `pos` on that a row of the tile reads, by all lanes' two rows.
__device__ __forceinline__ int first_wanted(int pos, int lo0, int hi0, int lo1, int hi1) {
  const int c0 = hi0 > pos && hi0 > lo0 ? (lo0 > pos ? lo0 : pos) : FARTHEST;
  const int c1 = hi1 > pos && hi1 > lo1 ? (lo1 > pos ? lo1 : pos) : FARTHEST;
  return __reduce_min_sync(FULL, c0 < c1 ? c0 : c1);
}

// cross_mma.cu: the 16-bit types on the tensor cores; cross_tf32.cu: fp32, likewise.
int cross_mma(int32_t dtype, const CaArgs& a, cudaStream_t st);
int cross_tf32(const CaArgs& a, cudaStream_t st);
// cross_tc.cu: sequences of at least CROSS_TC_FROM states, 128 rows at a time.
constexpr int CROSS_TC_FROM = 64;
int cross_tc(int32_t dtype, const CaArgs& a, cudaStream_t st);

}  // namespace seqops
