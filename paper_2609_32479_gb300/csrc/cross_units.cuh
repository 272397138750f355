// Attention of packed queries to packed states: arguments and how the work is cut.
//
// The G = q_heads / kv_heads heads of a query that share a head of the states are rows of the
// same products: row i G + j stands for query i, head (kv head) G + j.  A tile is 16 (or, many
// queries to many states, 128) of these rows, counted from row 0 whatever the sequences; each
// row has the range of states of its own sequence.  Where tiles are few, each row's range is
// cut into `splits` parts, and the parts' sums are joined by a second kernel.
#pragma once

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
  uint32_t q_and, q_xor;         // on two 16-bit queries: zeroed with a scale of 0, negated below it
  int splits;
  float* ws_o;                   // [splits][rows][Hk][D], sums not yet divided
  float2* ws_ml;                 // [splits][rows][Hk]: the largest score (base 2), the sum of weights
};

// cross_mma.cu: the 16-bit types on the tensor cores.
int cross_mma(int32_t dtype, const CaArgs& a, cudaStream_t st);

}  // namespace seqops
