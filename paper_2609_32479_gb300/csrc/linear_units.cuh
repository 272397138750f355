// How linear attention over packed sequences is cut into units of work, none of which the
// host knows: only the offsets on the device say where a sequence begins.
//
// A tile is `seg` rows of the packed arrays, counted from row 0.  The unit of a tile takes
// the sequences that begin in it, to their ends, however far these reach.  Only sequences
// of more than `longest` rows are cut, at the rows that are multiples of `lseg` (a multiple
// of `seg`): the unit of the tile that begins at such a row takes the next lseg rows of the
// sequence that runs across it.  The state that crosses boundary i (row i * lseg) in the
// direction of the recurrence stands in the workspace: state_kernel leaves there what its
// own lseg rows add, carry_kernel then adds what comes from before.
#pragma once

#include "seq_ops.cuh"

namespace seqops {

struct Units {
  const int64_t* offs;     // [n_seq + 1]
  int64_t n_seq, n_rows;
  int64_t tiles;           // >= 1
  int seg, lseg;
  int64_t longest;         // longer sequences are cut
  int reverse;
};

// A run of rows of one sequence, taken in the direction of the recurrence.
struct Piece {
  int64_t lo, hi;          // rows
  int64_t seq;
  int64_t from;            // boundary whose state it goes on from; -1: the sequence's beginning
  bool ends;               // it reaches the sequence's end
};

// The sequences' rows, a warp reading 32 offsets at a time.
class Offsets {
 public:
  __device__ __forceinline__ Offsets(const Units& u, int lane) : u_(u), lane_(lane), base_(-64), mine_(0) {}
  __device__ __forceinline__ int64_t at(int64_t i) {
    if (i < base_ || i >= base_ + 32) {
      base_ = i;
      const int64_t j = i + lane_ < u_.n_seq ? i + lane_ : u_.n_seq;
      mine_ = clamp64(u_.offs[j], 0, u_.n_rows);
    }
    return __shfl_sync(FULL, mine_, (int)(i - base_));
  }

 private:
  const Units& u_;
  int lane_;
  int64_t base_, mine_;
};

// The pieces of a tile's unit, one after the other (all lanes alike).
class TilePieces {
 public:
  // (idle: no piece will be asked for)
  __device__ __forceinline__ TilePieces(const Units& u, int64_t tile, int lane, bool idle)
      : u_(u), offs_(u, lane), r0_(tile * u.seg), r1_(tile * u.seg + u.seg), last_(tile + 1 == u.tiles) {
    b_ = r0_ == 0 || idle ? 0 : first_at_least(u.offs, u.n_seq, r0_, lane);
    across_ = r0_ != 0 && r0_ % u.lseg == 0 && b_ > 0;
  }
  __device__ __forceinline__ bool next(Piece& p) {
    if (across_) {
      across_ = false;
      const int64_t lo = offs_.at(b_ - 1), hi = offs_.at(b_);
      if (hi - lo > u_.longest && lo < r0_ && hi > r0_) {
        p.seq = b_ - 1, p.lo = r0_, p.hi = hi < r0_ + u_.lseg ? hi : r0_ + u_.lseg;
        bounds(p, lo, hi);
        return true;
      }
    }
    if (b_ >= u_.n_seq) return false;
    const int64_t lo = offs_.at(b_);
    if (!(lo < r1_ || last_)) return false;
    int64_t hi = offs_.at(b_ + 1);
    if (hi < lo) hi = lo;
    p.seq = b_++, p.lo = lo, p.hi = hi;
    if (hi - lo > u_.longest) {
      const int64_t cut = (lo / u_.lseg + 1) * u_.lseg;
      if (cut < hi) p.hi = cut;
    }
    bounds(p, lo, hi);
    return true;
  }

 private:
  __device__ __forceinline__ void bounds(Piece& p, int64_t lo, int64_t hi) {
    const bool first = u_.reverse ? p.hi == hi : p.lo == lo;
    p.from = first ? -1 : (u_.reverse ? p.hi : p.lo) / u_.lseg;
    p.ends = u_.reverse ? p.lo == lo : p.hi == hi;
  }
  const Units& u_;
  Offsets offs_;
  int64_t r0_, r1_, b_;
  bool last_, across_;
};

// The piece whose end leaves a state at boundary `i`, if a cut sequence runs across it.
// `from` is -1 where the piece holds the sequence's beginning; else the state that comes
// from before is added later.
__device__ __forceinline__ bool boundary_piece(const Units& u, int64_t i, int lane, Piece& p) {
  const int64_t row = i * u.lseg;
  const int64_t b = first_at_least(u.offs, u.n_seq, row, lane);
  if (b == 0) return false;
  Offsets offs(u, lane);
  const int64_t lo = offs.at(b - 1), hi = offs.at(b);
  if (!(hi - lo > u.longest && lo < row && hi > row)) return false;
  p.seq = b - 1;
  p.ends = false;
  if (u.reverse) {
    p.lo = row, p.hi = hi < row + u.lseg ? hi : row + u.lseg;
    p.from = p.hi == hi ? -1 : i + 1;
  } else {
    p.lo = lo > row - u.lseg ? lo : row - u.lseg, p.hi = row;
    p.from = p.lo == lo ? -1 : i - 1;
  }
  return true;
}

constexpr int NW = 4;            // warps of a CTA, each with a unit of its own

struct LaArgs {
  Units u;
  const void *q, *k, *v;
  const float* g;
  void* out;
  int64_t qs, ks, vs, gs, os;    // row strides in elements
  const float* state_in;
  float* state_out;
  float* ws_state;               // [boundaries][H][K][V]
  float* ws_decay;               // [boundaries][H], sums of g
  int32_t* ws_flag;              // [boundaries]: 0 no cut sequence, 1 its first piece, 2 a later one
  int64_t bounds;                // boundaries 1 .. bounds - 1
  int H, K, V, slices;
  float scale;
};

// linear_mma.cu: the 16-bit types on the tensor cores.  Channels of v that a warp takes:
inline int linear_mma_cols(int K, int V) { return V > 16 && K <= 64 ? 32 : 16; }
int linear_mma(int32_t dtype, const LaArgs& a, bool state_only, cudaStream_t st);

}  // namespace seqops
