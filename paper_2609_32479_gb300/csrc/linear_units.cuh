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
  int longest;             // longer sequences are cut
  int reverse;
};

// A run of rows of one sequence, taken in the direction of the recurrence.  Rows count from
// a base row near them (a tile's or a boundary's), in 32 bits; a sequence's ends that are
// further than FAR from it are held there.
struct Piece {
  int lo, hi;
  int seq;
  bool goes_on;            // it does not hold the sequence's beginning
  bool ends;               // it holds the sequence's end
};
constexpr int FAR = 1 << 29;      // (the distance of two ends, too, fits 32 bits)

// The sequences' offsets from the base row, a warp reading 32 at a time.
class Offsets {
 public:
  __device__ __forceinline__ Offsets(const Units& u, int64_t base, int lane)
      : u_(u), base_(base), lane_(lane), first_(0), mine_(0), loaded_(false) {}
  __device__ __forceinline__ int at(int i) {
    if (!loaded_ || (unsigned)(i - first_) >= 32u) {
      loaded_ = true;
      first_ = i;
      const int64_t j = (int64_t)i + lane_ < u_.n_seq ? (int64_t)i + lane_ : u_.n_seq;
      mine_ = (int)clamp64(clamp64(u_.offs[j], 0, u_.n_rows) - base_, -FAR, FAR);
    }
    return __shfl_sync(FULL, mine_, i - first_);
  }

 private:
  const Units& u_;
  int64_t base_;
  int lane_, first_, mine_;
  bool loaded_;
};

// The pieces of a tile's unit, one after the other (all lanes alike), from the tile's first
// row.
class TilePieces {
 public:
  // (idle: no piece will be asked for)
  __device__ __forceinline__ TilePieces(const Units& u, int64_t tile, int lane, bool idle)
      : u_(u), offs_(u, tile * u.seg, lane), last_(tile + 1 == u.tiles) {
    const int64_t r0 = tile * u.seg;
    b_ = r0 == 0 || idle ? 0 : (int)first_at_least(u.offs, u.n_seq, r0, lane);
    cut_ = u.lseg - (int)(r0 % u.lseg);
    across_ = r0 != 0 && cut_ == u.lseg && b_ > 0;
  }
  __device__ __forceinline__ bool next(Piece& p) {
    if (across_) {
      across_ = false;
      const int lo = offs_.at(b_ - 1), hi = offs_.at(b_);
      if (hi - lo > u_.longest && lo < 0 && hi > 0) {
        p.seq = b_ - 1, p.lo = 0, p.hi = hi < u_.lseg ? hi : u_.lseg;
        bounds(p, lo, hi);
        return true;
      }
    }
    if (b_ >= (int)u_.n_seq) return false;
    const int lo = offs_.at(b_);
    if (!(lo < u_.seg || last_)) return false;
    int hi = offs_.at(b_ + 1);
    if (hi < lo) hi = lo;
    p.seq = b_++, p.lo = lo, p.hi = hi;
    if (hi - lo > u_.longest && cut_ < hi) p.hi = cut_ > lo ? cut_ : lo;
    bounds(p, lo, hi);
    return true;
  }

 private:
  __device__ __forceinline__ void bounds(Piece& p, int lo, int hi) {
    p.goes_on = u_.reverse ? p.hi != hi : p.lo != lo;
    p.ends = u_.reverse ? p.lo == lo : p.hi == hi;
  }
  const Units& u_;
  Offsets offs_;
  int b_, cut_;
  bool last_, across_;
};

// The piece whose end leaves a state at boundary `i`, if a cut sequence runs across it, its
// rows from the boundary's.  Where it goes on, the state that comes from before is added
// later.
__device__ __forceinline__ bool boundary_piece(const Units& u, int64_t i, int lane, Piece& p) {
  const int64_t row = i * u.lseg;
  const int64_t b = first_at_least(u.offs, u.n_seq, row, lane);
  if (b == 0) return false;
  Offsets offs(u, row, lane);
  const int lo = offs.at((int)b - 1), hi = offs.at((int)b);
  if (!(hi - lo > u.longest && lo < 0 && hi > 0)) return false;
  p.seq = (int)b - 1;
  p.ends = false;
  if (u.reverse) {
    p.lo = 0, p.hi = hi < u.lseg ? hi : u.lseg;
    p.goes_on = p.hi != hi;
  } else {
    p.lo = lo > -u.lseg ? lo : -u.lseg, p.hi = 0;
    p.goes_on = p.lo != lo;
  }
  return true;
}

struct LaArgs {
  Units u;
  const void *q, *k, *v;
  const float* g;
  void* out;
  int64_t qs, ks, vs, gs, os;    // row strides in elements
  const float* state_in;
  float* state_out;
  float* ws_state;               // [boundaries][H][K][V]
  // states in place only, else null: [boundaries][H][K][V], the state that the cut sequence whose
  // first piece ends at the boundary begins with (its last piece may be done first, and put the
  // state after the sequence in its place)
  float* ws_begin;
  float* ws_decay;               // [boundaries][H], sums of g
  int32_t* ws_flag;              // [boundaries]: 0 no cut sequence, 1 its first piece, 2 a later one
  int64_t bounds;                // boundaries 1 .. bounds - 1
  int H, K, V, slices;
  float scale;
};

// All units, fewer than 2^31: a CTA of one warp each, so that what a unit is comes from the
// CTA's number (the same for all lanes, which the compiler then knows), and so that registers
// are given out by the warp.
inline unsigned linear_grid(const LaArgs& a, bool state_only) {
  return (unsigned)((state_only ? a.bounds - 1 : a.u.tiles) * a.H * a.slices);
}

// The lseg rows that a tile lies in: all of its pieces but a whole sequence end at their bounds,
// boundary `block` before them and `block` + 1 behind.
__device__ __forceinline__ int block_of(const Units& u, int64_t tile) { return (int)((unsigned)tile / (unsigned)(u.lseg / u.seg)); }

// Where the state that a piece of a tile begins with stands, null for zeros.
__device__ __forceinline__ const float* piece_begins_with(const LaArgs& a, int block, int seq, int h, bool goes_on, bool ends) {
  const int64_t KV = (int64_t)a.K * a.V;
  if (goes_on) return a.ws_state + ((int64_t)(block + a.u.reverse) * a.H + h) * KV;
  if (a.ws_begin && !ends) return a.ws_begin + ((int64_t)(block + 1 - a.u.reverse) * a.H + h) * KV;
  return a.state_in ? a.state_in + ((int64_t)seq * a.H + h) * KV : nullptr;
}
// The same of a boundary's piece: where it goes on, zeros (what comes from before is added later).
__device__ __forceinline__ const float* boundary_begins_with(const LaArgs& a, int seq, int h, bool goes_on) {
  return a.state_in && !goes_on ? a.state_in + ((int64_t)seq * a.H + h) * a.K * a.V : nullptr;
}

// linear_mma.cu: the 16-bit types on the tensor cores.  Channels of v that a warp takes:
inline int linear_mma_cols(int K) { return K <= 64 ? 32 : 16; }
int linear_mma(int32_t dtype, const LaArgs& a, bool state_only, cudaStream_t st);

}  // namespace seqops
