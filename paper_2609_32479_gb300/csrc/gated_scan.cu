// The gated recurrence over packed sequences and its gradients.
//
//   z = sigma(p), w = 1 - z,  h_t = w_t h_{t-1} + z_t n_t
//   back, from the direction's last row to its first:
//   D_t = g_t + e_t,  e_{t-1} = w_t D_t,  dn = z D,  dp = z w (n - h_{t-1}) D
//
// Bound by memory: three values a row and channel are moved forward, five backward.  The rows are cut
// into parts of up to 128, and a CTA of 8 warps takes 128 bytes of channels of a part: a lane has one
// channel (16 bits: two neighbouring ones), a warp 16 rows one after the other, which come by TMA.
//
// What stands before a run of rows acts on it through one number a channel: h_last = A h_before + B,
// with A the product of the w.  A warp forms (A, B) of its rows, the CTA those of the part, and
//   h after part k = A_k (h after part k - 1) + B_k
// goes from part to part: through the workspace, in which a part leaves (A, B) as soon as it has
// them and h when it knows it.  A part looks back at up to WIN parts for one with h and then
// applies the (A, B) of those between, in their order: the result does not depend on when it
// looked.  Each word carries what it holds beside its 32 bits, so no fence is needed; parts are
// taken in order from a counter, so those a CTA waits for are done or under way.  A sequence's first
// row ends the look back: what came before it is left out by choice, not multiplied by 0 (it may
// not be finite).  Where sequences are short, a part begins with the last sequence that begins in the
// 20 rows before its place: then it has nothing to look back for.
//
// Few rows in short sequences: every part forms what is before it again from its sequence's first
// row on, by the same operations; no workspace has to be cleared and no part is waited for.
#include "seq_ops.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>

namespace {
using namespace seqops;

constexpr int TILE = 128;                  // rows of a part at most
constexpr int WARPS = 8, RPW = TILE / WARPS, NT = WARPS * 32;
constexpr int SHIFT = 20;                  // rows that a part may begin earlier, to begin with a sequence
constexpr int PIECE = TILE * 128;          // bytes of one array of a part
constexpr int MAX_CHANNELS = 1 << 16;
constexpr int64_t FEW_ROWS = 4096;
constexpr uint32_t PARTIAL = 1, WHOLE = 2; // what a word of the workspace holds

// A part's rows, and where sequences begin among them: bit i of `bound` says that an offset is row0 + i,
// i <= count.
struct Info {
  long long row0, first;                   // first: the number of the first offset at or behind row0
  int count;                               // 0: no more parts
  uint32_t plain;                          // no two offsets here are the same
  uint32_t bound[6];
};

struct GsArgs {
  CUtensorMap tp, tn, tg;                  // boxes of 128 bytes x 128 rows
  void *out, *dp, *dn;
  int64_t os, dps, dns;                    // row strides in elements
  const int64_t* offs;
  int64_t n_rows, n_seq;
  int C, reverse;
  const float *state_in, *d_state_out;
  float *state_out, *d_state_in;
  float* saved;                            // [parts][C]: the state before a part
  int64_t parts;
  int span, shift;                         // rows from one part's place to the next; SHIFT or 0
  int blocks;                              // CTAs side by side in a part
  unsigned long long* ticket;
  Info* info;                              // [parts]
  ulonglong2* words;                       // [parts][C]: A and B or h
  uint64_t limit_ns;
  unsigned long long* expired;
};

__device__ __forceinline__ float lds(uint32_t at) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void sts(uint32_t at, float x) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory"); }
__device__ __forceinline__ float rcp(float x) {   // (1 ulp; for x in [1, 2])
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// z and w of a gate, each accurate however near to 0: from 2^(-|p| log2 e) and 1 over one more than it.
__device__ __forceinline__ void gate(float p, float& z, float& w) {
  const float e = ex2(-LOG2E * fabsf(p)), r = rcp(1.0f + e), s = e * r;
  z = p < 0.0f ? s : r, w = p < 0.0f ? r : s;
}

// A lane's channels of a row: 4 bytes, one or two fp32 values (two in the instructions that take two).
template <class T>
struct Lane;
template <>
struct Lane<float> {
  static constexpr int V = 1;
  using P = float;
  static __device__ __forceinline__ P make(float a, float) { return a; }
  static __device__ __forceinline__ P get(uint32_t at) {
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
    return x;
  }
  static __device__ __forceinline__ void put(void* p, P x) { *(float*)p = x; }
  static __device__ __forceinline__ P mul(P a, P b) { return a * b; }
  static __device__ __forceinline__ P add(P a, P b) { return a + b; }
  static __device__ __forceinline__ P sub(P a, P b) { return a - b; }
  static __device__ __forceinline__ P fma(P a, P b, P c) { return fmaf(a, b, c); }
  static __device__ __forceinline__ P pick(bool first, P a, P b) { return first ? a : b; }
  static __device__ __forceinline__ void gates(P p, P& z, P& w) { gate(p, z, w); }
  static __device__ __forceinline__ float part(P a, int) { return a; }
};
template <class T>
struct Lane16 {
  static constexpr int V = 2;
  using P = uint64_t;
  static __device__ __forceinline__ P make(float a, float b) { return both(a, b); }
  static __device__ __forceinline__ uint32_t word(uint32_t at) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
    return x;
  }
  static __device__ __forceinline__ void put(void* p, P x) {
    const float2 f = parts(x);
    *(uint32_t*)p = pack2(f.x, f.y, T());
  }
  static __device__ __forceinline__ P mul(P a, P b) { return mul2(a, b); }
  static __device__ __forceinline__ P add(P a, P b) { return add2(a, b); }
  static __device__ __forceinline__ P sub(P a, P b) { return fma2(b, both(-1.0f, -1.0f), a); }
  static __device__ __forceinline__ P fma(P a, P b, P c) { return fma2(a, b, c); }
  static __device__ __forceinline__ P pick(bool first, P a, P b) { return first ? a : b; }
  static __device__ __forceinline__ void gates(P p, P& z, P& w) {
    const float2 f = parts(p);
    const float2 x = parts(mul2(both(fabsf(f.x), fabsf(f.y)), both(-LOG2E, -LOG2E)));
    const P e = both(ex2(x.x), ex2(x.y));
    const float2 y = parts(add2(e, both(1.0f, 1.0f)));
    const float2 r = make_float2(rcp(y.x), rcp(y.y)), s = parts(mul2(e, both(r.x, r.y)));
    z = both(f.x < 0.0f ? s.x : r.x, f.y < 0.0f ? s.y : r.y), w = both(f.x < 0.0f ? r.x : s.x, f.y < 0.0f ? r.y : s.y);
  }
  static __device__ __forceinline__ float part(P a, int v) { return v ? parts(a).y : parts(a).x; }
};
template <>
struct Lane<__nv_bfloat16> : Lane16<__nv_bfloat16> {
  static __device__ __forceinline__ P get(uint32_t at) {
    const uint32_t u = word(at);
    return both(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
};
template <>
struct Lane<__half> : Lane16<__half> {
  static __device__ __forceinline__ P get(uint32_t at) {
    const uint32_t u = word(at);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
    return both(f.x, f.y);
  }
};
template <class L>
__device__ __forceinline__ typename L::P get_state(const float* s) {
  if constexpr (L::V == 1) return s[0];
  else return *reinterpret_cast<const uint64_t*>(s);
}
template <class L>
__device__ __forceinline__ void put_state(float* s, typename L::P x) {
  if constexpr (L::V == 1) s[0] = x;
  else *reinterpret_cast<uint64_t*>(s) = x;
}

template <class L>
struct Shared {
  static constexpr int WIN = 32 / L::V;    // parts looked back at
  typename L::P agg_a[WARPS][32], agg_b[WARPS][32];   // A and B of the warps' rows
  typename L::P agg_e[WARPS][32];                     // backward: B of what comes from behind
  typename L::P win_a[WIN][32], win_b[WIN][32];       // of the parts before, nearest first
  uint32_t has[2][WARPS];                  // a sequence begins (ends) in a warp's rows: A does not count
  uint32_t status[WIN];
  Info info[2];
  uint64_t full[2];
  long long start;
  int from;
  int abort, never;
};
// The buffers come behind it: a part of fewer rows, taken backwards, has positions whose rows would lie
// up to 15 rows below its buffer; they are read there with the others and not used.
template <class L>
constexpr int SHARED = ((int)sizeof(Shared<L>) + 1023) / 1024 * 1024;

// ---------------------------------------------------------------- parts

// Part k's Info, by a whole warp.
__device__ __forceinline__ Info find_part(const GsArgs& a, int64_t k, int lane) {
  Info f;
  const int64_t place = k * a.span, next = (k + 1) * a.span;
  // the first offset beyond the part's place; the one before it is at or before the place
  int64_t j = first_at_least(a.offs, a.n_seq + 1, place + 1, lane);
  f.row0 = place;
  if (a.shift > 0 && j > 0 && k > 0) {
    const int64_t o = a.offs[j - 1];
    if (o > place - a.shift && o <= place) f.row0 = o;
  }
  // back to the first offset at or behind row0: those between are equal to row0 (32 at a time)
  for (;;) {
    const int64_t i = j - 1 - lane;
    const uint32_t ge = __ballot_sync(FULL, i >= 0 && a.offs[i] >= f.row0);
    const int n = ge == FULL ? 32 : __ffs(~ge) - 1;
    j -= n;
    if (n < 32) break;
  }
  f.first = j;
  // the offsets from there on, to the end of the part: the last one that the part behind it begins with
  int64_t end = next < a.n_rows ? next : a.n_rows;
  const int64_t most = end;                                  // no row of the part beyond this
  uint32_t bits[5] = {};
  uint32_t count = 0;
  for (int64_t i = j;; i += 32) {
    const int64_t o = i + lane <= a.n_seq ? a.offs[i + lane] : INT64_MAX;
    const int64_t d = o - f.row0;
    const bool here = o <= most && d >= 0 && d <= TILE;
    count += __popc(__ballot_sync(FULL, here));
#pragma unroll
    for (int w = 0; w < 5; ++w) bits[w] |= __reduce_or_sync(FULL, here && (d >> 5) == w ? 1u << (d & 31) : 0u);
    if (__any_sync(FULL, o > most)) break;
  }
  if (a.shift > 0 && next < a.n_rows) {
    // the highest bit, if it is within the last `shift` rows
    int top = -1;
#pragma unroll
    for (int w = 0; w < 5; ++w)
      if (bits[w]) top = 32 * w + 31 - __clz(bits[w]);
    if (top >= 0 && f.row0 + top > next - a.shift && f.row0 + top <= next) end = f.row0 + top;
  }
  f.count = (int)(end - f.row0);
  uint32_t ones = 0;
#pragma unroll
  for (int w = 0; w < 5; ++w) f.bound[w] = bits[w], ones += __popc(bits[w]);
  f.bound[5] = 0;
  f.plain = ones == count;
  return f;
}

// Before the parts' kernel: the workspace cleared, and each part found; a warp a part.
__global__ void __launch_bounds__(256) prepare_kernel(const __grid_constant__ GsArgs a) {
  const int64_t k = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  if (k >= a.parts) return;
  if (k == 0 && lane == 0) *a.ticket = 0;
  for (int c = lane; c < a.C; c += 32) a.words[k * a.C + c] = make_ulonglong2(0, 0);
  const Info f = find_part(a, k, lane);
  if (lane == 0) a.info[k] = f;
}

// Position i of a part in the direction of the recurrence -> its row, as a distance from row0.
__device__ __forceinline__ int row_in(const GsArgs& a, const Info& f, int i) { return a.reverse ? f.count - 1 - i : i; }
__device__ __forceinline__ bool bound(const Info& f, int d) { return (f.bound[d >> 5] >> (d & 31)) & 1u; }

// 16 of the bits from number `low` on (below 0: zeros).
__device__ __forceinline__ uint32_t bits16(const Info& f, int low) {
  if (low <= -16) return 0;
  const int l = low < 0 ? 0 : low, w = l >> 5;
  const uint32_t x = __funnelshift_r(f.bound[w], f.bound[w + 1 < 6 ? w + 1 : 5], l & 31);
  return (low < 0 ? x << -low : x) & 0xffffu;
}
// Of a warp's 16 positions, bit i for the i-th: rows of sequences, first rows, last rows.
struct Mine {
  uint32_t valid, begins, ends;
};
__device__ __forceinline__ Mine mine_of(const GsArgs& a, const Info& f, int64_t row_lo, int64_t row_hi, int warp) {
  const int i0 = warp * RPW;
  const int l = (int)clamp64(row_lo - f.row0, 0, f.count), h = (int)clamp64(row_hi - f.row0, 0, f.count);
  const int lo = (a.reverse ? f.count - h : l) - i0, hi = (a.reverse ? f.count - l : h) - i0;
  Mine r;
  r.valid = (hi <= 0 ? 0u : hi >= RPW ? 0xffffu : (1u << hi) - 1u) & (lo <= 0 ? 0xffffu : lo >= RPW ? 0u : 0xffffu << lo);
  if (a.reverse) {   // position i is row count - 1 - i: it begins with the row's upper border
    r.begins = __brev(bits16(f, f.count - i0 - RPW + 1)) >> 16;
    r.ends = __brev(bits16(f, f.count - i0 - RPW)) >> 16;
  } else {
    r.begins = bits16(f, i0), r.ends = bits16(f, i0 + 1);
  }
  r.begins &= r.valid, r.ends &= r.valid;
  return r;
}
// The sequence that begins or ends with position i, by the lower or the upper border of its row: a whole
// warp.  The offsets' bits are counted, or, where empty sequences make offsets equal, they are.
__device__ __noinline__ int64_t sequence(const GsArgs& a, const Info& f, int i, bool lower) {
  const int d = row_in(a, f, i) + (lower ? 0 : 1);
  int64_t j = f.first;
  if (f.plain) {
#pragma unroll
    for (int w = 0; w < 5; ++w) {
      const int n = d - 32 * w;
      j += __popc(n >= 32 ? f.bound[w] : n > 0 ? f.bound[w] & ((1u << n) - 1u) : 0u);
    }
    j -= lower ? 0 : 1;
  } else {
    // lower border: the last offset at the row; upper: the one before the first there
    const int64_t row = f.row0 + d;
    for (int64_t at = f.first;; at += 32) {
      const int64_t o = at + (threadIdx.x & 31) <= a.n_seq ? a.offs[at + (threadIdx.x & 31)] : INT64_MAX;
      const int n = __popc(__ballot_sync(FULL, lower ? o <= row : o < row));
      j += n;
      if (n < 32) break;
    }
    j -= 1;
  }
  return clamp64(j, 0, a.n_seq - 1);
}

// Among the warps of the CTA.
__device__ __forceinline__ void meet() { __syncthreads(); }

// A part's rows on their way (one lane): their bytes and the Info's arrival complete full[buf].
template <class L, bool BACK>
__device__ __forceinline__ void fetch(const GsArgs& a, Shared<L>* s, uint8_t* smem, int buf, int64_t row0, int c0) {
  constexpr int ARRAYS = BACK ? 3 : 2;
  const uint32_t full = smem_addr(&s->full[buf]), to = smem_addr(smem + buf * ARRAYS * PIECE);
  sm100::mbar_arrive_expect_tx(full, ARRAYS * PIECE);
  sm100::tma_load_2d(to, &a.tp, full, c0, (int)row0);
  sm100::tma_load_2d(to + PIECE, &a.tn, full, c0, (int)row0);
  if constexpr (BACK) sm100::tma_load_2d(to + 2 * PIECE, &a.tg, full, c0, (int)row0);
}

// The warps' (A, B), in their order (BACK: the last first), as one; A does not count if `has`.
template <class L, bool BACK>
__device__ __forceinline__ void joined(const Shared<L>* s, int lane, typename L::P& fa, typename L::P& fb, bool& has) {
  fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f), has = false;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    const int u = BACK ? WARPS - 1 - i : i;
    const typename L::P ga = s->agg_a[u][lane], gb = BACK ? s->agg_e[u][lane] : s->agg_b[u][lane];
    const bool h = s->has[BACK][u];
    has = has || h;
    fb = L::pick(h, gb, L::fma(ga, fb, gb));
    fa = L::mul(ga, fa);
  }
}

__device__ __forceinline__ unsigned long long word(uint32_t what, float x) {
  return (unsigned long long)what << 32 | __float_as_uint(x);
}
__device__ __forceinline__ void leave(unsigned long long* p, unsigned long long v) {
  asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ ulonglong2 look(const ulonglong2* p) {
  ulonglong2 v;
  asm volatile("ld.relaxed.gpu.global.v2.u64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "l"(p));
  return v;
}

// What the parts before part k in the pass's direction leave for this CTA's channels: false if the wait for
// them expired.  All warps; `in`: the lane has channels, c the first of them.
template <class L>
__device__ __forceinline__ bool look_back(const GsArgs& a, bool up, Shared<L>* s, int64_t k, int c, bool in, typename L::P& carry) {
  constexpr int V = L::V, WIN = Shared<L>::WIN, EACH = WIN / WARPS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t there = up ? a.parts - 1 - k : k;             // so many parts there are (up: of higher numbers)
  uint64_t t0 = 0;
  for (int round = 0;; ++round) {
    ulonglong2 u[EACH][V];                                    // all under way before the first is used
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int d = warp * EACH + i;
      const int64_t at = up ? k + 1 + d : k - 1 - d;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        u[i][v] = make_ulonglong2(0, (unsigned long long)WHOLE << 32);
        if (d < there && in) u[i][v] = look(a.words + at * a.C + c + v);
      }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int d = warp * EACH + i;
      bool ready = true, whole = true, some = false;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const uint32_t what = (uint32_t)(u[i][v].y >> 32);
        whole = whole && what == WHOLE, some = some || (in && what == WHOLE);
        ready = ready && (what == WHOLE || (what == PARTIAL && u[i][v].x >> 32 == PARTIAL));
      }
      s->win_a[d][lane] = L::make(__uint_as_float((uint32_t)u[i][0].x), __uint_as_float((uint32_t)u[i][V - 1].x));
      s->win_b[d][lane] = L::make(__uint_as_float((uint32_t)u[i][0].y), __uint_as_float((uint32_t)u[i][V - 1].y));
      // all channels of a part alike: a part seen while h replaces B counts as not there
      const bool all_whole = __all_sync(FULL, whole), all_ready = __all_sync(FULL, ready), any = __any_sync(FULL, some);
      if (lane == 0) s->status[d] = all_whole ? WHOLE : all_ready && !any ? PARTIAL : 0u;
    }
    meet();
    if (warp == 0) {
      const uint32_t st = lane < WIN ? s->status[lane] : 0u;
      const uint32_t whole = __ballot_sync(FULL, st == WHOLE), none = __ballot_sync(FULL, st == 0u);
      const int w = whole ? __ffs(whole) - 1 : 32, z = none ? __ffs(none) - 1 : 32;
      if (lane == 0) {
        s->from = w < z ? w : -1;
        if (w >= z && (round & 7) == 7) {
          const uint64_t now = sm100::globaltimer();
          if (t0 == 0) t0 = now;
          else if (now - t0 > a.limit_ns) s->abort = 1;
        }
      }
    }
    meet();
    if (s->from >= 0) break;
    if (*(volatile int*)&s->abort) return false;
  }
  const int from = s->from;
  carry = s->win_b[from][lane];
  for (int d = from - 1; d >= 0; --d) carry = L::fma(s->win_a[d][lane], carry, s->win_b[d][lane]);
  return true;
}

// (A, B) of a part, or B alone where the part holds a sequence's beginning, for those behind it.
template <class L>
__device__ __forceinline__ void leave_part(const GsArgs& a, int64_t k, int c, typename L::P fa, typename L::P fb, bool has) {
#pragma unroll
  for (int v = 0; v < L::V; ++v) {
    unsigned long long* w = &a.words[k * a.C + c + v].x;
    if (!has) leave(w, word(PARTIAL, L::part(fa, v)));
    leave(w + 1, word(has ? WHOLE : PARTIAL, L::part(fb, v)));
  }
}

// What a pass holds of the part in hand.
struct Hand {
  int64_t k;
  int c;                                   // the lane's first channel
  bool in;                                 // there is one
  Mine my;
};

// The carry into the part, once its (A, B) are in shared memory and left for others (warp 0: fa, fb, has
// are the part's): false if a wait expired.
template <class L, bool BACK>
__device__ __forceinline__ bool carry_into(const GsArgs& a, Shared<L>* s, const Hand& h, bool inside, typename L::P fa,
                                           typename L::P fb, bool has, typename L::P& carry) {
  carry = L::make(0.0f, 0.0f);
  if (!inside) return true;
  if (!look_back<L>(a, BACK != (a.reverse != 0), s, h.k, h.c, h.in, carry)) return false;
  if (threadIdx.x < 32 && h.in && !has) {
    const typename L::P x = L::fma(fa, carry, fb);
#pragma unroll
    for (int v = 0; v < L::V; ++v) leave(&a.words[h.k * a.C + h.c + v].y, word(WHOLE, L::part(x, v)));
  }
  return true;
}
// What is before the part counts if its first position in the pass's direction is within a sequence.
template <bool BACK>
__device__ __forceinline__ bool is_inside(const GsArgs& a, const Info& f, int64_t row_lo, int64_t row_hi) {
  const int d = row_in(a, f, BACK ? f.count - 1 : 0);
  const int64_t r = f.row0 + d;
  return r >= row_lo && r < row_hi && !bound(f, BACK != (a.reverse != 0) ? d + 1 : d);
}

// Rows one after the other in shared memory.
struct Walk {
  uint32_t at;
  int step;
};
__device__ __forceinline__ Walk walk_of(const GsArgs& a, const Info& f, const uint8_t* raw, const Mine& my) {
  const int d0 = row_in(a, f, (int)(threadIdx.x >> 5) * RPW);
  Walk w;
  w.at = smem_addr(raw) + (my.valid ? d0 * 128 + (threadIdx.x & 31) * 4 : 0);
  w.step = my.valid ? (a.reverse ? -128 : 128) : 0;
  return w;
}

template <class T>
struct Forward {
  using L = Lane<T>;
  using P = typename L::P;
  static constexpr bool BACK = false;
  static constexpr int BUFS = 1, CTAS = 4, ARRAYS = 2;
  P w[RPW];

  // A and B of the warp's rows; each row's w, and its z n in the place of p (16 bits: of p and n).  A
  // sequence's first row gets its h there: the state before is read once only, since the CTA with the
  // sequence's end may write the state after it to the same place as soon as this part has left its B.
  __device__ __forceinline__ void sums(const GsArgs& a, Shared<L>* s, const Info& f, const Hand& h, Walk k) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    P fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < RPW; ++i, k.at += k.step) {
      if (!((h.my.valid >> i) & 1u)) continue;
      P z;
      L::gates(L::get(k.at), z, w[i]);
      P x = L::mul(z, L::get(k.at + PIECE));
      if ((h.my.begins >> i) & 1u) {
        fb = L::make(0.0f, 0.0f);
        if (a.state_in) {
          const int64_t b = sequence(a, f, warp * RPW + i, !a.reverse);
          if (h.in) fb = get_state<L>(a.state_in + b * a.C + h.c);
        }
        x = fb = L::fma(w[i], fb, x);
      } else {
        fb = L::fma(w[i], fb, x);
      }
      fa = L::mul(fa, w[i]);
      sts(k.at, L::part(x, 0));
      if constexpr (L::V == 2) sts(k.at + PIECE, L::part(x, 1));
    }
    s->agg_a[warp][lane] = fa, s->agg_b[warp][lane] = fb;
    if (lane == 0) s->has[0][warp] = h.my.begins != 0;
  }
  __device__ __forceinline__ void before_carry(const GsArgs&, Shared<L>*, const Info&, const Hand&, Walk) {}
  __device__ __forceinline__ void finish(const GsArgs& a, Shared<L>* s, const Info& f, const Hand& hd, Walk k, P carry) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (a.saved && warp == 0 && hd.in) put_state<L>(a.saved + hd.k * a.C + hd.c, carry);
    P h = carry;
    for (int u = 0; u < warp; ++u) h = L::pick(s->has[0][u], s->agg_b[u][lane], L::fma(s->agg_a[u][lane], h, s->agg_b[u][lane]));
    const uint32_t put = hd.in ? hd.my.valid : 0u, ends = a.state_out ? hd.my.ends : 0u;
    const int64_t step = a.reverse ? -a.os : a.os;
    T* out = (T*)a.out + (f.row0 + row_in(a, f, warp * RPW)) * a.os + hd.c;
#pragma unroll
    for (int i = 0; i < RPW; ++i, out += step, k.at += k.step) {
      const P x = L::make(lds(k.at), L::V == 2 ? lds(k.at + PIECE) : 0.0f);
      h = L::pick((hd.my.begins >> i) & 1u, x, L::fma(w[i], h, x));
      if ((put >> i) & 1u) L::put(out, h);
      if ((ends >> i) & 1u) {
        const int64_t b = sequence(a, f, warp * RPW + i, a.reverse);
        if (hd.in) put_state<L>(a.state_out + b * a.C + hd.c, h);
      }
    }
  }
};

template <class T>
struct Backward {
  using L = Lane<T>;
  using P = typename L::P;
  static constexpr bool BACK = true;
  static constexpr int BUFS = 2, CTAS = 2, ARRAYS = 3;
  P z[RPW], w[RPW];

  // In the recurrence's direction: (A, B) of the states, and of what goes back through the warp's rows, in
  // which a row's g counts with the w up to it, as far as the first sequence's end.  There D is known, and
  // waits in the place of p (16 bits: of p and g): what the state's gradient is may be written over once
  // this part has left its B.
  __device__ __forceinline__ void sums(const GsArgs& a, Shared<L>* s, const Info& f, const Hand& h, Walk k) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    P fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f), fe = L::make(0.0f, 0.0f);
    uint32_t alive = h.my.valid;
    if (h.my.ends) alive &= ((h.my.ends & -h.my.ends) << 1) - 1u;
#pragma unroll
    for (int i = 0; i < RPW; ++i, k.at += k.step) {
      if (!((h.my.valid >> i) & 1u)) continue;
      L::gates(L::get(k.at), z[i], w[i]);
      if ((h.my.begins >> i) & 1u) {
        fb = L::make(0.0f, 0.0f);
        if (a.state_in) {
          const int64_t b = sequence(a, f, warp * RPW + i, !a.reverse);
          if (h.in) fb = get_state<L>(a.state_in + b * a.C + h.c);
        }
      }
      fb = L::fma(w[i], fb, L::mul(z[i], L::get(k.at + PIECE)));
      fa = L::mul(fa, w[i]);
      P g = L::get(k.at + 2 * PIECE);
      if ((h.my.ends >> i) & 1u) {
        if (a.d_state_out) {
          const int64_t b = sequence(a, f, warp * RPW + i, a.reverse);
          if (h.in) g = L::add(g, get_state<L>(a.d_state_out + b * a.C + h.c));
        }
        sts(k.at, L::part(g, 0));
        if constexpr (L::V == 2) sts(k.at + 2 * PIECE, L::part(g, 1));
      }
      if ((alive >> i) & 1u) fe = L::fma(fa, g, fe);
    }
    s->agg_a[warp][lane] = fa, s->agg_b[warp][lane] = fb, s->agg_e[warp][lane] = fe;
    if (lane == 0) s->has[0][warp] = h.my.begins != 0, s->has[1][warp] = h.my.ends != 0;
  }
  // The states again, from the one saved before the part: z w (n - h) takes the place of p (16 bits: of p
  // and n).  At a sequence's last row D is known: its results, and e before it instead of w.
  __device__ __forceinline__ void before_carry(const GsArgs& a, Shared<L>* s, const Info& f, const Hand& hd, Walk k) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    P h = L::make(0.0f, 0.0f);
    if (hd.in) h = get_state<L>(a.saved + hd.k * a.C + hd.c);
    for (int u = 0; u < warp; ++u) h = L::pick(s->has[0][u], s->agg_b[u][lane], L::fma(s->agg_a[u][lane], h, s->agg_b[u][lane]));
#pragma unroll
    for (int i = 0; i < RPW; ++i, k.at += k.step) {
      if (!((hd.my.valid >> i) & 1u)) continue;
      const P n = L::get(k.at + PIECE);
      if ((hd.my.begins >> i) & 1u) {
        h = L::make(0.0f, 0.0f);
        if (a.state_in) {
          const int64_t b = sequence(a, f, warp * RPW + i, !a.reverse);
          if (hd.in) h = get_state<L>(a.state_in + b * a.C + hd.c);
        }
      }
      P q = L::mul(L::mul(z[i], w[i]), L::sub(n, h));
      h = L::fma(w[i], h, L::mul(z[i], n));
      if ((hd.my.ends >> i) & 1u) {
        const P D = L::make(lds(k.at), L::V == 2 ? lds(k.at + 2 * PIECE) : 0.0f);
        q = L::mul(q, D), z[i] = L::mul(z[i], D), w[i] = L::mul(w[i], D);
      }
      sts(k.at, L::part(q, 0));
      if constexpr (L::V == 2) sts(k.at + PIECE, L::part(q, 1));
    }
  }
  __device__ __forceinline__ void finish(const GsArgs& a, Shared<L>* s, const Info& f, const Hand& hd, Walk k, P carry) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    P e = carry;
    for (int u = WARPS - 1; u > warp; --u)
      e = L::pick(s->has[1][u], s->agg_e[u][lane], L::fma(s->agg_a[u][lane], e, s->agg_e[u][lane]));
    const uint32_t begins = a.d_state_in ? hd.my.begins : 0u;
    const int64_t last = f.row0 + row_in(a, f, warp * RPW + RPW - 1);
    const int64_t step1 = a.reverse ? -a.dps : a.dps, step2 = a.reverse ? -a.dns : a.dns;
    T *dp = (T*)a.dp + last * a.dps + hd.c, *dn = (T*)a.dn + last * a.dns + hd.c;
    k.at += (RPW - 1) * k.step;
#pragma unroll
    for (int i = RPW - 1; i >= 0; --i, k.at -= k.step, dp -= step1, dn -= step2) {
      if (!((hd.my.valid >> i) & 1u)) continue;
      const P D = L::pick((hd.my.ends >> i) & 1u, L::make(1.0f, 1.0f), L::add(L::get(k.at + 2 * PIECE), e));
      const P q = L::make(lds(k.at), L::V == 2 ? lds(k.at + PIECE) : 0.0f);
      e = L::mul(w[i], D);
      if (hd.in) {
        L::put(dp, L::mul(q, D));
        L::put(dn, L::mul(z[i], D));
      }
      if ((begins >> i) & 1u) {
        const int64_t b = sequence(a, f, warp * RPW + i, !a.reverse);
        if (hd.in) put_state<L>(a.d_state_in + b * a.C + hd.c, e);
      }
    }
  }
};

template <class Pass, bool ALONE>
__global__ void __launch_bounds__(NT, Pass::CTAS) scan_kernel(const __grid_constant__ GsArgs a) {
  using L = typename Pass::L;
  using P = typename L::P;
  constexpr bool BACK = Pass::BACK;
  constexpr bool TWO = Pass::BUFS == 2 && !ALONE;       // the next part's rows come beside this one's
  constexpr int BUFFER = Pass::ARRAYS * PIECE, WORDS = sizeof(Info) / 4;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Shared<L>* s = reinterpret_cast<Shared<L>*>(smem_raw);
  uint8_t* smem = smem_raw + SHARED<L>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // sequences of no rows: what is before them is what is after them
  float* to = BACK ? a.d_state_in : a.state_out;
  const float* from = BACK ? a.d_state_out : a.state_in;
  if (to)
    for (int64_t b = (int64_t)blockIdx.x * WARPS + warp; b < a.n_seq; b += (int64_t)gridDim.x * WARPS)
      if (a.offs[b] >= a.offs[b + 1])
        for (int c = lane; c < a.C; c += 32) to[b * a.C + c] = from ? from[b * a.C + c] : 0.0f;
  if (a.n_rows == 0) return;
  if (threadIdx.x == 0) {
    sm100::mbar_init(smem_addr(&s->full[0]), 2);        // the rows and the Info
    sm100::mbar_init(smem_addr(&s->full[1]), 2);
    sm100::fence_mbar_init();
    s->abort = s->never = 0;
  }
  __syncthreads();
  const bool up = BACK != (a.reverse != 0);             // parts are taken from the last to the first
  const int64_t total = a.parts * a.blocks;
  const int64_t row_lo = clamp64(a.offs[0], 0, a.n_rows), row_hi = clamp64(a.offs[a.n_seq], 0, a.n_rows);
  volatile int *abort = &s->abort, *never = &s->never;
  auto part_of = [&](int64_t unit) { return up ? a.parts - 1 - unit / a.blocks : unit / a.blocks; };
  auto channel_of = [&](int64_t unit) { return (int)(unit % a.blocks) * 32 * L::V; };
  // warp 0: the Info in the lanes' words, the rows on their way, all of it arrived
  auto bring = [&](int buf, uint32_t info_word, int64_t row0, int count, int c0) {
    if (lane < WORDS) reinterpret_cast<uint32_t*>(&s->info[buf])[lane] = info_word;
    __syncwarp();
    if (lane == 0) {
      if (count > 0) fetch<L, BACK>(a, s, smem, buf, row0, c0);
      else sm100::mbar_arrive(smem_addr(&s->full[buf]));
      sm100::mbar_arrive(smem_addr(&s->full[buf]));
    }
  };
  auto bring_found = [&](int64_t k, int c0) {           // ALONE
    const Info f = find_part(a, k, lane);
    if (lane == 0) {
      s->info[0] = f;
      fetch<L, BACK>(a, s, smem, 0, f.row0, c0);
      sm100::mbar_arrive(smem_addr(&s->full[0]));
    }
  };

  int64_t unit = blockIdx.x, k = 0, own = 0;
  if constexpr (ALONE) {
    if (unit >= total) return;
    k = own = part_of(unit);
    if (warp == 0) bring_found(k, channel_of(unit));
  } else {
    if (warp == 0) {
      if (lane == 0) unit = (int64_t)atomicAdd(a.ticket, 1ull);
      unit = __shfl_sync(FULL, unit, 0);
      const bool more = unit < total;
      const uint32_t x = more && lane < WORDS ? reinterpret_cast<const uint32_t*>(a.info + part_of(unit))[lane] : 0u;
      const int64_t row0 = (int64_t)__shfl_sync(FULL, x, 0) | (int64_t)__shfl_sync(FULL, x, 1) << 32;
      bring(0, x, row0, __shfl_sync(FULL, x, 4), more ? channel_of(unit) : 0);
      if (lane == 0) s->start = unit;
    }
    __syncthreads();
    unit = s->start;
  }
  Pass pass;
  P carry = L::make(0.0f, 0.0f);
  bool ok = true, first = true;
  int n = 0;
  for (;; ++n) {
    const int buf = TWO ? n & 1 : 0;
    const uint32_t parity = TWO ? (n >> 1) & 1 : n & 1;
    int64_t next = total;
    if (!ALONE && threadIdx.x == 0 && unit < total) next = (int64_t)atomicAdd(a.ticket, 1ull);
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->full[buf]), parity, abort, a.limit_ns));
    if (!ok) break;
    const Info& f = s->info[buf];
    if (f.count == 0) break;
    if constexpr (!ALONE) k = part_of(unit);
    const bool inside = is_inside<BACK>(a, f, row_lo, row_hi);
    if constexpr (ALONE) {
      if (first && inside) {
        // what is before this part begins (BACK: ends) with its first position's sequence: from there on
        first = false;
        const int64_t r = f.row0 + row_in(a, f, BACK ? f.count - 1 : 0);
        __syncthreads();
        if (warp == 0) {
          const int64_t j = first_at_least(a.offs, a.n_seq + 1, r + 1, lane);
          int64_t p = own;
          if (j > 0 && j <= a.n_seq) {
            // (a row may be in the part after the one its place says)
            p = up ? clamp64(a.offs[j], 1, a.n_rows) / a.span + 1 : clamp64(a.offs[j - 1], 0, a.n_rows) / a.span;
            p = up ? clamp64(p, own, a.parts - 1) : clamp64(p, 0, own);
          }
          if (lane == 0) s->start = p;
          if (p != own) bring_found(p, channel_of(unit));
        }
        __syncthreads();
        k = s->start;
        if (k != own) continue;
      }
    }
    Hand h;
    h.k = k, h.c = channel_of(unit) + lane * L::V, h.in = h.c < a.C;
    h.my = mine_of(a, f, row_lo, row_hi, warp);
    const Walk walk = walk_of(a, f, smem + buf * BUFFER, h.my);
    const bool passing = ALONE && k != own;
    pass.sums(a, s, f, h, walk);
    meet();
    P fa = carry, fb = carry;
    bool has = false;
    uint32_t info_word = 0;
    if constexpr (ALONE) {
      if (passing) {
        joined<L, BACK>(s, lane, fa, fb, has);
        carry = L::pick(has, fb, L::fma(fa, carry, fb));
        sm100::fence_proxy_async_smem();   // (what was written into the buffer, before the next copy into it)
        meet();
        k += up ? -1 : 1;
        if (warp == 0) bring_found(k, channel_of(unit));
        continue;
      }
    } else if (warp == 0) {
      joined<L, BACK>(s, lane, fa, fb, has);
      if (h.in) leave_part<L>(a, k, h.c, fa, fb, has);
      next = __shfl_sync(FULL, next, 0);
      if (next < total && lane < WORDS) info_word = reinterpret_cast<const uint32_t*>(a.info + part_of(next))[lane];
    }
    pass.before_carry(a, s, f, h, walk);
    auto bring_next = [&] {
      if (warp != 0) return;
      const int64_t row0 = (int64_t)__shfl_sync(FULL, info_word, 0) | (int64_t)__shfl_sync(FULL, info_word, 1) << 32;
      bring(TWO ? buf ^ 1 : 0, info_word, row0, __shfl_sync(FULL, info_word, 4), next < total ? channel_of(next) : 0);
      if (lane == 0) s->start = next;
    };
    if constexpr (!ALONE) {
      if constexpr (TWO) bring_next();
      ok = carry_into<L, BACK>(a, s, h, inside, fa, fb, has, carry);
      if (!ok) break;
    }
    pass.finish(a, s, f, h, walk, carry);
    if constexpr (ALONE) break;
    sm100::fence_proxy_async_smem();       // (what was written into the buffer, before the next copy into it)
    meet();
    if constexpr (!TWO) {
      bring_next();
      meet();
    }
    unit = s->start;
  }
  if (!ok) {
    if (lane == 0 && atomicExch(&s->abort, 1) == 0) atomicAdd(a.expired, 1ull);
    // copies under way land before the CTA goes
    __syncthreads();
    if (threadIdx.x == 0)
      for (int i = n; i <= n + (TWO ? 1 : 0); ++i)
        sm100::mbar_wait(smem_addr(&s->full[TWO ? i & 1 : 0]), TWO ? (i >> 1) & 1 : i & 1, never, 200000000ull);
  }
}

// ---------------------------------------------------------------- a single row

struct StepArgs {
  const void *p, *n;
  void* out;
  int64_t ps, ns, os;
  const int32_t* slots;
  const float* state_in;
  float* state_out;
  int64_t n_seq, n_slots;
  int C, per;                              // per: 16-byte pieces of a row
};

// A thread has 16 bytes of a row; each value is read once and written once.
constexpr int STEP_NT = 256;

template <class T>
__global__ void __launch_bounds__(STEP_NT) step_kernel(const StepArgs a) {
  constexpr int VE = 16 / sizeof(T);
  const int64_t i = (int64_t)blockIdx.x * STEP_NT + threadIdx.x;
  if (i >= a.n_seq * a.per) return;
  // (a division of 32 bits where it does)
  const int64_t b = a.n_seq * a.per <= 0xffffffffll ? (int64_t)((uint32_t)i / (uint32_t)a.per) : i / a.per;
  const int c = (int)(i - b * a.per) * VE;
  const uint4 pu = *reinterpret_cast<const uint4*>((const T*)a.p + b * a.ps + c);
  const uint4 nu = *reinterpret_cast<const uint4*>((const T*)a.n + b * a.ns + c);
  uint4* out = reinterpret_cast<uint4*>((T*)a.out + b * a.os + c);
  const int64_t slot = a.slots ? a.slots[b] : b;
  float h[VE], p[VE], n[VE];
  if (slot < 0 || slot >= a.n_slots) {
#pragma unroll
    for (int e = 0; e < VE; ++e) h[e] = __uint_as_float(0x7fffffffu);
    *out = pack(h, T());
    return;
  }
  const float* from = a.state_in + slot * a.C + c;
#pragma unroll
  for (int e = 0; e < VE; e += 4) *reinterpret_cast<float4*>(&h[e]) = *reinterpret_cast<const float4*>(from + e);
  unpack(pu, p, T());
  unpack(nu, n, T());
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    float z, w;
    gate(p[e], z, w);
    h[e] = fmaf(w, h[e], z * n[e]);
  }
  float* to = a.state_out + slot * a.C + c;
#pragma unroll
  for (int e = 0; e < VE; e += 4) *reinterpret_cast<float4*>(to + e) = *reinterpret_cast<const float4*>(&h[e]);
  *out = pack(h, T());
}

// ---------------------------------------------------------------- the host's side

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return fn;
}

// [rows][channels] with a row stride, boxes of 128 bytes x TILE rows; zeros beyond the array.
bool make_map(CUtensorMap* m, int32_t dtype, const void* p, int64_t rows, int64_t channels, int64_t stride) {
  const auto fn = encode_fn();
  if (!fn) return false;
  const int size = type_size(dtype);
  const cuuint64_t dims[2] = {(cuuint64_t)channels, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * size};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / size), TILE}, step[2] = {1, 1};
  const CUtensorMapDataType type = dtype == TRACKFIT_FP32        ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == TRACKFIT_BF16_PROJ ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return fn(m, type, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool channels_ok(int32_t c) { return c >= 8 && c <= MAX_CHANNELS && c % 8 == 0; }

// Parts need not wait for one another where rows are few and sequences no longer than a part on
// average, or the parts are up to four; but with states after the call in the place of those before
// it a part may only read a state that no other writes yet, and does wait.
bool alone(int64_t n_rows, int64_t n_seq, bool in_place) {
  return n_rows <= TILE - SHIFT || (!in_place && (n_rows <= 4 * TILE || (n_rows <= FEW_ROWS && n_rows <= n_seq * TILE)));
}

// Rows from one part's place to the next: all of a part's, or, where a sequence has no more than 128 rows
// on average, as many as leave room for a part to begin earlier.  (By the counts alone: what a forward
// call saves goes by the same parts.)
int span_of(int64_t n_rows, int64_t n_seq) { return n_rows <= n_seq * TILE ? TILE - SHIFT : TILE; }
int64_t parts_at_most(int64_t n_rows) { return (n_rows + TILE - SHIFT - 1) / (TILE - SHIFT); }

size_t workspace_bytes(int64_t n_rows, int32_t channels) {
  if (n_rows <= TILE - SHIFT) return 0;
  return 256 + (size_t)parts_at_most(n_rows) * (sizeof(Info) + channels * sizeof(ulonglong2));
}

// A call of the scan, forward or backward.
struct Call {
  int32_t dtype;
  const void *p, *n, *g;                   // gate, cand; d_out (backward)
  int64_t ps, ns, gs;
  void* workspace;
  size_t size;
};

// The checks that forward and backward share.
int check(const Call& f, const GsArgs& a) {
  if (!type_ok(f.dtype) || a.n_rows < 0 || a.n_rows > (int64_t)1 << 40 || a.n_seq < 0 || a.n_seq >= 0x7fffffff)
    return TRACKFIT_ERR_INVALID_ARG;
  if (!channels_ok(a.C)) return TRACKFIT_ERR_UNSUPPORTED;
  if (a.reverse != 0 && a.reverse != 1) return TRACKFIT_ERR_INVALID_ARG;
  if (mis16(f.workspace)) return TRACKFIT_ERR_INVALID_ARG;
  if (a.n_seq == 0) return TRACKFIT_OK;
  if (!a.offs || (reinterpret_cast<uintptr_t>(a.offs) & 7u)) return TRACKFIT_ERR_INVALID_ARG;
  if (mis16(a.state_in) || mis16(a.state_out) || mis16(a.d_state_in) || mis16(a.d_state_out) || mis16(a.saved))
    return TRACKFIT_ERR_INVALID_ARG;
  const int sz = type_size(f.dtype);
  if (a.n_rows > 0 && (!rows_ok(f.p, f.ps, a.C, sz) || !rows_ok(f.n, f.ns, a.C, sz))) return TRACKFIT_ERR_INVALID_ARG;
  if (a.n_rows > 0x7fffff00) return TRACKFIT_ERR_UNSUPPORTED;    // a copy's coordinates have 32 bits
  const size_t need = workspace_bytes(a.n_rows, a.C);
  if (need > 0 && (!f.workspace || f.size < need)) return TRACKFIT_ERR_INVALID_ARG;
  return TRACKFIT_OK;
}

template <class Pass, bool ALONE>
int launch(const Call& f, GsArgs& a, cudaStream_t st) {
  using L = typename Pass::L;
  constexpr auto kern = scan_kernel<Pass, ALONE>;
  a.span = span_of(a.n_rows, a.n_seq), a.shift = TILE - a.span;
  a.parts = (a.n_rows + a.span - 1) / a.span, a.blocks = (a.C + 32 * L::V - 1) / (32 * L::V);
  a.limit_ns = operator_limit_ns(), a.expired = operator_expired();
  if (!a.expired) return TRACKFIT_ERR_CUDA;
  if (a.n_rows > 0 && (!make_map(&a.tp, f.dtype, f.p, a.n_rows, a.C, f.ps) || !make_map(&a.tn, f.dtype, f.n, a.n_rows, a.C, f.ns) ||
                       (Pass::BACK && !make_map(&a.tg, f.dtype, f.g, a.n_rows, a.C, f.gs))))
    return TRACKFIT_ERR_CUDA;
  const size_t smem = (ALONE ? 1 : Pass::BUFS) * Pass::ARRAYS * PIECE + SHARED<L>;
  const cudaError_t e = allow_smem<kern>(smem);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  int64_t grid = a.parts * a.blocks;
  if (!ALONE) {
    char* ws = (char*)f.workspace;
    a.ticket = (unsigned long long*)ws, a.info = (Info*)(ws + 256), a.words = (ulonglong2*)(a.info + a.parts);
    prepare_kernel<<<(unsigned)((a.parts + 7) / 8), 256, 0, st>>>(a);
    if (grid > 152 * Pass::CTAS) grid = 152 * Pass::CTAS;
  }
  if (grid < 1) grid = a.n_seq < 8 * 152 ? (a.n_seq + WARPS - 1) / WARPS : 152;    // states of empty sequences only
  kern<<<(unsigned)grid, NT, smem, st>>>(a);
  return launched();
}

template <template <class> class Pass, bool ALONE>
int by_type(const Call& f, GsArgs& a, cudaStream_t st) {
  return f.dtype == TRACKFIT_FP32        ? launch<Pass<float>, ALONE>(f, a, st)
         : f.dtype == TRACKFIT_BF16_PROJ ? launch<Pass<__nv_bfloat16>, ALONE>(f, a, st)
                                         : launch<Pass<__half>, ALONE>(f, a, st);
}
template <template <class> class Pass>
int by_rows(const Call& f, GsArgs& a, bool in_place, cudaStream_t st) {
  return alone(a.n_rows, a.n_seq, in_place) ? by_type<Pass, true>(f, a, st) : by_type<Pass, false>(f, a, st);
}

}  // namespace

extern "C" size_t trackfit_gated_scan_saved(int64_t n_rows, int32_t channels) {
  if (n_rows < 0 || n_rows > (int64_t)1 << 40 || !channels_ok(channels)) return 0;
  return (size_t)parts_at_most(n_rows) * channels * 4;
}

extern "C" size_t trackfit_gated_scan_workspace(int32_t dtype, int64_t n_rows, int64_t n_seq, int32_t channels) {
  if (!type_ok(dtype) || n_rows < 0 || n_rows > (int64_t)1 << 40 || n_seq < 0 || !channels_ok(channels)) return 0;
  return workspace_bytes(n_rows, channels);
}

extern "C" int trackfit_gated_scan(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                   int64_t cand_stride, int64_t n_rows, const int64_t* offsets, int64_t n_seq,
                                   int32_t channels, int32_t reverse, const float* state_in, float* state_out,
                                   float* saved, void* out, int64_t out_stride, void* workspace, size_t workspace_size,
                                   void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan");
  const Call f = {dtype, gate, cand, nullptr, gate_stride, cand_stride, 0, workspace, workspace_size};
  GsArgs a = {};
  a.out = out, a.os = out_stride;
  a.offs = offsets, a.n_rows = n_rows, a.n_seq = n_seq, a.C = channels, a.reverse = reverse;
  a.state_in = state_in, a.state_out = state_out, a.saved = saved;
  const int rc = check(f, a);
  if (rc != TRACKFIT_OK || n_seq == 0) return rc;
  if (n_rows > 0 && !rows_ok(out, out_stride, channels, type_size(dtype))) return TRACKFIT_ERR_INVALID_ARG;
  return by_rows<Forward>(f, a, state_out && state_out == state_in, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int trackfit_gated_scan_backward(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                            int64_t cand_stride, int64_t n_rows, const int64_t* offsets,
                                            int64_t n_seq, int32_t channels, int32_t reverse, const float* state_in,
                                            const float* saved, const void* d_out, int64_t d_out_stride,
                                            const float* d_state_out, float* d_state_in, void* d_gate,
                                            int64_t d_gate_stride, void* d_cand, int64_t d_cand_stride, void* workspace,
                                            size_t workspace_size, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan_backward");
  const Call f = {dtype, gate, cand, d_out, gate_stride, cand_stride, d_out_stride, workspace, workspace_size};
  GsArgs a = {};
  a.dp = d_gate, a.dps = d_gate_stride, a.dn = d_cand, a.dns = d_cand_stride;
  a.offs = offsets, a.n_rows = n_rows, a.n_seq = n_seq, a.C = channels, a.reverse = reverse;
  a.state_in = state_in, a.saved = const_cast<float*>(saved), a.d_state_out = d_state_out, a.d_state_in = d_state_in;
  const int rc = check(f, a);
  if (rc != TRACKFIT_OK || n_seq == 0) return rc;
  const int sz = type_size(dtype);
  if (n_rows > 0 && (!saved || !rows_ok(d_out, d_out_stride, channels, sz) || !rows_ok(d_gate, d_gate_stride, channels, sz) ||
                     !rows_ok(d_cand, d_cand_stride, channels, sz)))
    return TRACKFIT_ERR_INVALID_ARG;
  return by_rows<Backward>(f, a, d_state_in && d_state_in == d_state_out, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int trackfit_gated_scan_step(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                        int64_t cand_stride, int64_t n_seq, int32_t channels, const int32_t* slots,
                                        int64_t n_slots, const float* state_in, float* state_out, void* out,
                                        int64_t out_stride, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan_step");
  if (!type_ok(dtype) || n_seq < 0 || n_seq > 0x7fffffff || n_slots < 0) return TRACKFIT_ERR_INVALID_ARG;
  if (!channels_ok(channels)) return TRACKFIT_ERR_UNSUPPORTED;
  if (!slots && n_slots < n_seq) return TRACKFIT_ERR_INVALID_ARG;
  if (n_seq == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!rows_ok(gate, gate_stride, channels, sz) || !rows_ok(cand, cand_stride, channels, sz) ||
      !rows_ok(out, out_stride, channels, sz))
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(slots) || !state_in || !state_out || mis16(state_in) || mis16(state_out)) return TRACKFIT_ERR_INVALID_ARG;
  StepArgs a;
  a.p = gate, a.ps = gate_stride, a.n = cand, a.ns = cand_stride, a.out = out, a.os = out_stride;
  a.slots = slots, a.state_in = state_in, a.state_out = state_out, a.n_seq = n_seq, a.n_slots = n_slots;
  a.C = channels, a.per = channels * sz / 16;
  const int64_t grid = (n_seq * a.per + STEP_NT - 1) / STEP_NT;
  if (grid > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) step_kernel<float><<<(unsigned)grid, STEP_NT, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) step_kernel<__nv_bfloat16><<<(unsigned)grid, STEP_NT, 0, st>>>(a);
  else step_kernel<__half><<<(unsigned)grid, STEP_NT, 0, st>>>(a);
  return launched();
}
