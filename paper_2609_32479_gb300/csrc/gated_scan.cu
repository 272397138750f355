// The gated recurrence over packed sequences and its gradients.
//
//   z = sigma(p), w = 1 - z,  h_t = w_t h_{t-1} + z_t n_t
//   back, from the direction's last row to its first:
//   D_t = g_t + e_t,  e_{t-1} = w_t D_t,  dn = z D,  dp = z w (n - h_{t-1}) D
//
// Bound by memory: three values a row and channel are moved forward, five backward.  Rows are taken
// in the order of the recurrence ("positions"), 128 at a time, a part of 128 bytes of channels by a
// CTA of 8 warps of 16 positions each; a lane has one channel (16 bits: two neighbouring ones).  A
// ninth warp brings the rows of the part after it, by TMA, and where sequences begin among them.
//
// What stands before a run of positions acts on it through one number a channel: h_last = A h_before
// + B, with A the product of the w.  A warp forms (A, B) of its rows, the CTA those of the part, and
//   h after part k = A_k (h after part k - 1) + B_k
// goes from part to part: through the workspace, in which a part leaves (A, B) as soon as it has
// them and h when it knows it.  A part looks back at up to WINDOW parts for one with h and then
// applies the (A, B) of those between, in their order: the result does not depend on when it
// looked.  Each word carries what it holds beside its 32 bits, so no fence is needed; parts are
// taken in order from a counter, so those a CTA waits for are done or under way.  A sequence's first
// row ends the look back: what came before it is left out by choice, not multiplied by 0 (it may
// not be finite).
//
// Few rows in short sequences: every part forms what is before it again from its sequence's first
// row on, by the same operations, and no workspace has to be cleared and no part is waited for.
#include "seq_ops.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>

namespace {
using namespace seqops;

constexpr int TILE = 128;                  // positions of a part, and from one saved state to the next
constexpr int WARPS = 8, RPW = TILE / WARPS;
constexpr int NT = (WARPS + 1) * 32;       // the ninth warp brings the rows
constexpr int PIECE = TILE * 128;          // bytes of one array of a part
constexpr int MAX_CHANNELS = 1 << 16;
constexpr int64_t FEW_ROWS = 4096;
constexpr int CTAS = 2;                    // of an SM
constexpr uint32_t PARTIAL = 1, WHOLE = 2; // what a word of the workspace holds

// Of a part, found before the parts' kernel: the number of the first offset at or behind its first row,
// and Marks::bound.
struct PartInfo {
  long long first;
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
  int blocks;                              // CTAs side by side in a part
  unsigned long long* ticket;
  PartInfo* info;                          // [parts]
  ulonglong2* words;                       // [parts][C]: A and B or h
  uint64_t limit_ns;
  unsigned long long* expired;
};

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

// Where sequences begin and end among the rows of a part.  Row r0 + i stands for bit i, i <= TILE.
struct Marks {
  uint32_t bound[6];                       // an offset equals the row
  int first[TILE + 1], last[TILE + 1];     // the least and the largest number of such an offset (with states)
};
enum { END = 0, PASS = 1, OWN = 2 };       // of what the ninth warp brings: no more, a part before this CTA's, a part
struct Brought {
  long long k;
  int c0, kind;
  Marks marks;
};

template <class L>
struct Shared {
  static constexpr int WIN = 32 / L::V;    // parts looked back at
  typename L::P agg_a[WARPS][32], agg_b[WARPS][32];   // A and B of the warps' rows
  typename L::P win_a[WIN][32], win_b[WIN][32];       // of the parts before, nearest first
  uint32_t has[WARPS];                     // a warp's rows hold a sequence's beginning: A does not count
  uint32_t status[WIN];
  Brought brought[2];
  uint64_t full[2], marked[2], empty[2];
  long long lo, hi;                        // rows of sequences
  int from;
  int abort, never;
};

// The buffers come behind it: a part of fewer rows, taken backwards, has positions whose rows would lie
// up to 15 rows below its buffer; they are read there with the others and not used.
template <class L>
constexpr int SHARED = ((int)sizeof(Shared<L>) + 1023) / 1024 * 1024;

// The rows of a part.
struct Part {
  int64_t row0;                            // the lowest; positions go backwards from the highest with `reverse`
  int count;
  int lo, hi;                              // those of sequences, as distances from row0
};

template <class S>
__device__ __forceinline__ Part part_of(const GsArgs& a, const S* s, int64_t k) {
  Part t;
  const int64_t pos0 = k * TILE;
  t.count = a.n_rows - pos0 < TILE ? (int)(a.n_rows - pos0) : TILE;
  t.row0 = a.reverse ? a.n_rows - pos0 - t.count : pos0;
  t.lo = (int)clamp64(s->lo - t.row0, 0, t.count), t.hi = (int)clamp64(s->hi - t.row0, 0, t.count);
  return t;
}
// Position i of a part -> its row, as a distance from row0.
__device__ __forceinline__ int row_in(const GsArgs& a, const Part& t, int i) { return a.reverse ? t.count - 1 - i : i; }

__device__ __forceinline__ bool bound(const Marks& m, int d) { return (m.bound[d >> 5] >> (d & 31)) & 1u; }
// 16 of the bits from number `low` on (below 0: zeros).
__device__ __forceinline__ uint32_t bits16(const Marks& m, int low) {
  if (low <= -16) return 0;
  const int l = low < 0 ? 0 : low, w = l >> 5;
  const uint32_t x = __funnelshift_r(m.bound[w], m.bound[w + 1 < 6 ? w + 1 : 5], l & 31);
  return (low < 0 ? x << -low : x) & 0xffffu;
}
// Of a warp's 16 positions, bit i for the i-th: rows of sequences, first rows, last rows.
struct Mine {
  uint32_t valid, begins, ends;
};
__device__ __forceinline__ Mine mine_of(const GsArgs& a, const Part& t, const Marks& m, int warp) {
  const int i0 = warp * RPW;
  const int lo = (a.reverse ? t.count - t.hi : t.lo) - i0, hi = (a.reverse ? t.count - t.lo : t.hi) - i0;
  Mine r;
  r.valid = (hi <= 0 ? 0u : hi >= RPW ? 0xffffu : (1u << hi) - 1u) & (lo <= 0 ? 0xffffu : lo >= RPW ? 0u : 0xffffu << lo);
  if (a.reverse) {   // position i is row count - 1 - i: it begins with the row's upper border
    r.begins = __brev(bits16(m, t.count - i0 - RPW + 1)) >> 16;
    r.ends = __brev(bits16(m, t.count - i0 - RPW)) >> 16;
  } else {
    r.begins = bits16(m, i0), r.ends = bits16(m, i0 + 1);
  }
  r.begins &= r.valid, r.ends &= r.valid;
  return r;
}
// The sequence of a row that is its first (or last), by the row's lower or upper border.
__device__ __forceinline__ int64_t sequence(const GsArgs& a, const Marks& m, int d, bool lower) {
  return clamp64(lower ? m.last[d] : (int64_t)m.first[d + 1] - 1, 0, a.n_seq - 1);
}

// The bits of the offsets from number j on among `count` rows from row0 on: a whole warp; `each`
// gets every number and its row.
template <class F>
__device__ __forceinline__ void bounds_of(const GsArgs& a, int64_t j, int64_t row0, int count, int lane, uint32_t (&bits)[5],
                                          F&& each) {
#pragma unroll
  for (int w = 0; w < 5; ++w) bits[w] = 0;
  for (;; j += 32) {
    const int64_t d = j + lane <= a.n_seq ? a.offs[j + lane] - row0 : INT64_MAX;
    const bool here = d >= 0 && d <= count;
#pragma unroll
    for (int w = 0; w < 5; ++w) bits[w] |= __reduce_or_sync(FULL, here && (d >> 5) == w ? 1u << (d & 31) : 0u);
    if (here) each(j + lane, (int)d);
    if (__any_sync(FULL, d > count)) break;
  }
}

// Before the parts' kernel: the workspace cleared, and each part's sequences found; a warp a part.
__global__ void __launch_bounds__(256) prepare_kernel(const __grid_constant__ GsArgs a) {
  const int64_t k = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  if (k >= a.parts) return;
  if (k == 0 && lane == 0) *a.ticket = 0;
  for (int c = lane; c < a.C; c += 32) a.words[k * a.C + c] = make_ulonglong2(0, 0);
  const int64_t pos0 = k * TILE;
  const int count = a.n_rows - pos0 < TILE ? (int)(a.n_rows - pos0) : TILE;
  const int64_t row0 = a.reverse ? a.n_rows - pos0 - count : pos0;
  const int64_t j = first_at_least(a.offs, a.n_seq + 1, row0, lane);
  uint32_t bits[5];
  bounds_of(a, j, row0, count, lane, bits, [](int64_t, int) {});
  if (lane == 0) {
    PartInfo f;
    f.first = j;
#pragma unroll
    for (int w = 0; w < 5; ++w) f.bound[w] = bits[w];
    f.bound[5] = 0;
    a.info[k] = f;
  }
}

// The ninth warp: the rows of one part after the other, ahead of the warps that compute.
template <class T, bool BACK, bool ALONE, class S>
__device__ __forceinline__ void bring(const GsArgs& a, S* s, uint8_t* smem) {
  constexpr int ARRAYS = BACK ? 3 : 2, WIDE = 32 * Lane<T>::V;
  const int lane = threadIdx.x & 31;
  const int64_t total = a.parts * a.blocks;
  const bool numbers = a.state_in || a.state_out || a.d_state_in || a.d_state_out;
  volatile int *abort = &s->abort, *never = &s->never;
  int64_t unit = blockIdx.x, k = 0, own = 0;
  if constexpr (!ALONE) {
    if (lane == 0) unit = (int64_t)atomicAdd(a.ticket, 1ull);
    unit = __shfl_sync(FULL, unit, 0);
  } else {
    // from the part in which the sequence of this part's first position (BACK: last position) begins (ends)
    k = own = BACK ? a.parts - 1 - unit / a.blocks : unit / a.blocks;
    const Part t = part_of(a, s, k);
    const int64_t r = t.row0 + row_in(a, t, BACK ? t.count - 1 : 0);
    const int64_t j = first_at_least(a.offs, a.n_seq + 1, r + 1, lane);     // the first offset beyond the row
    if (j > 0 && j <= a.n_seq) {
      const int64_t o = clamp64(a.offs[BACK != (a.reverse != 0) ? j : j - 1], 0, a.n_rows);
      int64_t pos;                                                           // the first (last) position
      if constexpr (BACK) pos = a.reverse ? a.n_rows - 1 - o : o - 1;
      else pos = a.reverse ? a.n_rows - o : o;
      pos = clamp64(pos, 0, a.n_rows - 1) / TILE;
      if (BACK ? pos > own : pos < own) k = pos;
    }
  }
  int n = 0;
  bool ok = true, more = unit < total;
  for (;; ++n) {
    const int buf = n & 1;
    Brought& b = s->brought[buf];
    const uint32_t full = smem_addr(&s->full[buf]), marked = smem_addr(&s->marked[buf]);
    int64_t next = 0;
    if (!ALONE && more && lane == 0) next = (int64_t)atomicAdd(a.ticket, 1ull);   // (used in the next round)
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->empty[buf]), ((n >> 1) & 1) ^ 1u, abort, a.limit_ns));
    if (!ok || !more) break;
    if constexpr (!ALONE) k = BACK ? a.parts - 1 - unit / a.blocks : unit / a.blocks;
    const int c0 = (int)(unit % a.blocks) * WIDE;
    const Part t = part_of(a, s, k);
    if (lane == 0) {
      const uint32_t to = smem_addr(smem + buf * ARRAYS * PIECE);
      sm100::mbar_arrive_expect_tx(full, ARRAYS * PIECE);
      sm100::tma_load_2d(to, &a.tp, full, c0, (int)t.row0);
      sm100::tma_load_2d(to + PIECE, &a.tn, full, c0, (int)t.row0);
      if constexpr (BACK) sm100::tma_load_2d(to + 2 * PIECE, &a.tg, full, c0, (int)t.row0);
      b.k = k, b.c0 = c0, b.kind = ALONE && k != own ? PASS : OWN;
    }
    if (!ALONE && !numbers) {
      if (lane < 6) b.marks.bound[lane] = a.info[k].bound[lane];
    } else {
      const int64_t j = ALONE ? first_at_least(a.offs, a.n_seq + 1, t.row0, lane) : (int64_t)a.info[k].first;
      if (numbers) {
        for (int i = lane; i <= TILE; i += 32) b.marks.first[i] = 0x7fffffff, b.marks.last[i] = -1;
        __syncwarp();
      }
      uint32_t bits[5];
      bounds_of(a, j, t.row0, t.count, lane, bits, [&](int64_t j, int d) {
        if (numbers) atomicMin(&b.marks.first[d], (int)j), atomicMax(&b.marks.last[d], (int)j);
      });
#pragma unroll
      for (int w = 0; w < 5; ++w)
        if (lane == w) b.marks.bound[w] = bits[w];
    }
    __syncwarp();
    if (lane == 0) sm100::mbar_arrive(marked);
    if constexpr (ALONE) {
      more = k != own;
      k += BACK ? -1 : 1;
    } else {
      unit = __shfl_sync(FULL, next, 0);
      more = unit < total;
    }
  }
  if (ok) {
    if (lane == 0) {
      s->brought[n & 1].kind = END;
      sm100::mbar_arrive(smem_addr(&s->marked[n & 1]));
    }
  } else if (lane == 0) {
    for (int i = n < 2 ? 0 : n - 2; i < n; ++i)   // the copies under way land before the CTA goes
      sm100::mbar_wait(smem_addr(&s->full[i & 1]), (i >> 1) & 1, never, 200000000ull);
  }
  __syncwarp();
}

// The barriers and what all parts need, by all threads.
template <class S>
__device__ __forceinline__ void begin(const GsArgs& a, S* s) {
  if (threadIdx.x == 0) {
    for (int b = 0; b < 2; ++b) {
      sm100::mbar_init(smem_addr(&s->full[b]), 1);
      sm100::mbar_init(smem_addr(&s->marked[b]), 1);
      sm100::mbar_init(smem_addr(&s->empty[b]), WARPS);
    }
    sm100::fence_mbar_init();
    s->abort = s->never = 0;
    s->lo = clamp64(a.offs[0], 0, a.n_rows), s->hi = clamp64(a.offs[a.n_seq], 0, a.n_rows);
  }
  __syncthreads();
}
// Among the warps that compute.
__device__ __forceinline__ void meet() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// The warps' (A, B), in their order (BACK: the last first), as one; A does not count if `has`.
template <class L, bool BACK>
__device__ __forceinline__ void joined(const Shared<L>* s, int lane, typename L::P& fa, typename L::P& fb, bool& has) {
  fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f), has = false;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    const int u = BACK ? WARPS - 1 - i : i;
    const typename L::P ga = s->agg_a[u][lane], gb = s->agg_b[u][lane];
    const bool h = s->has[u];
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

// What the parts before part k (BACK: behind it) leave for this CTA's channels: false if the wait for
// them expired.  All warps that compute; `in`: the lane has channels, c the first of them.
template <class L, bool BACK>
__device__ __forceinline__ bool look_back(const GsArgs& a, Shared<L>* s, int64_t k, int c, bool in, typename L::P& carry) {
  constexpr int V = L::V, WIN = Shared<L>::WIN, EACH = WIN / WARPS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t there = BACK ? a.parts - 1 - k : k;           // so many parts there are
  uint64_t t0 = 0;
  for (int round = 0;; ++round) {
    ulonglong2 u[EACH][V];                                    // all under way before the first is used
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int d = warp * EACH + i;
      const int64_t at = BACK ? k + 1 + d : k - 1 - d;
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

__device__ __forceinline__ float lds(uint32_t at) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void sts(uint32_t at, float x) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory"); }

// The barrier between what a warp has read of a buffer and the next copy into it.
template <class S>
__device__ __forceinline__ void release(S* s, int buf, int lane) {
  __syncwarp();
  if (lane == 0) sm100::mbar_arrive(smem_addr(&s->empty[buf]));
}

// The carry into the part, given the warps' (A, B): false if a wait expired.  ALONE: `carry` is already
// what the parts before have made of it.
template <class L, bool BACK, bool ALONE>
__device__ __forceinline__ bool carry_into(const GsArgs& a, Shared<L>* s, int64_t k, int c, bool in, const Part& t,
                                           const Marks& m, typename L::P& carry) {
  if constexpr (ALONE) return true;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // what is before this part counts if its first position is a row within a sequence
  const int d = row_in(a, t, BACK ? t.count - 1 : 0);
  const bool inside = d >= t.lo && d < t.hi && !bound(m, BACK != (a.reverse != 0) ? d + 1 : d);
  typename L::P fa, fb;
  bool has = false;
  if (warp == 0) {
    joined<L, BACK>(s, lane, fa, fb, has);
    if (in) leave_part<L>(a, k, c, fa, fb, has);
  }
  carry = L::make(0.0f, 0.0f);
  if (!inside) return true;
  if (!look_back<L, BACK>(a, s, k, c, in, carry)) return false;
  if (warp == 0 && in && !has) {
    const typename L::P h = L::fma(fa, carry, fb);
#pragma unroll
    for (int v = 0; v < L::V; ++v) leave(&a.words[k * a.C + c + v].y, word(WHOLE, L::part(h, v)));
  }
  return true;
}

static_assert(sizeof(Shared<Lane<float>>) >= RPW * 128, "room below the buffers");

// ---------------------------------------------------------------- forward

// A and B of the warp's rows; of each row w and z n (KEEP_Z: z).  At a sequence's first
// row z n is its h: the state before is read once only, since the CTA with the sequence's end may write
// the state after it to the same place as soon as this part has left its B.
// (Rows of no sequence are computed with: none of a sequence's comes after them without its first.)
template <class L, bool KEEP_Z>
__device__ __forceinline__ void rows_forward(const GsArgs& a, const Part& t, const Marks& m, const Mine& my, uint32_t at,
                                             int step, int c, bool in, typename L::P (&z)[RPW], typename L::P (&w)[RPW],
                                             typename L::P& fa, typename L::P& fb) {
  using P = typename L::P;
  fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < RPW; ++i, at += step) {
    const P p = L::get(at), n = L::get(at + PIECE);
    const bool begins = (my.begins >> i) & 1u;
    L::gates(p, z[i], w[i]);
    const P x = L::mul(z[i], n);
    if (begins) {
      fb = L::make(0.0f, 0.0f);
      if (a.state_in && in)
        fb = get_state<L>(a.state_in + sequence(a, m, row_in(a, t, (threadIdx.x >> 5) * RPW + i), !a.reverse) * a.C + c);
    }
    fa = L::mul(fa, w[i]);
    fb = L::fma(w[i], fb, x);
    if constexpr (!KEEP_Z) z[i] = L::pick(begins, fb, x);
  }
}

template <class T, bool ALONE>
__global__ void __launch_bounds__(NT, CTAS) scan_kernel(const __grid_constant__ GsArgs a) {
  using L = Lane<T>;
  using P = typename L::P;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Shared<L>* s = reinterpret_cast<Shared<L>*>(smem_raw);
  uint8_t* smem = smem_raw + SHARED<L>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // sequences of no rows: what is before them is what is after them
  if (a.state_out)
    for (int64_t b = (int64_t)blockIdx.x * (WARPS + 1) + warp; b < a.n_seq; b += (int64_t)gridDim.x * (WARPS + 1))
      if (a.offs[b] >= a.offs[b + 1])
        for (int c = lane; c < a.C; c += 32) a.state_out[b * a.C + c] = a.state_in ? a.state_in[b * a.C + c] : 0.0f;
  if (a.n_rows == 0) return;
  begin(a, s);
  if (warp == WARPS) {
    bring<T, false, ALONE>(a, s, smem);
    return;
  }
  volatile int* abort = &s->abort;
  P carry = L::make(0.0f, 0.0f);
  bool ok = true;
  for (int n = 0;; ++n) {
    const int buf = n & 1;
    Brought& b = s->brought[buf];
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->marked[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok || b.kind == END) break;
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->full[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok) break;
    const int64_t k = b.k;
    const int c = b.c0 + lane * L::V;
    const bool in = c < a.C, pass = ALONE && b.kind == PASS;
    const Part t = part_of(a, s, k);
    const Marks& m = b.marks;
    const Mine my = mine_of(a, t, m, warp);
    const int d0 = row_in(a, t, warp * RPW), dir = a.reverse ? -1 : 1;
    const uint32_t at = smem_addr(smem + buf * 2 * PIECE) + (my.valid ? d0 * 128 + lane * 4 : 0);
    P x[RPW], w[RPW], fa, fb;
    rows_forward<L, false>(a, t, m, my, at, my.valid ? 128 * dir : 0, c, in, x, w, fa, fb);
    s->agg_a[warp][lane] = fa, s->agg_b[warp][lane] = fb;
    if (lane == 0) s->has[warp] = my.begins != 0;
    meet();
    if (pass) {
      bool has;
      joined<L, false>(s, lane, fa, fb, has);
      carry = L::pick(has, fb, L::fma(fa, carry, fb));
      release(s, buf, lane);
      meet();
      continue;
    }
    ok = carry_into<L, false, ALONE>(a, s, k, c, in, t, m, carry);
    if (!ok) break;
    if (a.saved && warp == 0 && in) put_state<L>(a.saved + k * a.C + c, carry);
    P h = carry;
    for (int u = 0; u < warp; ++u) h = L::pick(s->has[u], s->agg_b[u][lane], L::fma(s->agg_a[u][lane], h, s->agg_b[u][lane]));
    const uint32_t put = in ? my.valid : 0u, ends = in && a.state_out ? my.ends : 0u;
    T* out = (T*)a.out + (t.row0 + d0) * a.os + c;
    const int64_t step = dir * a.os;
#pragma unroll
    for (int i = 0; i < RPW; ++i, out += step) {
      h = L::pick((my.begins >> i) & 1u, x[i], L::fma(w[i], h, x[i]));
      if ((put >> i) & 1u) L::put(out, h);
      if ((ends >> i) & 1u) put_state<L>(a.state_out + sequence(a, m, row_in(a, t, warp * RPW + i), a.reverse) * a.C + c, h);
    }
    release(s, buf, lane);
    meet();
  }
  if (!ok && lane == 0 && atomicExch(&s->abort, 1) == 0) atomicAdd(a.expired, 1ull);
}

// ---------------------------------------------------------------- backward

template <class T, bool ALONE>
__global__ void __launch_bounds__(NT, CTAS) backward_kernel(const __grid_constant__ GsArgs a) {
  using L = Lane<T>;
  using P = typename L::P;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Shared<L>* s = reinterpret_cast<Shared<L>*>(smem_raw);
  uint8_t* smem = smem_raw + SHARED<L>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // sequences of no rows: what is behind them is what is before them
  if (a.d_state_in)
    for (int64_t b = (int64_t)blockIdx.x * (WARPS + 1) + warp; b < a.n_seq; b += (int64_t)gridDim.x * (WARPS + 1))
      if (a.offs[b] >= a.offs[b + 1])
        for (int c = lane; c < a.C; c += 32) a.d_state_in[b * a.C + c] = a.d_state_out ? a.d_state_out[b * a.C + c] : 0.0f;
  if (a.n_rows == 0) return;
  begin(a, s);
  if (warp == WARPS) {
    bring<T, true, ALONE>(a, s, smem);
    return;
  }
  volatile int* abort = &s->abort;
  P carry = L::make(0.0f, 0.0f);
  bool ok = true;
  for (int n = 0;; ++n) {
    const int buf = n & 1;
    Brought& b = s->brought[buf];
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->marked[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok || b.kind == END) break;
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->full[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok) break;
    const int64_t k = b.k;
    const int c = b.c0 + lane * L::V;
    const bool in = c < a.C, pass = ALONE && b.kind == PASS;
    const Part t = part_of(a, s, k);
    const Marks& m = b.marks;
    const Mine my = mine_of(a, t, m, warp);
    const int d0 = row_in(a, t, warp * RPW), dir = a.reverse ? -1 : 1;
    const uint32_t at0 = smem_addr(smem + buf * 3 * PIECE) + (my.valid ? d0 * 128 + lane * 4 : 0);
    const int step0 = my.valid ? 128 * dir : 0;
    P z[RPW], w[RPW], fa, fb;
    {
      // the states again, from the one saved before the part
      rows_forward<L, true>(a, t, m, my, at0, step0, c, in, z, w, fa, fb);
      s->agg_a[warp][lane] = fa, s->agg_b[warp][lane] = fb;
      if (lane == 0) s->has[warp] = my.begins != 0;
      P h = L::make(0.0f, 0.0f);
      if (in) h = get_state<L>(a.saved + k * a.C + c);
      meet();
      for (int u = 0; u < warp; ++u) h = L::pick(s->has[u], s->agg_b[u][lane], L::fma(s->agg_a[u][lane], h, s->agg_b[u][lane]));
      // z w (n - h) takes the place of p and n, 4 bytes a channel
      uint32_t at = at0;
      if (my.valid) {
#pragma unroll
        for (int i = 0; i < RPW; ++i, at += step0) {
          const P n = L::get(at + PIECE);
          if ((my.begins >> i) & 1u) {
            h = L::make(0.0f, 0.0f);
            if (a.state_in && in)
              h = get_state<L>(a.state_in + sequence(a, m, row_in(a, t, warp * RPW + i), !a.reverse) * a.C + c);
          }
          const P q = L::mul(L::mul(z[i], w[i]), L::sub(n, h));
          h = L::fma(w[i], h, L::mul(z[i], n));
          if ((my.valid >> i) & 1u) {
            sts(at, L::part(q, 0));
            if constexpr (L::V == 2) sts(at + PIECE, L::part(q, 1));
          }
        }
      }
      meet();
    }
    // what comes from behind: e before the warp's rows = A e after them + B.  A sequence's last row gets
    // its results here: what its state's gradient is may be written over once this part has left its B.
    fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f);
    if (my.valid) {
      uint32_t at = at0 + (RPW - 1) * step0;
#pragma unroll
      for (int i = RPW - 1; i >= 0; --i, at -= step0) {
        if (!((my.valid >> i) & 1u)) continue;
        const bool ends = (my.ends >> i) & 1u;
        if (ends) {
          fb = L::make(0.0f, 0.0f);
          if (a.d_state_out && in)
            fb = get_state<L>(a.d_state_out + sequence(a, m, row_in(a, t, warp * RPW + i), a.reverse) * a.C + c);
        }
        const P D = L::add(L::get(at + 2 * PIECE), fb);
        fa = L::mul(fa, w[i]), fb = L::mul(w[i], D);
        if (ends) {
          z[i] = L::mul(z[i], D), w[i] = fb;
          sts(at, lds(at) * L::part(D, 0));
          if constexpr (L::V == 2) sts(at + PIECE, lds(at + PIECE) * L::part(D, 1));
        }
      }
    }
    s->agg_a[warp][lane] = fa, s->agg_b[warp][lane] = fb;
    if (lane == 0) s->has[warp] = my.ends != 0;
    meet();
    if (pass) {
      bool has;
      joined<L, true>(s, lane, fa, fb, has);
      carry = L::pick(has, fb, L::fma(fa, carry, fb));
      release(s, buf, lane);
      meet();
      continue;
    }
    ok = carry_into<L, true, ALONE>(a, s, k, c, in, t, m, carry);
    if (!ok) break;
    P e = carry;
    for (int u = WARPS - 1; u > warp; --u)
      e = L::pick(s->has[u], s->agg_b[u][lane], L::fma(s->agg_a[u][lane], e, s->agg_b[u][lane]));
    const uint32_t put = in ? my.valid : 0u, begins = in && a.d_state_in ? my.begins : 0u;
    const int64_t step1 = dir * a.dps, step2 = dir * a.dns;
    T* dp = (T*)a.dp + (t.row0 + d0) * a.dps + (RPW - 1) * step1 + c;
    T* dn = (T*)a.dn + (t.row0 + d0) * a.dns + (RPW - 1) * step2 + c;
    if (my.valid) {
      uint32_t at = at0 + (RPW - 1) * step0;
#pragma unroll
      for (int i = RPW - 1; i >= 0; --i, at -= step0, dp -= step1, dn -= step2) {
        if (!((my.valid >> i) & 1u)) continue;
        const P D = L::pick((my.ends >> i) & 1u, L::make(1.0f, 1.0f), L::add(L::get(at + 2 * PIECE), e));
        const P q = L::make(lds(at), L::V == 2 ? lds(at + PIECE) : 0.0f);
        e = L::mul(w[i], D);
        if ((put >> i) & 1u) {
          L::put(dp, L::mul(q, D));
          L::put(dn, L::mul(z[i], D));
        }
        if ((begins >> i) & 1u)
          put_state<L>(a.d_state_in + sequence(a, m, row_in(a, t, warp * RPW + i), !a.reverse) * a.C + c, e);
      }
    }
    release(s, buf, lane);
    meet();
  }
  if (!ok && lane == 0 && atomicExch(&s->abort, 1) == 0) atomicAdd(a.expired, 1ull);
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
  return n_rows <= TILE || (!in_place && (n_rows <= 4 * TILE || (n_rows <= FEW_ROWS && n_rows <= n_seq * TILE)));
}

size_t workspace_bytes(int64_t n_rows, int32_t channels) {
  if (n_rows <= TILE) return 0;
  return 256 + (size_t)((n_rows + TILE - 1) / TILE) * (sizeof(PartInfo) + channels * sizeof(ulonglong2));
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

template <class T, bool BACK, bool ALONE>
int launch(const Call& f, GsArgs& a, cudaStream_t st) {
  constexpr int V = Lane<T>::V;
  constexpr auto kern = [] {
    if constexpr (BACK) return &backward_kernel<T, ALONE>;
    else return &scan_kernel<T, ALONE>;
  }();
  a.parts = (a.n_rows + TILE - 1) / TILE, a.blocks = (a.C + 32 * V - 1) / (32 * V);
  a.limit_ns = operator_limit_ns(), a.expired = operator_expired();
  if (!a.expired) return TRACKFIT_ERR_CUDA;
  if (a.n_rows > 0 && (!make_map(&a.tp, f.dtype, f.p, a.n_rows, a.C, f.ps) || !make_map(&a.tn, f.dtype, f.n, a.n_rows, a.C, f.ns) ||
                       (BACK && !make_map(&a.tg, f.dtype, f.g, a.n_rows, a.C, f.gs))))
    return TRACKFIT_ERR_CUDA;
  const size_t smem = (BACK ? 6 : 4) * PIECE + SHARED<Lane<T>>;
  const cudaError_t e = allow_smem<kern>(smem);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  int64_t grid = a.parts * a.blocks;
  if (!ALONE) {
    char* ws = (char*)f.workspace;
    a.ticket = (unsigned long long*)ws, a.info = (PartInfo*)(ws + 256), a.words = (ulonglong2*)(a.info + a.parts);
    prepare_kernel<<<(unsigned)((a.parts + 7) / 8), 256, 0, st>>>(a);
    if (grid > 152 * CTAS) grid = 152 * CTAS;
  }
  if (grid < 1) grid = a.n_seq < 8 * 152 ? (a.n_seq + WARPS - 1) / WARPS : 152;    // states of empty sequences only
  kern<<<(unsigned)grid, NT, smem, st>>>(a);
  return launched();
}

template <bool BACK>
int by_type(const Call& f, GsArgs& a, cudaStream_t st) {
  if (!alone(a.n_rows, a.n_seq, BACK ? a.d_state_in && a.d_state_in == a.d_state_out : a.state_out && a.state_out == a.state_in))
    return f.dtype == TRACKFIT_FP32        ? launch<float, BACK, false>(f, a, st)
           : f.dtype == TRACKFIT_BF16_PROJ ? launch<__nv_bfloat16, BACK, false>(f, a, st)
                                           : launch<__half, BACK, false>(f, a, st);
  return f.dtype == TRACKFIT_FP32        ? launch<float, BACK, true>(f, a, st)
         : f.dtype == TRACKFIT_BF16_PROJ ? launch<__nv_bfloat16, BACK, true>(f, a, st)
                                         : launch<__half, BACK, true>(f, a, st);
}

}  // namespace

extern "C" size_t trackfit_gated_scan_saved(int64_t n_rows, int32_t channels) {
  if (n_rows < 0 || n_rows > (int64_t)1 << 40 || !channels_ok(channels)) return 0;
  return (size_t)((n_rows + TILE - 1) / TILE) * channels * 4;
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
  return by_type<false>(f, a, reinterpret_cast<cudaStream_t>(stream));
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
  return by_type<true>(f, a, reinterpret_cast<cudaStream_t>(stream));
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
