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

// z and w of a gate, each accurate however near to 0: 2^(-|p| log2 e) and 1 over one more than it.
__device__ __forceinline__ void gate(float p, float& z, float& w) {
  const float e = ex2(-LOG2E * fabsf(p)), r = __fdividef(1.0f, 1.0f + e), s = e * r;
  z = p < 0.0f ? s : r, w = p < 0.0f ? r : s;
}

template <class T>
struct Lane;                               // a lane's channels of a row: 4 bytes
template <>
struct Lane<float> {
  static constexpr int V = 1;
  static __device__ __forceinline__ void get(const void* p, float (&x)[1]) { x[0] = *(const float*)p; }
  static __device__ __forceinline__ void put(void* p, const float (&x)[1]) { *(float*)p = x[0]; }
};
template <class T>
struct Lane16 {
  static constexpr int V = 2;
  static __device__ __forceinline__ void put(void* p, const float (&x)[2]) { *(uint32_t*)p = pack2(x[0], x[1], T()); }
};
template <>
struct Lane<__nv_bfloat16> : Lane16<__nv_bfloat16> {
  static __device__ __forceinline__ void get(const void* p, float (&x)[2]) {
    const uint32_t u = *(const uint32_t*)p;
    x[0] = __uint_as_float(u << 16), x[1] = __uint_as_float(u & 0xffff0000u);
  }
};
template <>
struct Lane<__half> : Lane16<__half> {
  static __device__ __forceinline__ void get(const void* p, float (&x)[2]) {
    const float2 f = __half22float2(*(const __half2*)p);
    x[0] = f.x, x[1] = f.y;
  }
};

// fp32 channels of a state array, V at a time (even channels: 8 bytes aligned)
template <int V>
__device__ __forceinline__ void get_state(const float* s, float (&x)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = s[v];
}
template <int V>
__device__ __forceinline__ void put_state(float* s, const float (&x)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = x[v];
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

template <int V, int WIN>
struct Shared {
  float2 agg[WARPS][32 * V];               // (A, B) of the warps' rows
  float2 win[WIN][32 * V];                 // of the parts before, nearest first
  uint32_t has[WARPS];                     // a warp's rows hold a sequence's beginning: A does not count
  uint32_t status[WIN];
  Brought brought[2];
  uint64_t full[2], marked[2], empty[2];
  long long lo, hi;                        // rows of sequences
  int from;
  int abort, never;
};

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

// What a run of rows makes of what comes before it.
__device__ __forceinline__ float through(bool has, float2 f, float before) { return has ? f.y : fmaf(f.x, before, f.y); }

// The warps' (A, B), in their order (BACK: the last first), as one; `before` only where no
// sequence begins.
template <bool BACK, class S>
__device__ __forceinline__ float2 joined(const S* s, int c, bool& has) {
  float2 f = make_float2(1.0f, 0.0f);
  has = false;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    const int u = BACK ? WARPS - 1 - i : i;
    const float2 g = s->agg[u][c];
    if (s->has[u]) f = make_float2(0.0f, g.y), has = true;
    else f.x *= g.x, f.y = fmaf(g.x, f.y, g.y);
  }
  return f;
}

__device__ __forceinline__ unsigned long long word(uint32_t what, float x) {
  return (unsigned long long)what << 32 | __float_as_uint(x);
}
__device__ __forceinline__ void leave(unsigned long long* p, unsigned long long v) {
  asm volatile("st.relaxed.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ ulonglong2 look(const ulonglong2* p) {
  ulonglong2 v;
  asm volatile("ld.relaxed.gpu.global.v2.u64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "l"(p) : "memory");
  return v;
}

// What the parts before part k (BACK: behind it) leave for this CTA's channels: false if the wait for
// them expired.  All warps that compute; `in`: the lane has channels, c the first of them.
template <bool BACK, int V, int WIN>
__device__ __forceinline__ bool look_back(const GsArgs& a, Shared<V, WIN>* s, int64_t k, int c, bool in, float (&carry)[V]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t there = BACK ? a.parts - 1 - k : k;           // so many parts there are
  uint64_t t0 = 0;
  for (int round = 0;; ++round) {
#pragma unroll
    for (int i = 0; i < WIN / WARPS; ++i) {
      const int d = warp * (WIN / WARPS) + i;
      bool ready = true, whole = true, some = false;
      if (d < there && in) {
        const int64_t at = BACK ? k + 1 + d : k - 1 - d;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const ulonglong2 u = look(a.words + at * a.C + c + v);
          const uint32_t what = (uint32_t)(u.y >> 32);
          whole = whole && what == WHOLE, some = some || what == WHOLE;
          ready = ready && (what == WHOLE || (what == PARTIAL && u.x >> 32 == PARTIAL));
          s->win[d][lane * V + v] = make_float2(__uint_as_float((uint32_t)u.x), __uint_as_float((uint32_t)u.y));
        }
      }
      // all channels of a part alike: a part seen while h replaces B counts as not there
      const bool all_whole = __all_sync(FULL, whole), all_ready = __all_sync(FULL, ready), any = __any_sync(FULL, some);
      if (lane == 0) s->status[d] = d >= there || all_whole ? WHOLE : all_ready && !any ? PARTIAL : 0u;
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
#pragma unroll
  for (int v = 0; v < V; ++v) carry[v] = from < there ? s->win[from][lane * V + v].y : 0.0f;
  for (int d = from - 1; d >= 0; --d)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float2 f = s->win[d][lane * V + v];
      carry[v] = fmaf(f.x, carry[v], f.y);
    }
  return true;
}

// (A, B) of a part, or B alone where the part holds a sequence's beginning, for those behind it.
template <bool BACK, int V, int WIN>
__device__ __forceinline__ void leave_part(const GsArgs& a, const Shared<V, WIN>* s, int64_t k, int c, int lane) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    bool has;
    const float2 f = joined<BACK>(s, lane * V + v, has);
    unsigned long long* w = &a.words[k * a.C + c + v].x;
    if (!has) leave(w, word(PARTIAL, f.x));
    leave(w + 1, word(has ? WHOLE : PARTIAL, f.y));
  }
}
template <bool BACK, int V, int WIN>
__device__ __forceinline__ void leave_whole(const GsArgs& a, const Shared<V, WIN>* s, int64_t k, int c, int lane,
                                            const float (&carry)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    bool has;
    const float2 f = joined<BACK>(s, lane * V + v, has);
    if (!has) leave(&a.words[k * a.C + c + v].y, word(WHOLE, fmaf(f.x, carry[v], f.y)));
  }
}

// ---------------------------------------------------------------- forward

// (A, B) of the warp's rows, and their z and w.  KEEP: a sequence's first row has its h for a z (its
// state before is read once only: the CTA with the sequence's end may write the state after it to the
// same place as soon as this part has left its B).
template <class T, int V, bool KEEP>
__device__ __forceinline__ bool rows_forward(const GsArgs& a, const Part& t, const Marks& m, const uint8_t* raw, int c,
                                             bool in, float (&z)[RPW][V], float (&w)[RPW][V], float2 (&f)[V]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool has = false;
#pragma unroll
  for (int v = 0; v < V; ++v) f[v] = make_float2(1.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int d = row_in(a, t, warp * RPW + i);
    if (d < t.lo || d >= t.hi) continue;
    const bool begins = bound(m, a.reverse ? d + 1 : d);
    if (begins) {
      has = true;
      float s0[V] = {};
      if (a.state_in && in) get_state<V>(a.state_in + sequence(a, m, d, !a.reverse) * a.C + c, s0);
#pragma unroll
      for (int v = 0; v < V; ++v) f[v] = make_float2(0.0f, s0[v]);
    }
    float p[V], n[V];
    Lane<T>::get(raw + d * 128 + 4 * lane, p);
    Lane<T>::get(raw + PIECE + d * 128 + 4 * lane, n);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      gate(p[v], z[i][v], w[i][v]);
      f[v].x *= w[i][v];
      f[v].y = fmaf(w[i][v], f[v].y, z[i][v] * n[v]);
      if (KEEP && begins) z[i][v] = f[v].y;
    }
  }
  return has;
}

template <class T, int WIN, bool ALONE>
__global__ void __launch_bounds__(NT, CTAS) scan_kernel(const __grid_constant__ GsArgs a) {
  constexpr int V = Lane<T>::V, WIDE = 32 * V;
  extern __shared__ __align__(128) uint8_t smem[];
  Shared<V, WIN>* s = reinterpret_cast<Shared<V, WIN>*>(smem + 4 * PIECE);
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
  float carry[V] = {};
  bool ok = true;
  for (int n = 0;; ++n) {
    const int buf = n & 1;
    Brought& b = s->brought[buf];
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->marked[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok || b.kind == END) break;
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->full[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok) break;
    const int64_t k = b.k;
    const int c = b.c0 + lane * V;
    const bool in = c < a.C;
    const Part t = part_of(a, s, k);
    const Marks& m = b.marks;
    const uint8_t* raw = smem + buf * 2 * PIECE;
    float z[RPW][V], w[RPW][V];
    float2 f[V];
    const bool has = rows_forward<T, V, true>(a, t, m, raw, c, in, z, w, f);
#pragma unroll
    for (int v = 0; v < V; ++v) s->agg[warp][lane * V + v] = f[v];
    if (lane == 0) s->has[warp] = has;
    meet();
    if constexpr (ALONE) {
      if (b.kind == PASS) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          bool h;
          const float2 g = joined<false>(s, lane * V + v, h);
          carry[v] = through(h, g, carry[v]);
        }
        __syncwarp();
        if (lane == 0) sm100::mbar_arrive(smem_addr(&s->empty[buf]));
        meet();
        continue;
      }
    } else {
      // what is before this part counts if its first position is a row within a sequence
      const int d0 = row_in(a, t, 0);
      const bool inside = d0 >= t.lo && d0 < t.hi && !bound(m, a.reverse ? d0 + 1 : d0);
      if (warp == 0 && in) leave_part<false>(a, s, k, c, lane);
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = 0.0f;
      if (inside) {
        if (!look_back<false, V, WIN>(a, s, k, c, in, carry)) {
          ok = false;
          break;
        }
        if (warp == 0 && in) leave_whole<false>(a, s, k, c, lane, carry);
      }
    }
    if (a.saved && warp == 0 && in) put_state<V>(a.saved + k * a.C + c, carry);
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      h[v] = carry[v];
      for (int u = 0; u < warp; ++u) h[v] = through(s->has[u], s->agg[u][lane * V + v], h[v]);
    }
    T* out = (T*)a.out + c;
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
      const int d = row_in(a, t, warp * RPW + i);
      const int64_t row = t.row0 + d;
      if (d < t.lo || d >= t.hi) continue;
      const bool begins = bound(m, a.reverse ? d + 1 : d);
      float n[V];
      Lane<T>::get(raw + PIECE + d * 128 + 4 * lane, n);
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = begins ? z[i][v] : fmaf(w[i][v], h[v], z[i][v] * n[v]);
      if (in) {
        Lane<T>::put(out + row * a.os, h);
        if (a.state_out && bound(m, a.reverse ? d : d + 1)) put_state<V>(a.state_out + sequence(a, m, d, a.reverse) * a.C + c, h);
      }
    }
    __syncwarp();
    if (lane == 0) sm100::mbar_arrive(smem_addr(&s->empty[buf]));
    meet();
  }
  if (!ok && lane == 0 && atomicExch(&s->abort, 1) == 0) atomicAdd(a.expired, 1ull);
}

// ---------------------------------------------------------------- backward

template <class T, int WIN, bool ALONE>
__global__ void __launch_bounds__(NT, CTAS) backward_kernel(const __grid_constant__ GsArgs a) {
  constexpr int V = Lane<T>::V, WIDE = 32 * V;
  extern __shared__ __align__(128) uint8_t smem[];
  Shared<V, WIN>* s = reinterpret_cast<Shared<V, WIN>*>(smem + 6 * PIECE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // sequences of no rows: what is before them is what is after them
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
  float carry[V] = {};
  bool ok = true;
  for (int n = 0;; ++n) {
    const int buf = n & 1;
    Brought& b = s->brought[buf];
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->marked[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok || b.kind == END) break;
    ok = __all_sync(FULL, sm100::mbar_wait(smem_addr(&s->full[buf]), (n >> 1) & 1, abort, a.limit_ns));
    if (!ok) break;
    const int64_t k = b.k;
    const int c = b.c0 + lane * V;
    const bool in = c < a.C;
    const Part t = part_of(a, s, k);
    const Marks& m = b.marks;
    uint8_t* raw = smem + buf * 3 * PIECE;
    float z[RPW][V], w[RPW][V];
    {
      // the states again, from the one saved before the part
      float2 f[V];
      const bool has = rows_forward<T, V, false>(a, t, m, raw, c, in, z, w, f);
#pragma unroll
      for (int v = 0; v < V; ++v) s->agg[warp][lane * V + v] = f[v];
      if (lane == 0) s->has[warp] = has;
      meet();
      float h[V] = {};
      if (in) get_state<V>(a.saved + k * a.C + c, h);
#pragma unroll
      for (int v = 0; v < V; ++v)
        for (int u = 0; u < warp; ++u) h[v] = through(s->has[u], s->agg[u][lane * V + v], h[v]);
      // z w (n - h) takes the place of p and n, 4 bytes a channel
#pragma unroll
      for (int i = 0; i < RPW; ++i) {
        const int d = row_in(a, t, warp * RPW + i);
        if (d < t.lo || d >= t.hi) continue;
        if (bound(m, a.reverse ? d + 1 : d)) {
#pragma unroll
          for (int v = 0; v < V; ++v) h[v] = 0.0f;
          if (a.state_in && in) get_state<V>(a.state_in + sequence(a, m, d, !a.reverse) * a.C + c, h);
        }
        float n[V];
        uint8_t* at = raw + d * 128 + 4 * lane;
        Lane<T>::get(at + PIECE, n);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          *reinterpret_cast<float*>(at + v * PIECE) = z[i][v] * w[i][v] * (n[v] - h[v]);
          h[v] = fmaf(w[i][v], h[v], z[i][v] * n[v]);
        }
      }
      meet();
    }
    // what comes from behind: e before the warp's rows = A e after them + B.  A sequence's last row gets
    // its results here: what its state's gradient is may be written over once this part has left its B.
    bool has = false;
    float2 f[V];
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = make_float2(1.0f, 0.0f);
#pragma unroll
    for (int i = RPW - 1; i >= 0; --i) {
      const int d = row_in(a, t, warp * RPW + i);
      if (d < t.lo || d >= t.hi) continue;
      const bool ends = bound(m, a.reverse ? d : d + 1);
      if (ends) {
        has = true;
        float e[V] = {};
        if (a.d_state_out && in) get_state<V>(a.d_state_out + sequence(a, m, d, a.reverse) * a.C + c, e);
#pragma unroll
        for (int v = 0; v < V; ++v) f[v] = make_float2(0.0f, e[v]);
      }
      float g[V];
      uint8_t* at = raw + d * 128 + 4 * lane;
      Lane<T>::get(at + 2 * PIECE, g);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float D = g[v] + f[v].y;
        f[v].x *= w[i][v], f[v].y = w[i][v] * D;
        if (ends) z[i][v] *= D, w[i][v] = f[v].y, *reinterpret_cast<float*>(at + v * PIECE) *= D;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) s->agg[warp][lane * V + v] = f[v];
    if (lane == 0) s->has[warp] = has;
    meet();
    if constexpr (ALONE) {
      if (b.kind == PASS) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          bool h;
          const float2 g = joined<true>(s, lane * V + v, h);
          carry[v] = through(h, g, carry[v]);
        }
        __syncwarp();
        if (lane == 0) sm100::mbar_arrive(smem_addr(&s->empty[buf]));
        meet();
        continue;
      }
    } else {
      const int d1 = row_in(a, t, t.count - 1);
      const bool inside = d1 >= t.lo && d1 < t.hi && !bound(m, a.reverse ? d1 : d1 + 1);
      if (warp == 0 && in) leave_part<true>(a, s, k, c, lane);
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = 0.0f;
      if (inside) {
        if (!look_back<true, V, WIN>(a, s, k, c, in, carry)) {
          ok = false;
          break;
        }
        if (warp == 0 && in) leave_whole<true>(a, s, k, c, lane, carry);
      }
    }
    float e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      e[v] = carry[v];
      for (int u = WARPS - 1; u > warp; --u) e[v] = through(s->has[u], s->agg[u][lane * V + v], e[v]);
    }
    T *dp = (T*)a.dp + c, *dn = (T*)a.dn + c;
#pragma unroll
    for (int i = RPW - 1; i >= 0; --i) {
      const int d = row_in(a, t, warp * RPW + i);
      const int64_t row = t.row0 + d;
      if (d < t.lo || d >= t.hi) continue;
      const bool ends = bound(m, a.reverse ? d : d + 1);
      float g[V], x[V], y[V];
      const uint8_t* at = raw + d * 128 + 4 * lane;
      Lane<T>::get(at + 2 * PIECE, g);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float D = ends ? 1.0f : g[v] + e[v];
        x[v] = *reinterpret_cast<const float*>(at + v * PIECE) * D;
        y[v] = z[i][v] * D;
        e[v] = w[i][v] * D;
      }
      if (in) {
        Lane<T>::put(dp + row * a.dps, x);
        Lane<T>::put(dn + row * a.dns, y);
        if (a.d_state_in && bound(m, a.reverse ? d + 1 : d)) put_state<V>(a.d_state_in + sequence(a, m, d, !a.reverse) * a.C + c, e);
      }
    }
    __syncwarp();
    if (lane == 0) sm100::mbar_arrive(smem_addr(&s->empty[buf]));
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
  constexpr int V = Lane<T>::V, WIN = BACK && V == 2 ? 16 : 32;
  constexpr auto kern = [] {
    if constexpr (BACK) return &backward_kernel<T, WIN, ALONE>;
    else return &scan_kernel<T, WIN, ALONE>;
  }();
  a.parts = (a.n_rows + TILE - 1) / TILE, a.blocks = (a.C + 32 * V - 1) / (32 * V);
  a.limit_ns = operator_limit_ns(), a.expired = operator_expired();
  if (!a.expired) return TRACKFIT_ERR_CUDA;
  if (a.n_rows > 0 && (!make_map(&a.tp, f.dtype, f.p, a.n_rows, a.C, f.ps) || !make_map(&a.tn, f.dtype, f.n, a.n_rows, a.C, f.ns) ||
                       (BACK && !make_map(&a.tg, f.dtype, f.g, a.n_rows, a.C, f.gs))))
    return TRACKFIT_ERR_CUDA;
  const size_t smem = (BACK ? 6 : 4) * PIECE + sizeof(Shared<V, WIN>);
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
