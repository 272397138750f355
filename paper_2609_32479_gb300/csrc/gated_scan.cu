// The gated recurrence over packed sequences and its gradients.
//
//   z = sigma(p), w = 1 - z,  h_t = w_t h_{t-1} + z_t n_t
//   back, from the direction's last row to its first:
//   D_t = g_t + e_t,  e_{t-1} = w_t D_t,  dn = z D,  dp = z w (n - h_{t-1}) D
//
// Bound by memory: three values a row and channel are moved forward, five backward.  A warp takes
// windows of 32 rows x 128 bytes of channels, brought by TMA; a lane has one channel (16 bits: two
// neighbouring ones, in instructions that take two).  The gates of eight rows are formed side by side, so
// that their latencies overlap, then the recurrence runs through them.  No warp waits for another.
//
// Short sequences (64 rows on average at most): a warp takes the sequences that begin in its rows, as
// far as they reach, so that it begins with a state that it knows.
//
// Long ones: what stands before a run of rows acts on it through one number a channel,
// h_last = A h_before + B with A the product of the w.  A first kernel forms (A, B) of every warp's windows
// and of segments (a CTA's windows), a second the states before the segments, one after the other; then
// the first state of every warp's windows is three loads and a multiply-add away.  So p and n are read
// twice, the second time in part from L2.  (One pass, in which parts of 128 rows look back for what the
// part before them left, moves less but was slower, 205 us for 5 sequences of up to 30,000 rows of 512
// channels in bf16: too few rows are under way on an SM for the waits.)
// A sequence's first row ends what comes from before by choice, not by a factor 0: it may not be finite.
//
// Backward, D runs the other way by the same steps: (A, B) of e from the segments' ends.  A window's
// states are formed again from the one before it that the forward pass saved.
//
// What bounds it: tracks of 8 to 20 rows, 192 channels in bf16, forward 181 us of the 156 that the bytes take,
// backward 361 of 261, with 12 warps on an SM (16 KB of rows each) and 57 % of the issue slots used; long
// sequences issued instructions (55 %) in the sums, some 40 a row of 64 channels, and the rows, 52.
#include "seq_ops.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>

#include <utility>

namespace {
using namespace seqops;

constexpr int WINDOW = 32;                 // positions, and from one saved state to the next
constexpr int GROUP = 8;                   // rows whose gates are formed side by side
constexpr uint32_t GROUP_BITS = (1u << GROUP) - 1u;
constexpr int WARPS = 8;                   // of a CTA, forward; of a segment
constexpr int BACK_WARPS = 4;
constexpr int MAX_CHANNELS = 1 << 16;
constexpr int SHORT = 64;                  // rows of a sequence on average
constexpr uint64_t LOAD_NS = 2000000000ull;

// Rows in the order of a recurrence: position = row + t, or t - row.
struct Order {
  int back;                                // t - row
  int64_t t;
};

struct GsArgs {
  const void *p, *n, *g;
  CUtensorMap tp, tn, tg;                  // boxes of 128 bytes x 32 rows
  void *out, *dp, *dn;
  int64_t ps, ns, gs, os, dps, dns;        // row strides in elements
  const int64_t* offs;
  int64_t n_rows, n_seq;
  int C, blocks;                           // blocks: warps side by side in a window
  Order order, flipped;                    // of the recurrence, and of what goes back through it
  const float *state_in, *d_state_out;
  float *state_out, *d_state_in;
  float* saved;                            // [windows][C]: the state before a window
  int64_t windows, segments;
  int each, chunk;                         // windows of a segment's warp; positions whose sequences a warp takes
  // long sequences: by warp, what comes before its windows in its segment; by segment, all of it and the
  // state before it
  int64_t units;                           // warps' windows
  float *warp_a, *warp_b, *seg_a, *seg_b, *seg_s;
  uint32_t *warp_has, *seg_has;
  unsigned long long* expired;
};

// z and w of a gate: the smaller, e / (1 + e) with e = 2^(-|p| log2 e), accurate however near to 0, and one
// less that, so that they add up to 1 (in the 1,000 rows that a slow channel remembers an error of their
// sum, always of one sign, would add up too: the states' error was ten times as large).
__device__ __forceinline__ void gate(float p, float& z, float& w) {
  const float e = ex2(-LOG2E * fabsf(p)), s = e * rcp(1.0f + e), b = 1.0f - s;
  z = p < 0.0f ? s : b, w = p < 0.0f ? b : s;
}

// A lane's channels of a row: 4 bytes, one or two fp32 values (two in the instructions that take two).
template <class T>
struct Lane;
template <>
struct Lane<float> {
  static constexpr int V = 1;
  using P = float;
  static __device__ __forceinline__ P make(float a, float) { return a; }
  static __device__ __forceinline__ P get(uint32_t u) { return __uint_as_float(u); }
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
    const P small = mul2(e, both(rcp(y.x), rcp(y.y)));
    const float2 s = parts(small), b = parts(fma2(small, both(-1.0f, -1.0f), both(1.0f, 1.0f)));
    z = both(f.x < 0.0f ? s.x : b.x, f.y < 0.0f ? s.y : b.y), w = both(f.x < 0.0f ? b.x : s.x, f.y < 0.0f ? b.y : s.y);
  }
  static __device__ __forceinline__ float part(P a, int v) { return v ? parts(a).y : parts(a).x; }
};
template <>
struct Lane<__nv_bfloat16> : Lane16<__nv_bfloat16> {
  static __device__ __forceinline__ P get(uint32_t u) {
    return both(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
};
template <>
struct Lane<__half> : Lane16<__half> {
  static __device__ __forceinline__ P get(uint32_t u) {
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

__device__ __forceinline__ int64_t row_of(const Order& o, int64_t pos) { return o.back ? o.t - pos : pos - o.t; }
// The i-th border of sequences in the order of positions, 0 <= i <= n_seq, and that order's i-th sequence.
__device__ __forceinline__ int64_t border(const GsArgs& a, const Order& o, int64_t i) {
  return o.back ? o.t + 1 - a.offs[a.n_seq - i] : a.offs[i] + o.t;
}
__device__ __forceinline__ int64_t sequence_of(const GsArgs& a, const Order& o, int64_t i) {
  i = clamp64(i, 0, a.n_seq - 1);
  return o.back ? a.n_seq - 1 - i : i;
}
// The first border at or behind a position (its number, or n_seq + 1): a whole warp, 33 parts a round.
__device__ __forceinline__ int64_t border_at(const GsArgs& a, const Order& o, int64_t pos, int lane) {
  int64_t lo = 0, hi = a.n_seq + 1;
  while (hi > lo) {
    const int64_t step = (hi - lo + 32) / 33;
    const int64_t at = lo + (lane + 1) * step - 1;
    const int k = __popc(__ballot_sync(FULL, at < hi && border(a, o, at) < pos));
    const int64_t nlo = lo + k * step, nhi = k == 32 ? hi : nlo + step - 1;
    lo = nlo < hi ? nlo : hi;
    hi = nhi < hi ? nhi : hi;
  }
  return lo;
}

// The same, given the number j of one at or behind it: the borders below it, 32 at a time.
__device__ __forceinline__ int64_t border_down(const GsArgs& a, const Order& o, int64_t pos, int64_t j, int lane) {
  for (;;) {
    const int n = __popc(__ballot_sync(FULL, j - 1 - lane >= 0 && border(a, o, j - 1 - lane) >= pos));
    j -= n;
    if (n < 32) return j;
  }
}

// A window: up to 32 positions, all rows of sequences, and the sequences among them, bit i for the i-th.
struct Window {
  int64_t pos;
  int count;
  int64_t first;                           // the first border at or behind it
  uint32_t begins, ends;                   // first rows, last rows
};
// From `pos` on, in [lo, hi), given the first border's number; `after` gets that of the next window's.  A whole warp.
__device__ __forceinline__ Window window_at(const GsArgs& a, const Order& o, int64_t pos, int64_t lo, int64_t hi, int64_t first,
                                            int lane, int64_t& after) {
  Window m;
  m.pos = pos < lo ? lo : pos;
  m.count = (int)clamp64((pos + WINDOW < hi ? pos + WINDOW : hi) - m.pos, 0, WINDOW);
  m.first = after = first;
  uint32_t bits = 0, last = 0;
  for (;;) {
    const int64_t b = after + lane <= a.n_seq ? border(a, o, after + lane) - m.pos : INT64_MAX;
    const int d = b > WINDOW ? WINDOW + 1 : b < 0 ? -1 : (int)b;
    bits |= __reduce_or_sync(FULL, d >= 0 && d < WINDOW ? 1u << d : 0u);
    last |= __any_sync(FULL, d == WINDOW) ? 1u : 0u;
    const int n = __popc(__ballot_sync(FULL, b < pos + WINDOW - m.pos));
    after += n;
    if (n < 32) break;
  }
  const uint32_t valid = m.count >= 32 ? FULL : (1u << m.count) - 1u;
  m.begins = bits & valid, m.ends = (bits >> 1 | last << 31) & valid;
  return m;
}
// The positions that are rows of sequences (and, whatever the offsets say, of the array).
__device__ __forceinline__ void extent(const GsArgs& a, const Order& o, int64_t& lo, int64_t& hi) {
  const int64_t p0 = o.back ? o.t + 1 - a.n_rows : o.t;
  lo = clamp64(border(a, o, 0), p0, p0 + a.n_rows), hi = clamp64(border(a, o, a.n_seq), lo, p0 + a.n_rows);
}
// The sequence that begins with position i of the window (or, `ends`, ends with it): the last border there,
// or the one before the first behind it.  A whole warp.
__device__ __noinline__ int64_t sequence(const GsArgs& a, const Order& o, const Window& m, int i, bool ends) {
  const int64_t pos = m.pos + i + (ends ? 1 : 0);
  int64_t j = m.first;
  for (int64_t at = m.first;; at += 32) {
    const int64_t b = at + (threadIdx.x & 31) <= a.n_seq ? border(a, o, at + (threadIdx.x & 31)) : INT64_MAX;
    const int n = __popc(__ballot_sync(FULL, ends ? b < pos : b <= pos));
    j += n;
    if (n < 32) break;
  }
  return sequence_of(a, o, j - 1);
}
// What is before position i, a sequence's first (`ends`: behind its last): the state given, or zeros.  A whole warp.
template <class L>
__device__ __forceinline__ typename L::P given(const GsArgs& a, const Order& o, const Window& m, int i, bool ends,
                                               const float* states, int c, bool in) {
  typename L::P h = L::make(0.0f, 0.0f);
  if (states) {
    const int64_t b = sequence(a, o, m, i, ends);
    if (in) h = get_state<L>(states + b * a.C + c);
  }
  return h;
}

// A warp's buffer for a window: 32 rows of 128 bytes of each array, brought by one lane.
constexpr int BLOCK = WINDOW * 128;
template <int ARRAYS>
__device__ __forceinline__ void bring(uint32_t to, uint32_t full, const Order& o, int64_t pos, int c, const CUtensorMap* x,
                                      const CUtensorMap* y, const CUtensorMap* z) {
  sm100::fence_proxy_async_smem();         // (what was written into the buffer, before the copy into it)
  __syncwarp();
  if ((threadIdx.x & 31) == 0) {
    const int r0 = (int)row_of(o, o.back ? pos + WINDOW - 1 : pos);   // the lowest row (it may be below the array)
    sm100::mbar_arrive_expect_tx(full, ARRAYS * BLOCK);
    sm100::tma_load_2d(to, x, full, c, r0);
    sm100::tma_load_2d(to + BLOCK, y, full, c, r0);
    if constexpr (ARRAYS == 3) sm100::tma_load_2d(to + 2 * BLOCK, z, full, c, r0);
  }
}
__device__ __forceinline__ bool brought(uint32_t full, uint32_t parity) {
  int never = 0;
  return __all_sync(FULL, sm100::mbar_wait(full, parity, &never, LOAD_NS));
}
__device__ __forceinline__ uint32_t lds(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ void sts(uint32_t at, float x) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory"); }
// A lane's word of position i in a buffer is at `at` + i `step`.
struct Walk {
  uint32_t at;
  int step;
};
__device__ __forceinline__ Walk walk_of(const Order& o, uint32_t buffer) {
  return {buffer + 4 * (threadIdx.x & 31) + (o.back ? (WINDOW - 1) * 128 : 0), o.back ? -128 : 128};
}

// The three kernels of long sequences begin while the one before them ends, with what does not need its
// results, and wait for these here (a kernel is done only after the one before it is).
__device__ __forceinline__ void after_kernels_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Sequences of no rows: what is before them is what is after them.
__device__ __forceinline__ void empty_sequences(const GsArgs& a, float* to, const float* from) {
  if (!to) return;
  const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / 32, step = (int64_t)gridDim.x * blockDim.x / 32;
  for (int64_t b = warp; b < a.n_seq; b += step)
    if (a.offs[b] >= a.offs[b + 1])
      for (int c = threadIdx.x & 31; c < a.C; c += 32) to[b * a.C + c] = from ? from[b * a.C + c] : 0.0f;
}

// ---------------------------------------------------------------- long sequences: before the rows

// (A, B) of the warps' windows: of h, or (BACK) of e in the flipped order, where B = w (g + B).
template <class T, bool BACK>
__global__ void __launch_bounds__(WARPS * 32, 3) sums_kernel(const __grid_constant__ GsArgs a) {
  using L = Lane<T>;
  using P = typename L::P;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ P sum_a[WARPS][32], sum_b[WARPS][32];
  __shared__ uint32_t sum_has[WARPS];
  __shared__ uint64_t bars[WARPS];
  const Order& o = BACK ? a.flipped : a.order;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t seg = blockIdx.x / a.blocks;
  const int block = (int)(blockIdx.x % a.blocks), c0 = block * 32 * L::V, c = c0 + lane * L::V;
  const bool in = c < a.C;
  const uint32_t full = smem_addr(&bars[warp]), buffer = smem_addr(smem) + warp * 2 * BLOCK;
  if (lane == 0) {
    sm100::mbar_init(full, 1);
    sm100::fence_mbar_init();
  }
  __syncwarp();
  const Walk walk = walk_of(o, buffer);
  const float* states = BACK ? a.d_state_out : a.state_in;
  const int64_t unit = seg * WARPS + warp, w0 = unit * a.each;
  P fa = L::make(1.0f, 1.0f), fb = L::make(0.0f, 0.0f);
  bool has = false, ok = true;
  uint32_t parity = 0;
  int64_t lo, hi, next = 0;
  extent(a, o, lo, hi);
  if (w0 < a.windows) next = border_at(a, o, w0 * WINDOW > lo ? w0 * WINDOW : lo, lane);
  for (int e = 0; e < a.each && w0 + e < a.windows; ++e) {
    const int64_t pos = (w0 + e) * WINDOW;
    if (pos >= hi || pos + WINDOW <= lo) continue;
    const Window m = window_at(a, o, pos, lo, hi, next, lane, next);
    bring<2>(buffer, full, o, m.pos, c0, &a.tp, BACK ? &a.tg : &a.tn, nullptr);
    ok = brought(full, parity) && ok;
    parity ^= 1;
    for (int i0 = 0; i0 < m.count; i0 += GROUP) {
      P w[GROUP], x[GROUP];
#pragma unroll
      for (int i = 0; i < GROUP; ++i) {
        const uint32_t at = walk.at + (i0 + i) * walk.step;
        P z;
        L::gates(L::get(lds(at)), z, w[i]);
        const P y = L::get(lds(at + BLOCK));
        x[i] = BACK ? y : L::mul(z, y);
      }
      const int left = m.count - i0;
      has = has || (m.begins >> i0 & GROUP_BITS) != 0;
      auto row = [&](int i, P before) {
        fa = L::mul(fa, w[i]);
        if constexpr (BACK) fb = L::mul(w[i], L::add(x[i], before));
        else fb = L::fma(w[i], before, x[i]);
      };
      if (left >= GROUP && (m.begins >> i0 & GROUP_BITS) == 0) {
#pragma unroll
        for (int i = 0; i < GROUP; ++i) row(i, fb);
      } else {
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
          if (i >= left) break;
          row(i, (m.begins >> (i0 + i)) & 1u ? given<L>(a, o, m, i0 + i, false, states, c, in) : fb);
        }
      }
    }
    __syncwarp();
  }
  sum_a[warp][lane] = fa, sum_b[warp][lane] = fb;
  if (lane == 0) sum_has[warp] = has;
  __syncthreads();
  if (!ok && lane == 0) atomicAdd(a.expired, 1ull);
  // from the segment's first row on
  P ga = L::make(1.0f, 1.0f), gb = L::make(0.0f, 0.0f);
  bool gh = false;
  auto on = [&](int u) {
    const bool h = sum_has[u];
    gb = L::pick(h, sum_b[u][lane], L::fma(sum_a[u][lane], gb, sum_b[u][lane]));
    ga = L::mul(sum_a[u][lane], ga);
    gh = gh || h;
  };
  for (int u = 0; u < warp; ++u) on(u);
  if (w0 < a.windows) {
    if (in) put_state<L>(a.warp_a + unit * a.C + c, ga), put_state<L>(a.warp_b + unit * a.C + c, gb);
    if (lane == 0 && block == 0) a.warp_has[unit] = gh;
  }
  if (warp == WARPS - 1) {
    on(warp);
    if (in) put_state<L>(a.seg_a + seg * a.C + c, ga), put_state<L>(a.seg_b + seg * a.C + c, gb);
    if (lane == 0 && block == 0) a.seg_has[seg] = gh;
  }
}

// The states before the segments, a thread a channel.
__global__ void __launch_bounds__(64) chain_kernel(const __grid_constant__ GsArgs a) {
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c >= a.C) return;
  constexpr int AHEAD = 16;
  float s = 0.0f;
  after_kernels_before();
  for (int64_t g = 0; g < a.segments; g += AHEAD) {
    float x[AHEAD], y[AHEAD];
    bool h[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int64_t at = g + i < a.segments ? g + i : a.segments - 1;
      x[i] = a.seg_a[at * a.C + c], y[i] = a.seg_b[at * a.C + c], h[i] = a.seg_has[at] != 0;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (g + i >= a.segments) break;
      a.seg_s[(g + i) * a.C + c] = s;
      s = h[i] ? y[i] : fmaf(x[i], s, y[i]);
    }
  }
}

// What comes into a warp's windows from before them.
template <class L>
__device__ __forceinline__ typename L::P into(const GsArgs& a, int64_t unit, int c, bool in) {
  typename L::P h = L::make(0.0f, 0.0f);
  if (in) {
    h = get_state<L>(a.warp_b + unit * a.C + c);
    if (!a.warp_has[unit]) h = L::fma(get_state<L>(a.warp_a + unit * a.C + c), get_state<L>(a.seg_s + unit / WARPS * a.C + c), h);
  }
  return h;
}

// ---------------------------------------------------------------- forward

// A window's rows, brought, from the state h before them to the one after.
template <class T>
__device__ __forceinline__ void window_forward(const GsArgs& a, const Window& m, const Walk& walk, int c, bool in,
                                               typename Lane<T>::P& h) {
  using L = Lane<T>;
  using P = typename L::P;
  const Order& o = a.order;
  T* out = (T*)a.out + row_of(o, m.pos) * a.os + c;
  const int64_t step = o.back ? -a.os : a.os;
  const uint32_t slow = a.state_in ? m.begins : 0u, ends = a.state_out ? m.ends : 0u;
#pragma unroll 1
  for (int i0 = 0; i0 < m.count; i0 += GROUP) {
    P w[GROUP], x[GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const uint32_t at = walk.at + (i0 + i) * walk.step;
      P z;
      L::gates(L::get(lds(at)), z, w[i]);
      x[i] = L::mul(z, L::get(lds(at + BLOCK)));
    }
    const bool whole = m.count - i0 >= GROUP;   // (else row by row: the state goes on behind the last one)
    const uint32_t begins = m.begins >> i0;
    if (whole && ((m.begins | ends) >> i0 & GROUP_BITS) == 0) {
#pragma unroll
      for (int i = 0; i < GROUP; ++i, out += step) {
        h = L::fma(w[i], h, x[i]);
        if (in) L::put(out, h);
      }
    } else if (whole && ((slow | ends) >> i0 & GROUP_BITS) == 0) {
#pragma unroll
      for (int i = 0; i < GROUP; ++i, out += step) {
        h = L::fma(w[i], L::pick((begins >> i) & 1u, L::make(0.0f, 0.0f), h), x[i]);
        if (in) L::put(out, h);
      }
    } else {
#pragma unroll
      for (int i = 0; i < GROUP; ++i, out += step) {
        if (i0 + i >= m.count) break;
        if ((begins >> i) & 1u) h = given<L>(a, o, m, i0 + i, false, a.state_in, c, in);
        h = L::fma(w[i], h, x[i]);
        if (in) L::put(out, h);
        if ((ends >> (i0 + i)) & 1u) {
          const int64_t b = sequence(a, o, m, i0 + i, true);
          if (in) put_state<L>(a.state_out + b * a.C + c, h);
        }
      }
    }
  }
}

template <class T, bool LONG>
__global__ void __launch_bounds__(WARPS * 32, 3) rows_kernel(const __grid_constant__ GsArgs a) {
  using L = Lane<T>;
  using P = typename L::P;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t bars[WARPS];
  empty_sequences(a, a.state_out, a.state_in);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * WARPS + warp;
  const int64_t k = unit / a.blocks;
  const int c0 = (int)(unit % a.blocks) * 32 * L::V, c = c0 + lane * L::V;
  const bool in = c < a.C;
  const uint32_t full = smem_addr(&bars[warp]), buffer = smem_addr(smem) + warp * 2 * BLOCK;
  if (lane == 0) {
    sm100::mbar_init(full, 1);
    sm100::fence_mbar_init();
  }
  __syncwarp();
  const Order& o = a.order;
  const Walk walk = walk_of(o, buffer);
  P h = L::make(0.0f, 0.0f);
  bool ok = true;
  int64_t lo, hi, next;
  if (a.n_rows == 0) return;
  extent(a, o, lo, hi);
  if constexpr (LONG) {
    // the last windows first: their rows are in L2, from the sums
    const int64_t u = a.units - 1 - unit / a.blocks;
    const int64_t first = u * a.each * WINDOW, upto = first + a.each * WINDOW < hi ? first + a.each * WINDOW : hi;
    const int64_t from = first < lo ? lo : first;
    if (u < 0 || from >= upto) {
      after_kernels_before();
      return;
    }
    uint32_t parity = 0;
    next = border_at(a, o, from, lane);
    for (int64_t pos = from / WINDOW * WINDOW; pos < upto && ok; pos += WINDOW, parity ^= 1) {
      bring<2>(buffer, full, o, pos < lo ? lo : pos, c0, &a.tp, &a.tn, nullptr);
      const Window m = window_at(a, o, pos, lo, hi, next, lane, next);
      if (parity == 0 && pos <= from) {
        after_kernels_before();
        if (!(m.begins & 1u)) h = into<L>(a, u, c, in);
      }
      if (a.saved && in) put_state<L>(a.saved + pos / WINDOW * a.C + c, h);
      ok = brought(full, parity);
      window_forward<T>(a, m, walk, c, in, h);
    }
  } else {
    // the sequences that begin in [from, from + chunk)
    const int64_t from = k * a.chunk, upto = from + a.chunk;
    if (from >= hi) return;
    next = border_at(a, o, from, lane);
    if (next > a.n_seq) return;
    int64_t pos = border(a, o, next);
    if (pos >= upto || pos >= hi || pos < lo) return;
    uint32_t parity = 0;
    bool begun = false;
    for (bool more = true; more && ok; pos += WINDOW, parity ^= 1) {
      bring<2>(buffer, full, o, pos, c0, &a.tp, &a.tn, nullptr);
      Window m = window_at(a, o, pos, lo, hi, next, lane, next);
      // as far as the first row of the sequences behind these
      const uint32_t behind = upto <= pos ? FULL : upto - pos < WINDOW ? FULL << (upto - pos) : 0u;
      const uint32_t stop = m.begins & behind;
      more = stop == 0 && pos + WINDOW < hi && !(pos + WINDOW >= upto && m.ends >> (WINDOW - 1));
      if (stop) {
        m.count = __ffs(stop) - 1;
        m.begins &= (stop & -stop) - 1u, m.ends &= (stop & -stop) - 1u;
      }
      if (a.saved && in && begun) put_state<L>(a.saved + pos / WINDOW * a.C + c, h);
      begun = true;
      ok = brought(full, parity);
      window_forward<T>(a, m, walk, c, in, h);
    }
  }
  if (!ok && lane == 0) atomicAdd(a.expired, 1ull);
}

// ---------------------------------------------------------------- backward

// A window's rows, brought: states from h upwards, D downwards.  e: what comes into the last row from behind
// it, and then out of the first.
template <class T>
__device__ __forceinline__ void window_backward(const GsArgs& a, const Window& m, const Walk& walk, int c, bool in,
                                                typename Lane<T>::P h, typename Lane<T>::P& e) {
  using L = Lane<T>;
  using P = typename L::P;
  const Order& o = a.order;
  const uint32_t slow = a.state_in ? m.begins : 0u;
#pragma unroll 1
  for (int i0 = 0; i0 < m.count; i0 += GROUP) {
    // z w (n - h) takes the place of n (16 bits: of n and a block more)
    P z[GROUP], w[GROUP], n[GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const uint32_t at = walk.at + (i0 + i) * walk.step;
      L::gates(L::get(lds(at)), z[i], w[i]);
      n[i] = L::get(lds(at + BLOCK));
    }
    const uint32_t firsts = m.begins >> i0;
    auto row = [&](int i) {
      const uint32_t at = walk.at + (i0 + i) * walk.step;
      const P q = L::mul(L::mul(z[i], w[i]), L::sub(n[i], h));
      h = L::fma(w[i], h, L::mul(z[i], n[i]));
      sts(at + BLOCK, L::part(q, 0));
      if constexpr (L::V == 2) sts(at + 3 * BLOCK, L::part(q, 1));
    };
    if ((slow >> i0 & GROUP_BITS) == 0) {
#pragma unroll
      for (int i = 0; i < GROUP; ++i) {
        h = L::pick((firsts >> i) & 1u, L::make(0.0f, 0.0f), h);
        row(i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < GROUP; ++i) {
        if ((firsts >> i) & 1u) h = given<L>(a, o, m, i0 + i, false, a.state_in, c, in);
        row(i);
      }
    }
  }
  const int top = (m.count - 1) / GROUP * GROUP;
  const int64_t row = row_of(o, m.pos + top + GROUP - 1);
  const int64_t step1 = o.back ? a.dps : -a.dps, step2 = o.back ? a.dns : -a.dns;
  T *dp = (T*)a.dp + row * a.dps + c, *dn = (T*)a.dn + row * a.dns + c;
  const uint32_t last = a.d_state_out ? m.ends : 0u, begins = a.d_state_in ? m.begins : 0u;
#pragma unroll 1
  for (int i0 = top; i0 >= 0; i0 -= GROUP) {
    P z[GROUP], w[GROUP], g[GROUP], q[GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const uint32_t at = walk.at + (i0 + i) * walk.step;
      L::gates(L::get(lds(at)), z[i], w[i]);
      g[i] = L::get(lds(at + 2 * BLOCK));
      q[i] = L::make(__uint_as_float(lds(at + BLOCK)), L::V == 2 ? __uint_as_float(lds(at + 3 * BLOCK)) : 0.0f);
    }
    const int left = m.count - i0;
    const uint32_t lasts = m.ends >> i0;
    if (left >= GROUP && ((last | begins) >> i0 & GROUP_BITS) == 0) {
#pragma unroll
      for (int i = GROUP - 1; i >= 0; --i, dp += step1, dn += step2) {
        const P D = L::add(g[i], L::pick((lasts >> i) & 1u, L::make(0.0f, 0.0f), e));
        e = L::mul(w[i], D);
        if (in) {
          L::put(dp, L::mul(q[i], D));
          L::put(dn, L::mul(z[i], D));
        }
      }
    } else {
#pragma unroll
      for (int i = GROUP - 1; i >= 0; --i, dp += step1, dn += step2) {
        if (i >= left) continue;
        if ((lasts >> i) & 1u) e = given<L>(a, o, m, i0 + i, true, a.d_state_out, c, in);
        const P D = L::add(g[i], e);
        e = L::mul(w[i], D);
        if (in) {
          L::put(dp, L::mul(q[i], D));
          L::put(dn, L::mul(z[i], D));
        }
        if ((begins >> (i0 + i)) & 1u) {
          const int64_t b = sequence(a, o, m, i0 + i, false);
          if (in) put_state<L>(a.d_state_in + b * a.C + c, e);
        }
      }
    }
  }
  __syncwarp();
}

template <class T, bool LONG>
__global__ void __launch_bounds__(BACK_WARPS * 32) back_kernel(const __grid_constant__ GsArgs a) {
  using L = Lane<T>;
  using P = typename L::P;
  constexpr int BLOCKS = L::V == 2 ? 4 : 3;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t bars[BACK_WARPS];
  empty_sequences(a, a.d_state_in, a.d_state_out);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full = smem_addr(&bars[warp]), buffer = smem_addr(smem) + warp * BLOCKS * BLOCK;
  if (lane == 0) {
    sm100::mbar_init(full, 1);
    sm100::fence_mbar_init();
  }
  __syncwarp();
  const int64_t unit = (int64_t)blockIdx.x * BACK_WARPS + warp;
  const int64_t k = unit / a.blocks;
  const int c0 = (int)(unit % a.blocks) * 32 * L::V, c = c0 + lane * L::V;
  const bool in = c < a.C;
  const Order& o = a.order;
  const Walk walk = walk_of(o, buffer);
  bool ok = true;
  P e = L::make(0.0f, 0.0f), h = e;
  int64_t lo, hi, next;
  if (a.n_rows == 0) return;
  extent(a, o, lo, hi);
  if constexpr (LONG) {
    // (windows as the flipped order's warps had them: from the last position on)
    const int64_t end = (a.windows - k * a.each) * WINDOW, first = end - a.each * WINDOW;
    const int64_t from = first < lo ? lo : first, upto = end < hi ? end : hi;
    if (k >= a.units || from >= upto) {
      after_kernels_before();
      return;
    }
    uint32_t parity = 0;
    int64_t j = border_at(a, o, upto, lane);
    for (int64_t pos = (upto - 1) / WINDOW * WINDOW; pos + WINDOW > from && pos >= 0 && ok; pos -= WINDOW, parity ^= 1) {
      const int64_t start = pos < lo ? lo : pos;
      bring<3>(buffer, full, o, start, c0, &a.tp, &a.tn, &a.tg);
      j = border_down(a, o, start, j, lane);
      const Window m = window_at(a, o, pos, lo, hi, j, lane, next);
      if (parity == 0 && pos + WINDOW >= upto) {
        after_kernels_before();
        if (!((m.ends >> (m.count - 1)) & 1u)) e = into<L>(a, k, c, in);
      }
      if (in) h = get_state<L>(a.saved + pos / WINDOW * a.C + c);
      ok = brought(full, parity);
      window_backward<T>(a, m, walk, c, in, h, e);
    }
  } else {
    // the sequences that begin in [from, upto), the last window first
    const int64_t from = k * a.chunk, upto = from + a.chunk;
    if (from >= hi) return;
    int64_t j = border_at(a, o, from, lane);
    if (j > a.n_seq) return;
    const int64_t run = border(a, o, j);
    if (run >= upto || run >= hi || run < lo) return;
    j = border_at(a, o, upto, lane);
    const int64_t end = j <= a.n_seq && border(a, o, j) < hi ? border(a, o, j) : hi;
    uint32_t parity = 0;
    for (int64_t pos = run + (end - run - 1) / WINDOW * WINDOW; ok && end > run && pos >= run; pos -= WINDOW, parity ^= 1) {
      bring<3>(buffer, full, o, pos, c0, &a.tp, &a.tn, &a.tg);
      j = border_down(a, o, pos, j, lane);
      const Window m = window_at(a, o, pos, lo, end, j, lane, next);
      if (in && pos > run) h = get_state<L>(a.saved + pos / WINDOW * a.C + c);
      ok = brought(full, parity);
      window_backward<T>(a, m, walk, c, in, h, e);
    }
  }
  if (!ok && lane == 0) atomicAdd(a.expired, 1ull);
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

// [rows][channels] with a row stride, boxes of 128 bytes x WINDOW rows; zeros beyond the array.
bool make_map(CUtensorMap* m, int32_t dtype, const void* p, int64_t rows, int64_t channels, int64_t stride) {
  const auto fn = encode_fn();
  if (!fn) return false;
  const int size = type_size(dtype);
  const cuuint64_t dims[2] = {(cuuint64_t)channels, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * size};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / size), WINDOW}, step[2] = {1, 1};
  const CUtensorMapDataType type = dtype == TRACKFIT_FP32        ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == TRACKFIT_BF16_PROJ ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return fn(m, type, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool channels_ok(int32_t c) { return c >= 8 && c <= MAX_CHANNELS && c % 8 == 0; }

// By the counts alone, since the lengths are on the device: 100,000 sequences of 31 rows, 192 channels in
// bf16, take 561 us as short ones, of 33 rows 656, as long ones 1,198.  (Lengths far apart cost it: 600 of 14
// rows and one of 12,000, which a warp walks alone, take 631 us, where they took 59 as long ones.)
bool is_long(int64_t n_rows, int64_t n_seq) { return n_rows > n_seq * SHORT; }
int64_t windows_of(int64_t n_rows) { return (n_rows + WINDOW - 1) / WINDOW; }

size_t workspace_bytes(int64_t n_rows, int64_t n_seq, int32_t channels) {
  if (!is_long(n_rows, n_seq)) return 0;
  const size_t w = windows_of(n_rows), s = (w + WARPS - 1) / WARPS;            // (segments at most)
  return (w * 2 + s * 3 + n_seq) * channels * 4 + (w + s) * 4;
}

// A call of the scan, forward or backward.
struct Call {
  int32_t dtype, reverse;
  void* workspace;
  size_t size;
};

// The checks that forward and backward share.
int check(const Call& f, const GsArgs& a) {
  if (!type_ok(f.dtype) || a.n_rows < 0 || a.n_rows > (int64_t)1 << 40 || a.n_seq < 0 || a.n_seq >= 0x7fffffff)
    return TRACKFIT_ERR_INVALID_ARG;
  if (!channels_ok(a.C)) return TRACKFIT_ERR_UNSUPPORTED;
  if (f.reverse != 0 && f.reverse != 1) return TRACKFIT_ERR_INVALID_ARG;
  if (mis16(f.workspace)) return TRACKFIT_ERR_INVALID_ARG;
  if (a.n_seq == 0) return TRACKFIT_OK;
  if (!a.offs || (reinterpret_cast<uintptr_t>(a.offs) & 7u)) return TRACKFIT_ERR_INVALID_ARG;
  if (mis16(a.state_in) || mis16(a.state_out) || mis16(a.d_state_in) || mis16(a.d_state_out) || mis16(a.saved))
    return TRACKFIT_ERR_INVALID_ARG;
  const int sz = type_size(f.dtype);
  if (a.n_rows > 0 && (!rows_ok(a.p, a.ps, a.C, sz) || !rows_ok(a.n, a.ns, a.C, sz))) return TRACKFIT_ERR_INVALID_ARG;
  if (a.n_rows > 0x7fffff00) return TRACKFIT_ERR_UNSUPPORTED;    // a copy's coordinates have 32 bits
  const size_t need = workspace_bytes(a.n_rows, a.n_seq, a.C);
  if (need > 0 && (!f.workspace || f.size < need)) return TRACKFIT_ERR_INVALID_ARG;
  return TRACKFIT_OK;
}

// A kernel that may begin before the one in front of it in the stream has ended.
inline cudaError_t follow(void (*kernel)(GsArgs), unsigned grid, int threads, size_t smem, cudaStream_t st, const GsArgs& a) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(grid), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st, cfg.attrs = &at, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <class T, bool BACK>
int launch(const Call& f, GsArgs& a, cudaStream_t st) {
  using L = Lane<T>;
  const int64_t N = a.n_rows;
  a.windows = windows_of(N), a.blocks = (a.C + 32 * L::V - 1) / (32 * L::V);
  a.order = f.reverse ? Order{1, N - 1} : Order{0, 0};
  // positions in the other order, windows the same: position' = 32 windows - 1 - position
  const int64_t end = a.windows * WINDOW;
  a.flipped = f.reverse ? Order{0, end - N} : Order{1, end - 1};
  a.expired = operator_expired();
  if (!a.expired) return TRACKFIT_ERR_CUDA;
  if (N > 0 && (!make_map(&a.tp, f.dtype, a.p, N, a.C, a.ps) || !make_map(&a.tn, f.dtype, a.n, N, a.C, a.ns) ||
                (BACK && !make_map(&a.tg, f.dtype, a.g, N, a.C, a.gs))))
    return TRACKFIT_ERR_CUDA;
  const bool lng = is_long(N, a.n_seq);
  int64_t n_units;
  if (lng) {
    // as many windows a warp as leave every SM two segments
    a.each = 8;
    while (a.each > 1 && (a.windows + WARPS * a.each - 1) / (WARPS * a.each) * a.blocks < 2 * 152) a.each /= 2;
    a.segments = (a.windows + WARPS * a.each - 1) / (WARPS * a.each);
    a.units = (a.windows + a.each - 1) / a.each;
    const int64_t seg = a.segments * a.C;
    a.warp_a = (float*)f.workspace, a.warp_b = a.warp_a + a.units * a.C;
    a.seg_a = a.warp_b + a.units * a.C, a.seg_b = a.seg_a + seg, a.seg_s = a.seg_b + seg;
    if (a.segments * a.blocks > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
    // the states given are read again where their sequences begin (end), when the state after a sequence
    // may already stand in the same place: then from a copy
    float* copy = a.seg_s + seg;
    const float*& given = BACK ? a.d_state_out : a.state_in;
    if (given && given == (BACK ? a.d_state_in : a.state_out)) {
      const cudaError_t e = cudaMemcpyAsync(copy, given, (size_t)a.n_seq * a.C * 4, cudaMemcpyDeviceToDevice, st);
      if (e != cudaSuccess) return tf_status_from_cuda(e);
      given = copy;
    }
    a.warp_has = (uint32_t*)(copy + a.n_seq * a.C), a.seg_has = a.warp_has + a.units;
    constexpr auto sums = sums_kernel<T, BACK>;
    constexpr size_t smem = 2 * BLOCK * WARPS;
    const cudaError_t e = allow_smem<sums>(smem + 8192);
    if (e != cudaSuccess) return tf_status_from_cuda(e);
    sums<<<(unsigned)(a.segments * a.blocks), WARPS * 32, smem, st>>>(a);
    const cudaError_t e1 = follow(chain_kernel, (unsigned)((a.C + 63) / 64), 64, 0, st, a);
    if (e1 != cudaSuccess) return tf_status_from_cuda(e1);
    n_units = a.units * a.blocks;
  } else {
    // 128 rows a warp: the rest of its last sequence is a few rows more; fewer where warps are few
    a.chunk = 128;
    while (a.chunk > 16 && (N + a.chunk - 1) / a.chunk * a.blocks < 152 * 24) a.chunk /= 2;
    n_units = (N + a.chunk - 1) / a.chunk * a.blocks;
  }
  constexpr int warps = BACK ? BACK_WARPS : WARPS;
  int64_t grid = (n_units + warps - 1) / warps;
  if (grid < 1) grid = a.n_seq < 8 * 152 ? (a.n_seq + warps - 1) / warps : 2 * 152;    // states of empty sequences only
  if (grid > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  constexpr size_t smem = (BACK ? (L::V == 2 ? 4 : 3) : 2) * BLOCK * warps;
  constexpr auto kernels = [] {
    if constexpr (BACK) return std::make_pair(&back_kernel<T, false>, &back_kernel<T, true>);
    else return std::make_pair(&rows_kernel<T, false>, &rows_kernel<T, true>);
  }();
  const cudaError_t e = lng ? allow_smem<kernels.second>(smem + 1024) : allow_smem<kernels.first>(smem + 1024);   // (with the barriers)
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  if (!lng) {
    kernels.first<<<(unsigned)grid, warps * 32, smem, st>>>(a);
  } else {
    const cudaError_t e2 = follow(kernels.second, (unsigned)grid, warps * 32, smem, st, a);
    if (e2 != cudaSuccess) return tf_status_from_cuda(e2);
  }
  return launched();
}

template <bool BACK>
int by_type(const Call& f, GsArgs& a, cudaStream_t st) {
  return f.dtype == TRACKFIT_FP32        ? launch<float, BACK>(f, a, st)
         : f.dtype == TRACKFIT_BF16_PROJ ? launch<__nv_bfloat16, BACK>(f, a, st)
                                         : launch<__half, BACK>(f, a, st);
}

}  // namespace

extern "C" size_t trackfit_gated_scan_saved(int64_t n_rows, int32_t channels) {
  if (n_rows < 0 || n_rows > (int64_t)1 << 40 || !channels_ok(channels)) return 0;
  return (size_t)windows_of(n_rows) * channels * 4;
}

extern "C" size_t trackfit_gated_scan_workspace(int32_t dtype, int64_t n_rows, int64_t n_seq, int32_t channels) {
  if (!type_ok(dtype) || n_rows < 0 || n_rows > (int64_t)1 << 40 || n_seq < 0 || !channels_ok(channels)) return 0;
  return workspace_bytes(n_rows, n_seq, channels);
}

extern "C" int trackfit_gated_scan(int32_t dtype, const void* gate, int64_t gate_stride, const void* cand,
                                   int64_t cand_stride, int64_t n_rows, const int64_t* offsets, int64_t n_seq,
                                   int32_t channels, int32_t reverse, const float* state_in, float* state_out,
                                   float* saved, void* out, int64_t out_stride, void* workspace, size_t workspace_size,
                                   void* stream) {
  tf_nvtx_range nvtx_range("trackfit_gated_scan");
  const Call f = {dtype, reverse, workspace, workspace_size};
  GsArgs a = {};
  a.p = gate, a.ps = gate_stride, a.n = cand, a.ns = cand_stride;
  a.out = out, a.os = out_stride;
  a.offs = offsets, a.n_rows = n_rows, a.n_seq = n_seq, a.C = channels;
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
  const Call f = {dtype, reverse, workspace, workspace_size};
  GsArgs a = {};
  a.p = gate, a.ps = gate_stride, a.n = cand, a.ns = cand_stride, a.g = d_out, a.gs = d_out_stride;
  a.dp = d_gate, a.dps = d_gate_stride, a.dn = d_cand, a.dns = d_cand_stride;
  a.offs = offsets, a.n_rows = n_rows, a.n_seq = n_seq, a.C = channels;
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
