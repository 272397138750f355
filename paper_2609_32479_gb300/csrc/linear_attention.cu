// Linear attention with a decay a head over packed sequences, and by single tokens.
//
//   S_t = exp(g_t) S_{t-1} + k_t v_t^T      S: K x V, fp32;  g_t: one value a row and head
//   o_t = scale S_t^T q_t
//
// A column of S needs its own channel of v only, so the columns are split over warps without any
// exchange.  How the packed rows are cut into units: see
// linear_units.cuh.
#include "linear_units.cuh"

namespace {
using namespace seqops;

// ---------------------------------------------------------------- fp32, on the CUDA cores
// A lane holds halves of CPL columns of S, K / 2 values each in registers; the lanes l and l + 16
// have a column's halves.  The rows of q and k are the same for all columns and come from shared
// memory as broadcasts, 8 rows at a time through a ring that the warp fills by asynchronous
// copies.  Several columns a lane share what a row costs whatever its columns (loads,
// exponentials, addresses: 90 of 116 instructions with one).  Measured: 20,011 tracks and parts
// of tracks, 4 heads of 32 x 48, states in and out: 774 us a call, 3.4 TB/s; one column a lane 1136.
// Every row decays the state itself: a factor kept beside it, which would save the product, makes
// values up to that factor larger than the state.  A small decay goes in as S + (e^g - 1) S: e^g
// rounded would be an error that all values of the state have in common, 2^-25 a row, which no sum
// over them lessens (over 2,000 rows 2.4e-6 of the output; 4e-7 are left).
constexpr int CH = 8, NST = 2;

template <int DK, int CPL>
struct __align__(16) SimtSlot {
  float q[CH][DK], k[CH][DK], v[CH][16 * CPL];
  float g[CH];
  int row, seq, flags, pad;      // the chunk, its first row in the direction of the recurrence
  // behind it, where sequences begin with a state: the state's columns of a piece's first chunk,
  // [K][16 CPL] (loaded when the chunk came up, they kept the warps waiting half of the time)
  __device__ float* state() { return reinterpret_cast<float*>(this + 1); }
};
template <int DK, int CPL>
inline int simt_slot_bytes(const LaArgs& a) {
  return (int)sizeof(SimtSlot<DK, CPL>) + (a.state_in || a.bounds > 1 ? a.K * 16 * CPL * 4 : 0);
}
enum { LEN = 0xff, FIRST = 0x100, LAST = 0x200, GOES_ON = 0x400, ENDS = 0x800, NONE = 0x1000 };

template <int DK, int CPL, bool STATE_ONLY>
__global__ void __launch_bounds__(32) la_simt_kernel(const __grid_constant__ LaArgs a, int slot_bytes) {
  extern __shared__ __align__(16) unsigned char smem[];
  using Slot = SimtSlot<DK, CPL>;
  constexpr int COLS = 16 * CPL;
  const int lane = threadIdx.x;
  const unsigned unit = blockIdx.x;
  const int sl = (int)(unit % a.slices), h = (int)(unit / a.slices % a.H);
  const int64_t tile = unit / a.slices / a.H;
  auto slot = [&](int s) -> Slot& { return *reinterpret_cast<Slot*>(smem + s * slot_bytes); };
  const int c0 = sl * COLS, width = a.V - c0 < COLS ? a.V - c0 : COLS;
  const int dir = a.u.reverse ? -1 : 1;
  constexpr int HALF = DK / 2;
  const int col = lane & 15, part = lane >> 4, i0 = part * HALF;   // this lane's columns: col + 16 j; first key channel
  // channels beyond K and V are zeros from here on: the copies leave them alone
  for (int i = lane * 4; i < NST * slot_bytes; i += 128) *reinterpret_cast<uint32_t*>(smem + i) = 0;
  __syncwarp();

  const int64_t base = STATE_ONLY ? (tile + 1) * a.u.lseg : tile * a.u.seg;
  const float* q = (const float*)a.q + base * a.qs + h * a.K;
  const float* k = (const float*)a.k + base * a.ks + h * a.K;
  const float* v = (const float*)a.v + base * a.vs + h * a.V + c0;
  const float* gr = a.g + base * a.gs + h;
  float* out = (float*)a.out + base * a.os + h * a.V + c0 + col;
  TilePieces pieces(a.u, tile, lane, STATE_ONLY);
  Piece p;
  bool more;
  if (STATE_ONLY) {
    more = boundary_piece(a.u, tile + 1, lane, p);
    if (sl == 0 && h == 0 && lane == 0) a.ws_flag[tile + 1] = !more ? 0 : p.goes_on ? 2 : 1;
  } else {
    more = pieces.next(p);
  }
  int done = 0;
  const int64_t KV = (int64_t)a.K * a.V;
  const int block = STATE_ONLY ? 0 : block_of(a.u, tile);
  auto beginning = [&](bool goes_on, bool ends, int seq) {
    return STATE_ONLY ? boundary_begins_with(a, seq, h, goes_on) : piece_begins_with(a, block, seq, h, goes_on, ends);
  };

  auto issue = [&](Slot& w) {
    if (more) {
      const int left = p.hi - p.lo - done;
      const int len = left < CH ? left : CH;
      const int row = a.u.reverse ? p.hi - 1 - done : p.lo + done;
      if (lane == 0) {
        w.row = row, w.seq = p.seq;
        w.flags = len | (done == 0 ? FIRST : 0) | (left <= CH ? LAST : 0) | (p.goes_on ? GOES_ON : 0) | (p.ends ? ENDS : 0);
      }
#pragma unroll
      for (int i = 0; i < CH * DK / 128; ++i) {
        const int r = (lane + 32 * i) / (DK / 4), e = (lane + 32 * i) % (DK / 4) * 4;
        if (e < a.K) {
          const int64_t at = row + dir * r;
          if (!STATE_ONLY) copy16(smem_addr(&w.q[r][e]), q + at * a.qs + e, r < len);
          copy16(smem_addr(&w.k[r][e]), k + at * a.ks + e, r < len);
        }
      }
#pragma unroll
      for (int i = 0; i < CPL; ++i) {
        const int r = (lane + 32 * i) / (COLS / 4), e = (lane + 32 * i) % (COLS / 4) * 4;
        if (e < width) copy16(smem_addr(&w.v[r][e]), v + (int64_t)(row + dir * r) * a.vs + e, r < len);
      }
      if (lane < CH) copy4(smem_addr(&w.g[lane]), gr + (int64_t)(row + dir * lane) * a.gs, lane < len);
      if (done == 0) {
        if (const float* src = beginning(p.goes_on, p.ends, p.seq)) {
          for (int i = lane; i < a.K * (COLS / 4); i += 32) {
            const int r = i / (COLS / 4), e = i % (COLS / 4) * 4;
            if (e < width) copy16(smem_addr(w.state() + 4 * i), src + r * a.V + c0 + e, true);
          }
        }
      }
      done += len;
      if (left <= CH) {
        done = 0;
        more = STATE_ONLY ? false : pieces.next(p);
      }
    } else if (lane == 0) {
      w.flags = NONE;
    }
    copy_commit();
  };

  for (int s = 0; s < NST; ++s) issue(slot(s));
  uint64_t S[CPL][HALF / 2];     // pairs of key channels, an instruction for two
#pragma unroll
  for (int j = 0; j < CPL; ++j)
#pragma unroll
    for (int i = 0; i < HALF / 2; ++i) S[j][i] = 0;
  auto put_state = [&](float* st) {
#pragma unroll
    for (int j = 0; j < CPL; ++j)
#pragma unroll
      for (int i = 0; i < HALF; i += 2)
        if (col + 16 * j < width && i0 + i < a.K) {
          const float2 x = parts(S[j][i / 2]);
          st[(i0 + i) * a.V + c0 + col + 16 * j] = x.x, st[(i0 + i + 1) * a.V + c0 + col + 16 * j] = x.y;
        }
  };
  float total = 0.0f;
  for (int s = 0;; s = s + 1 == NST ? 0 : s + 1) {
    Slot& w = slot(s);
    copy_wait<NST - 1>();
    __syncwarp();
    const int flags = w.flags, row = w.row, seq = w.seq, len = flags & LEN;
    if (flags & NONE) break;
    if (flags & FIRST) {
      const bool st = beginning(flags & GOES_ON, flags & ENDS, seq) != nullptr;
      const float* src = w.state() + i0 * COLS + col;
#pragma unroll
      for (int j = 0; j < CPL; ++j)
#pragma unroll
        for (int i = 0; i < HALF; i += 2)
          S[j][i / 2] = st && i0 + i < a.K ? both(src[i * COLS + 16 * j], src[(i + 1) * COLS + 16 * j]) : 0;
      if (STATE_ONLY && a.ws_begin && !(flags & GOES_ON)) put_state(a.ws_begin + ((tile + 1) * a.H + h) * KV);
    }
    // the rows' decays, a lane each: e^g - 1 of a small one, which is not positive, else e^g, which is
    // (-1 where it is zero)
    if (lane < len) {
      const float x = w.g[lane];
      float e = x > -0.5f && x <= 0.0f ? expm1f(x) : expf(x);
      if (e == 0.0f && x < 0.0f) e = x > -0.5f ? e : -1.0f;
      if (STATE_ONLY) total += x;
      w.g[lane] = e;
    }
    __syncwarp();
    for (int r = 0; r < len; ++r) {
      const float e = w.g[r];
      const uint64_t e2 = both(e, e);
      uint64_t x[CPL], acc[CPL];
#pragma unroll
      for (int j = 0; j < CPL; ++j) x[j] = both(w.v[r][col + 16 * j], w.v[r][col + 16 * j]), acc[j] = 0;
      auto step = [&](auto decayed) {
#pragma unroll
        for (int i = 0; i < HALF; i += 4) {
          const ulonglong2 k4 = *reinterpret_cast<const ulonglong2*>(&w.k[r][i0 + i]);
          ulonglong2 q4;
          if (!STATE_ONLY) q4 = *reinterpret_cast<const ulonglong2*>(&w.q[r][i0 + i]);
#pragma unroll
          for (int j = 0; j < CPL; ++j) {
            uint64_t &s0 = S[j][i / 2], &s1 = S[j][i / 2 + 1];
            s0 = fma2(k4.x, x[j], decayed(s0)), s1 = fma2(k4.y, x[j], decayed(s1));
            if (!STATE_ONLY) acc[j] = fma2(q4.y, s1, fma2(q4.x, s0, acc[j]));
          }
        }
      };
      if (e <= 0.0f) step([e2](uint64_t s) { return fma2(s, e2, s); });
      else step([e2](uint64_t s) { return mul2(s, e2); });
      if (!STATE_ONLY) {
        float* o = out + (int64_t)(row + dir * r) * a.os;
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
          const float2 p = parts(acc[j]);
          float y = p.x + p.y;
          y += __shfl_xor_sync(FULL, y, 16);
          if (part == 0 && col + 16 * j < width) o[16 * j] = a.scale * y;
        }
      }
    }
    if ((flags & LAST) && (STATE_ONLY || ((flags & ENDS) && a.state_out))) {
      put_state(STATE_ONLY ? a.ws_state + ((tile + 1) * a.H + h) * KV : a.state_out + ((int64_t)seq * a.H + h) * KV);
      if (STATE_ONLY) {
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) total += __shfl_xor_sync(FULL, total, o);
        if (sl == 0 && lane == 0) a.ws_decay[(tile + 1) * a.H + h] = total;
      }
    }
    __syncwarp();
    issue(w);
  }
}

// What crosses each boundary: the pieces' own states, in the direction of the recurrence,
// each with the decayed state of the boundary before it.  A thread takes one value of a
// head's state through all boundaries; the CTA looks at 128 boundaries' flags at a time and
// passes over those that no cut sequence crosses.
constexpr int CARRY_NT = 128;
__global__ void __launch_bounds__(CARRY_NT) la_carry_kernel(const __grid_constant__ LaArgs a) {
  __shared__ int flag[CARRY_NT];
  const int64_t KV = (int64_t)a.K * a.V;
  const int64_t e = (int64_t)blockIdx.x * CARRY_NT + threadIdx.x;
  const bool on = e < KV * a.H;
  const int h = on ? (int)(e / KV) : 0;
  float carry = 0.0f;
  constexpr int AHEAD = 16;      // boundaries whose loads are under way together
  for (int64_t j0 = 1; j0 < a.bounds; j0 += CARRY_NT) {
    const int64_t jt = j0 + threadIdx.x;
    const int mine = jt < a.bounds ? a.ws_flag[a.u.reverse ? a.bounds - jt : jt] : 0;
    const int any = __syncthreads_or(mine != 0);   // (also: the flags before are done with)
    if (!any) continue;                            // the next chain begins with a flag of 1
    flag[threadIdx.x] = mine;
    __syncthreads();
    for (int n0 = 0; n0 < CARRY_NT && on; n0 += AHEAD) {
      float x[AHEAD], d[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) {
        const int64_t j = j0 + n0 + n, i = a.u.reverse ? a.bounds - j : j;
        x[n] = d[n] = 0.0f;
        if (flag[n0 + n] != 0) x[n] = a.ws_state[i * a.H * KV + e], d[n] = a.ws_decay[i * a.H + h];
      }
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) {
        if (flag[n0 + n] == 0) continue;           // nothing was written there
        const int64_t j = j0 + n0 + n, i = a.u.reverse ? a.bounds - j : j;
        carry = flag[n0 + n] == 2 ? fmaf(expf(d[n]), carry, x[n]) : x[n];
        a.ws_state[i * a.H * KV + e] = carry;
      }
    }
  }
}

// ---------------------------------------------------------------- a single token
// A warp takes 32 columns of a head's state: 8 lanes hold four columns of a row each, and
// four rows are read, decayed, added to and written at a time.  The state's two crossings
// of memory are nearly all of the traffic, and bound it: 8,192 sequences, 8 heads of 64 x 64,
// 364 us, 6.0 TB/s of the 6.8 that a copy moves.
constexpr int NW = 4;            // warps of a CTA
constexpr int STEP_COLS = 32;    // columns that a warp takes
struct StepArgs {
  const void *q, *k, *v;
  const float* g;
  void* out;
  int64_t qs, ks, vs, gs, os;
  const int32_t* slots;
  const float* state_in;
  float* state_out;
  int64_t n, n_slots;
  int H, K, V, slices;
  float scale;
};

template <class T>
__global__ void __launch_bounds__(NW * 32) la_step_kernel(const __grid_constant__ StepArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = (int64_t)blockIdx.x * NW + warp;
  const int sl = (int)(unit % a.slices), h = (int)(unit / a.slices % a.H);
  const int64_t b = unit / a.slices / a.H;
  if (b >= a.n) return;
  const int c = sl * STEP_COLS + (lane & 7) * 4, r0 = lane >> 3;
  const bool on = c < a.V;
  T* out = (T*)a.out + b * a.os + h * a.V + c;
  const int64_t slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    if (on && r0 == 0)
      for (int j = 0; j < 4; ++j) put(out + j, __uint_as_float(0x7fffffffu));
    return;
  }
  const T* q = (const T*)a.q + b * a.qs + h * a.K;
  const T* k = (const T*)a.k + b * a.ks + h * a.K;
  const T* v = (const T*)a.v + b * a.vs + h * a.V + c;
  const float e = expf(a.g[b * a.gs + h]);
  float vr[4] = {0.0f, 0.0f, 0.0f, 0.0f}, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (on)
    for (int j = 0; j < 4; ++j) vr[j] = to_float(v[j]);
  const int64_t base = (slot * a.H + h) * (int64_t)a.K * a.V + c;
#pragma unroll 8
  for (int i = r0; i < a.K; i += 4) {
    if (!on) continue;
    const float4 s = *reinterpret_cast<const float4*>(a.state_in + base + (int64_t)i * a.V);
    const float ki = to_float(k[i]), qi = to_float(q[i]);
    float4 n;
    n.x = fmaf(ki, vr[0], e * s.x), n.y = fmaf(ki, vr[1], e * s.y);
    n.z = fmaf(ki, vr[2], e * s.z), n.w = fmaf(ki, vr[3], e * s.w);
    *reinterpret_cast<float4*>(a.state_out + base + (int64_t)i * a.V) = n;
    acc[0] = fmaf(qi, n.x, acc[0]), acc[1] = fmaf(qi, n.y, acc[1]);
    acc[2] = fmaf(qi, n.z, acc[2]), acc[3] = fmaf(qi, n.w, acc[3]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    acc[j] += __shfl_xor_sync(FULL, acc[j], 8);
    acc[j] += __shfl_xor_sync(FULL, acc[j], 16);
    if (on && r0 == 0) put(out + j, a.scale * acc[j]);
  }
}

// ---------------------------------------------------------------- host
// Rows a boundary: as many as leave one unit for each of the 152 x 8 warps that the widest
// kernels keep on the GPU, but not under 256 (a state is written and read twice a boundary).
int rows_a_boundary(int64_t n_rows, int H, int V) {
  const int64_t units_a_row = (int64_t)H * ((V + 31) / 32);
  const int64_t l = (n_rows * units_a_row / (152 * 8) + 255) / 256 * 256;
  return l < 256 ? 256 : l > 2048 ? 2048 : (int)l;
}
constexpr int LONGEST = 512;   // longer sequences are cut

// Whether any may be: not where there are few rows of sequences that are short on average, for which
// the two launches are the longer part of a call (an event of 211 tracks: 13 us instead of 6 on the
// device).  What that costs where a long one is among them: 250 tracks of 14 rows and a sequence of
// 12,000, 4 heads of 32, take 722 us uncut (fp32 2,268); with 200 tracks, cut, 55 (129).
bool cuts(int64_t n_rows, int64_t n_seq) { return n_rows > LONGEST && (n_rows > 16384 || n_rows > 64 * n_seq); }

size_t workspace_bytes(int64_t n_rows, int64_t n_seq, int H, int K, int V) {
  if (!cuts(n_rows, n_seq)) return 0;
  const int l = rows_a_boundary(n_rows, H, V);
  const size_t bounds = (size_t)((n_rows + l - 1) / l);
  const size_t flags = (bounds * 4 + 15) / 16 * 16, decay = (bounds * H * 4 + 15) / 16 * 16;
  return flags + decay + 2 * bounds * H * (size_t)K * V * 4;   // (the second: states in place)
}

template <int DK, int CPL, bool STATE_ONLY>
int launch_simt(const LaArgs& a, cudaStream_t st) {
  const int bytes = simt_slot_bytes<DK, CPL>(a);
  static_assert((sizeof(SimtSlot<DK, CPL>) + DK * 16 * CPL * 4) * NST <= 48 * 1024, "needs no leave");
  la_simt_kernel<DK, CPL, STATE_ONLY><<<linear_grid(a, STATE_ONLY), 32, NST * bytes, st>>>(a, bytes);
  return launched();
}
// Columns a lane, at most 64 registers of state, the slices alike.
int columns_a_lane(int K, int V) {
  const int most = K <= 32 ? 4 : K <= 64 ? 2 : 1, all = (V + 15) / 16, slices = (all + most - 1) / most;
  return (all + slices - 1) / slices;
}
template <int DK, bool STATE_ONLY>
int by_columns(const LaArgs& a, cudaStream_t st) {
  const int c = columns_a_lane(a.K, a.V);
  if constexpr (DK <= 32) {
    if (c == 4) return launch_simt<DK, 4, STATE_ONLY>(a, st);
    if (c == 3) return launch_simt<DK, 3, STATE_ONLY>(a, st);
  }
  if constexpr (DK <= 64) {
    if (c == 2) return launch_simt<DK, 2, STATE_ONLY>(a, st);
  }
  return launch_simt<DK, 1, STATE_ONLY>(a, st);
}
template <bool STATE_ONLY>
int run(int32_t dtype, const LaArgs& a, cudaStream_t st) {
  if (dtype != TRACKFIT_FP32) return linear_mma(dtype, a, STATE_ONLY, st);
  if (a.K <= 16) return by_columns<16, STATE_ONLY>(a, st);
  if (a.K <= 32) return by_columns<32, STATE_ONLY>(a, st);
  if (a.K <= 64) return by_columns<64, STATE_ONLY>(a, st);
  return by_columns<128, STATE_ONLY>(a, st);
}

}  // namespace

extern "C" size_t trackfit_linear_attention_workspace(int64_t n_rows, int64_t n_seq, int32_t n_heads,
                                                      int32_t key_dim, int32_t value_dim) {
  if (n_rows < 0 || n_rows > (int64_t)1 << 40 || n_seq <= 0 || !heads_ok(n_heads) || !dim_ok(key_dim) || !dim_ok(value_dim)) return 0;
  return workspace_bytes(n_rows, n_seq, n_heads, key_dim, value_dim);
}

extern "C" int trackfit_linear_attention(int32_t dtype, const void* q, int64_t q_stride, const void* k,
                                         int64_t k_stride, const void* v, int64_t v_stride, const float* log_decay,
                                         int64_t decay_stride, int64_t n_rows, const int64_t* offsets, int64_t n_seq,
                                         int32_t n_heads, int32_t key_dim, int32_t value_dim, float scale,
                                         int32_t reverse, const float* state_in, float* state_out, void* out,
                                         int64_t out_stride, void* workspace, size_t workspace_size, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_linear_attention");
  if (!type_ok(dtype) || n_rows < 0 || n_rows > (int64_t)1 << 40 || n_seq < 0 || n_seq > 0x7fffffff)
    return TRACKFIT_ERR_INVALID_ARG;
  if (!heads_ok(n_heads) || !dim_ok(key_dim) || !dim_ok(value_dim)) return TRACKFIT_ERR_UNSUPPORTED;
  if (!isfinite(scale) || (reverse != 0 && reverse != 1)) return TRACKFIT_ERR_INVALID_ARG;
  if (n_seq == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!offsets || (reinterpret_cast<uintptr_t>(offsets) & 7u)) return TRACKFIT_ERR_INVALID_ARG;
  if (mis16(state_in) || mis16(state_out)) return TRACKFIT_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!rows_ok(q, q_stride, (int64_t)n_heads * key_dim, sz) || !rows_ok(k, k_stride, (int64_t)n_heads * key_dim, sz) ||
        !rows_ok(v, v_stride, (int64_t)n_heads * value_dim, sz) ||
        !rows_ok(out, out_stride, (int64_t)n_heads * value_dim, sz))
      return TRACKFIT_ERR_INVALID_ARG;
    if (!log_decay || mis4(log_decay) || decay_stride < n_heads || decay_stride > MAX_STRIDE)
      return TRACKFIT_ERR_INVALID_ARG;
  }
  const size_t need = workspace_bytes(n_rows, n_seq, n_heads, key_dim, value_dim);
  if (need > 0 && (!workspace || mis16(workspace) || workspace_size < need)) return TRACKFIT_ERR_INVALID_ARG;
  LaArgs a;
  a.q = q, a.k = k, a.v = v, a.g = log_decay, a.out = out;
  a.qs = q_stride, a.ks = k_stride, a.vs = v_stride, a.gs = decay_stride, a.os = out_stride;
  a.state_in = state_in, a.state_out = state_out;
  const int cols = dtype == TRACKFIT_FP32 ? 16 * columns_a_lane(key_dim, value_dim) : linear_mma_cols(key_dim);
  a.H = n_heads, a.K = key_dim, a.V = value_dim, a.slices = (value_dim + cols - 1) / cols;
  a.scale = scale;
  a.u.offs = offsets, a.u.n_seq = n_seq, a.u.n_rows = n_rows, a.u.reverse = reverse;
  a.u.lseg = rows_a_boundary(n_rows, n_heads, value_dim);
  a.u.longest = need > 0 ? LONGEST : 0x7fffffff;
  // few rows: small tiles, so that there are units for every SM; long sequences: none that
  // would find nothing to do between two boundaries
  a.u.seg = 256;
  while (a.u.seg > 16 && n_rows / a.u.seg * n_heads * a.slices < 2400) a.u.seg /= 2;
  if (n_rows / n_seq >= LONGEST) a.u.seg = a.u.lseg;
  a.u.tiles = n_rows > 0 ? (n_rows + a.u.seg - 1) / a.u.seg : 1;
  a.bounds = 1;
  a.ws_begin = nullptr;
  if (a.u.tiles > (int64_t)0x7fffffff / (n_heads * a.slices)) return TRACKFIT_ERR_UNSUPPORTED;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (need > 0) {
    a.bounds = (n_rows + a.u.lseg - 1) / a.u.lseg;
    unsigned char* w = static_cast<unsigned char*>(workspace);
    a.ws_flag = reinterpret_cast<int32_t*>(w);
    w += (a.bounds * 4 + 15) / 16 * 16;
    a.ws_decay = reinterpret_cast<float*>(w);
    w += (a.bounds * n_heads * 4 + 15) / 16 * 16;
    a.ws_state = reinterpret_cast<float*>(w);
    if (state_in && state_in == state_out) a.ws_begin = a.ws_state + a.bounds * n_heads * key_dim * value_dim;
    if (a.bounds > 1) {
      int rc = run<true>(dtype, a, st);
      if (rc != TRACKFIT_OK) return rc;
      const int64_t n = (int64_t)n_heads * key_dim * value_dim;
      la_carry_kernel<<<(unsigned)((n + CARRY_NT - 1) / CARRY_NT), CARRY_NT, 0, st>>>(a);
      rc = launched();
      if (rc != TRACKFIT_OK) return rc;
    }
  } else {
    a.ws_flag = nullptr, a.ws_decay = a.ws_state = nullptr;
  }
  return run<false>(dtype, a, st);
}

extern "C" int trackfit_linear_attention_step(int32_t dtype, const void* q, int64_t q_stride, const void* k,
                                              int64_t k_stride, const void* v, int64_t v_stride,
                                              const float* log_decay, int64_t decay_stride, int64_t n_seq,
                                              int32_t n_heads, int32_t key_dim, int32_t value_dim, float scale,
                                              const int32_t* slots, int64_t n_slots, const float* state_in,
                                              float* state_out, void* out, int64_t out_stride, void* stream) {
  tf_nvtx_range nvtx_range("trackfit_linear_attention_step");
  if (!type_ok(dtype) || n_seq < 0 || n_seq > 0x7fffffff || n_slots < 0) return TRACKFIT_ERR_INVALID_ARG;
  if (!heads_ok(n_heads) || !dim_ok(key_dim) || !dim_ok(value_dim)) return TRACKFIT_ERR_UNSUPPORTED;
  if (!isfinite(scale) || (!slots && n_slots < n_seq)) return TRACKFIT_ERR_INVALID_ARG;
  if (n_seq == 0) return TRACKFIT_OK;
  const int sz = type_size(dtype);
  if (!rows_ok(q, q_stride, (int64_t)n_heads * key_dim, sz) || !rows_ok(k, k_stride, (int64_t)n_heads * key_dim, sz) ||
      !rows_ok(v, v_stride, (int64_t)n_heads * value_dim, sz) ||
      !rows_ok(out, out_stride, (int64_t)n_heads * value_dim, sz))
    return TRACKFIT_ERR_INVALID_ARG;
  if (!log_decay || mis4(log_decay) || decay_stride < n_heads || decay_stride > MAX_STRIDE)
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(slots) || !state_in || !state_out || mis16(state_in) || mis16(state_out)) return TRACKFIT_ERR_INVALID_ARG;
  StepArgs a;
  a.q = q, a.k = k, a.v = v, a.g = log_decay, a.out = out;
  a.qs = q_stride, a.ks = k_stride, a.vs = v_stride, a.gs = decay_stride, a.os = out_stride;
  a.slots = slots, a.state_in = state_in, a.state_out = state_out, a.n = n_seq, a.n_slots = n_slots;
  a.H = n_heads, a.K = key_dim, a.V = value_dim, a.slices = (value_dim + STEP_COLS - 1) / STEP_COLS, a.scale = scale;
  const int64_t units = n_seq * n_heads * a.slices;
  if ((units + NW - 1) / NW > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((units + NW - 1) / NW);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) la_step_kernel<float><<<grid, NW * 32, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) la_step_kernel<__nv_bfloat16><<<grid, NW * 32, 0, st>>>(a);
  else la_step_kernel<__half><<<grid, NW * 32, 0, st>>>(a);
  return launched();
}
