// Linear attention with a decay a head over packed sequences, and by single tokens.
//
//   S_t = exp(g_t) S_{t-1} + k_t v_t^T      S: K x V, fp32;  g_t: one value a row and head
//   o_t = scale S_t^T q_t
//
// A column of S needs its own channel of v only, so the columns are split over warps, 32
// channels each, without any exchange.  How the packed rows are cut into units: see
// linear_units.cuh.
#include "linear_units.cuh"

namespace {
using namespace seqops;

// A chunk of a piece: up to CH rows, in the direction of the recurrence.
struct Chunk {
  int64_t row;                   // its first row
  int64_t seq;
  int len;                       // rows; 0 only for a sequence without rows
  bool first, last;              // of its piece
  int64_t from;
  bool ends;
};

// ---------------------------------------------------------------- CUDA cores
// A lane holds a column of S: K values in registers.  The rows of q and k are the same for
// all lanes and come from shared memory as broadcasts.
constexpr int COLS = 32;         // channels of v that a warp takes
constexpr int CH = 8, NST = 3;

template <class T, int DK>
struct SimtSlot {
  T q[CH][DK], k[CH][DK], v[CH][COLS];
  float g[CH];
};

template <class T, int DK, bool STATE_ONLY>
__global__ void __launch_bounds__(NW * 32) la_simt_kernel(const __grid_constant__ LaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  using Slot = SimtSlot<T, DK>;
  constexpr int VE = 16 / sizeof(T);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = (int64_t)blockIdx.x * NW + warp;
  const int sl = (int)(unit % a.slices), h = (int)(unit / a.slices % a.H);
  const int64_t tile = unit / a.slices / a.H;
  if (tile >= (STATE_ONLY ? a.bounds - 1 : a.u.tiles)) return;
  Slot* slots = reinterpret_cast<Slot*>(smem) + warp * NST;
  const int c0 = sl * COLS, width = a.V - c0 < COLS ? a.V - c0 : COLS;
  const int dir = a.u.reverse ? -1 : 1;
  // channels beyond K and V are zeros from here on: the copies leave them alone
  for (uint32_t* p = reinterpret_cast<uint32_t*>(slots) + lane; p < reinterpret_cast<uint32_t*>(slots + NST); p += 32) *p = 0;
  __syncwarp();

  const T* q = (const T*)a.q + h * a.K;
  const T* k = (const T*)a.k + h * a.K;
  const T* v = (const T*)a.v + h * a.V + c0;
  TilePieces pieces(a.u, tile, lane, STATE_ONLY);
  Piece p;
  bool more;
  int64_t bound = 0;
  if (STATE_ONLY) {
    bound = tile + 1;
    more = boundary_piece(a.u, bound, lane, p);
    if (sl == 0 && h == 0 && lane == 0) a.ws_flag[bound] = !more ? 0 : p.from < 0 ? 1 : 2;
  } else {
    more = pieces.next(p);
  }
  int64_t done = 0;
  Chunk ring[NST];

  auto issue = [&](int s) {
    Chunk& c = ring[s];
    c.len = -1;
    if (more) {
      const int64_t left = p.hi - p.lo - done;
      c.len = (int)(left < CH ? left : CH);
      c.row = a.u.reverse ? p.hi - 1 - done : p.lo + done;
      c.first = done == 0, c.last = left <= CH;
      c.seq = p.seq, c.from = p.from, c.ends = p.ends;
      Slot& w = slots[s];
      const int kv = a.K / VE, vv = width / VE;
      for (int i = lane; i < CH * kv; i += 32) {
        const int r = i / kv, e = (i - r * kv) * VE;
        const bool on = r < c.len;
        const int64_t row = on ? c.row + dir * r : 0;
        if (!STATE_ONLY) copy16(smem_addr(&w.q[r][e]), q + row * a.qs + e, on);
        copy16(smem_addr(&w.k[r][e]), k + row * a.ks + e, on);
      }
      for (int i = lane; i < CH * vv; i += 32) {
        const int r = i / vv, e = (i - r * vv) * VE;
        const bool on = r < c.len;
        copy16(smem_addr(&w.v[r][e]), v + (on ? c.row + dir * r : 0) * a.vs + e, on);
      }
      if (lane < CH) copy4(smem_addr(&w.g[lane]), a.g + (lane < c.len ? c.row + dir * lane : 0) * a.gs + h, lane < c.len);
      done += c.len;
      if (c.last) {
        done = 0;
        more = STATE_ONLY ? false : pieces.next(p);
      }
    }
    copy_commit();
  };

#pragma unroll
  for (int s = 0; s < NST; ++s) issue(s);
  float S[DK];
#pragma unroll
  for (int i = 0; i < DK; ++i) S[i] = 0.0f;
  float total = 0.0f;
  const int64_t KV = (int64_t)a.K * a.V;
  for (;;) {
#pragma unroll
    for (int s = 0; s < NST; ++s) {
      const Chunk c = ring[s];
      if (c.len < 0) return;
      copy_wait<NST - 1>();
      __syncwarp();
      if (c.first) {
        const float* st = nullptr;
        if (c.from < 0) st = a.state_in ? a.state_in + (c.seq * a.H + h) * KV : nullptr;
        else if (!STATE_ONLY) st = a.ws_state + (c.from * a.H + h) * KV;
        st = st && lane < width ? st + c0 + lane : nullptr;
#pragma unroll
        for (int i = 0; i < DK; ++i) S[i] = st && i < a.K ? st[(int64_t)i * a.V] : 0.0f;
      }
      const Slot& w = slots[s];
      for (int r = 0; r < c.len; ++r) {
        const float e = expf(w.g[r]);
        const float vr = to_float(w.v[r][lane]);
        if (STATE_ONLY) total += w.g[r];
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < DK; i += 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            S[i + j] = fmaf(to_float(w.k[r][i + j]), vr, e * S[i + j]);
            if (!STATE_ONLY) acc[j] = fmaf(to_float(w.q[r][i + j]), S[i + j], acc[j]);
          }
        }
        if (!STATE_ONLY && lane < width)
          put((T*)a.out + (c.row + dir * r) * a.os + h * a.V + c0 + lane, a.scale * ((acc[0] + acc[1]) + (acc[2] + acc[3])));
      }
      if (c.last && (STATE_ONLY || (c.ends && a.state_out))) {
        float* st = STATE_ONLY ? a.ws_state + (bound * a.H + h) * KV : a.state_out + (c.seq * a.H + h) * KV;
        if (lane < width)
#pragma unroll
          for (int i = 0; i < DK; ++i)
            if (i < a.K) st[(int64_t)i * a.V + c0 + lane] = S[i];
        if (STATE_ONLY && sl == 0 && lane == 0) a.ws_decay[bound * a.H + h] = total;
      }
      __syncwarp();
      issue(s);
    }
  }
}

// What crosses each boundary: the pieces' own states, in the direction of the recurrence,
// each with the decayed state of the boundary before it.  A thread takes one value of a
// head's state through all boundaries.
__global__ void __launch_bounds__(128) la_carry_kernel(const __grid_constant__ LaArgs a) {
  const int64_t KV = (int64_t)a.K * a.V;
  const int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (e >= KV * a.H) return;
  const int h = (int)(e / KV);
  float carry = 0.0f;
  for (int64_t j = 1; j < a.bounds; ++j) {
    const int64_t i = a.u.reverse ? a.bounds - j : j;
    const int f = a.ws_flag[i];
    if (f == 0) continue;
    float* p = a.ws_state + i * a.H * KV + e;
    carry = f == 2 ? fmaf(expf(a.ws_decay[i * a.H + h]), carry, *p) : *p;
    *p = carry;
  }
}

// ---------------------------------------------------------------- a single token
// A warp takes 32 columns of a head's state: 8 lanes hold four columns of a row each, and
// four rows are read, decayed, added to and written at a time.  The state's two crossings
// of memory are nearly all of the traffic, and bound it.
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
  const int c = sl * COLS + (lane & 7) * 4, r0 = lane >> 3;
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
// Rows a boundary: as many as leave about 1,500 units, the warps that the GPU holds, but not
// under 256 (a state is written and read twice a boundary) nor over 2,048.
int rows_a_boundary(int64_t n_rows, int H, int V) {
  const int64_t per_row = (int64_t)H * ((V + COLS - 1) / COLS);
  int l = 256;
  while (l < 2048 && n_rows / l * per_row > 3000) l *= 2;
  return l;
}
constexpr int64_t LONGEST = 512;   // longer sequences are cut

size_t workspace_bytes(int64_t n_rows, int H, int K, int V) {
  if (n_rows <= LONGEST) return 0;
  const int l = rows_a_boundary(n_rows, H, V);
  const size_t bounds = (size_t)((n_rows + l - 1) / l);
  const size_t flags = (bounds * 4 + 15) / 16 * 16, decay = (bounds * H * 4 + 15) / 16 * 16;
  return flags + decay + bounds * H * (size_t)K * V * 4;
}

template <class T, int DK, bool STATE_ONLY>
int launch_simt(const LaArgs& a, cudaStream_t st) {
  const size_t sm = sizeof(SimtSlot<T, DK>) * NST * NW;
  auto kern = la_simt_kernel<T, DK, STATE_ONLY>;
  const cudaError_t e = tf_allow_smem(kern);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  const int64_t units = (STATE_ONLY ? a.bounds - 1 : a.u.tiles) * a.H * a.slices;
  if ((units + NW - 1) / NW > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  kern<<<(unsigned)((units + NW - 1) / NW), NW * 32, sm, st>>>(a);
  return launched();
}
template <class T, bool STATE_ONLY>
int by_width(const LaArgs& a, cudaStream_t st) {
  if (a.K <= 16) return launch_simt<T, 16, STATE_ONLY>(a, st);
  if (a.K <= 32) return launch_simt<T, 32, STATE_ONLY>(a, st);
  if (a.K <= 64) return launch_simt<T, 64, STATE_ONLY>(a, st);
  return launch_simt<T, 128, STATE_ONLY>(a, st);
}
template <bool STATE_ONLY>
int by_type(int32_t dtype, const LaArgs& a, cudaStream_t st) {
  if (dtype == TRACKFIT_FP32) return by_width<float, STATE_ONLY>(a, st);
  return linear_mma(dtype, a, STATE_ONLY, st);
}

}  // namespace

extern "C" size_t trackfit_linear_attention_workspace(int64_t n_rows, int32_t n_heads, int32_t key_dim,
                                                      int32_t value_dim) {
  if (n_rows < 0 || n_rows > (int64_t)1 << 40 || !heads_ok(n_heads) || !dim_ok(key_dim) || !dim_ok(value_dim)) return 0;
  return workspace_bytes(n_rows, n_heads, key_dim, value_dim);
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
    if (!log_decay || mis4(log_decay) || decay_stride < n_heads || decay_stride > (int64_t)1 << 40)
      return TRACKFIT_ERR_INVALID_ARG;
  }
  const size_t need = workspace_bytes(n_rows, n_heads, key_dim, value_dim);
  if (need > 0 && (!workspace || mis16(workspace) || workspace_size < need)) return TRACKFIT_ERR_INVALID_ARG;
  LaArgs a;
  a.q = q, a.k = k, a.v = v, a.g = log_decay, a.out = out;
  a.qs = q_stride, a.ks = k_stride, a.vs = v_stride, a.gs = decay_stride, a.os = out_stride;
  a.state_in = state_in, a.state_out = state_out;
  const int cols = dtype == TRACKFIT_FP32 ? COLS : linear_mma_cols(key_dim, value_dim);
  a.H = n_heads, a.K = key_dim, a.V = value_dim, a.slices = (value_dim + cols - 1) / cols;
  a.scale = scale;
  a.u.offs = offsets, a.u.n_seq = n_seq, a.u.n_rows = n_rows, a.u.reverse = reverse;
  a.u.lseg = rows_a_boundary(n_rows, n_heads, value_dim);
  a.u.longest = LONGEST;
  // few rows: small tiles, so that there are units for every SM
  a.u.seg = 256;
  while (a.u.seg > 16 && n_rows / a.u.seg * n_heads * a.slices < 2400) a.u.seg /= 2;
  a.u.tiles = n_rows > 0 ? (n_rows + a.u.seg - 1) / a.u.seg : 1;
  a.bounds = 1;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (need > 0) {
    a.bounds = (n_rows + a.u.lseg - 1) / a.u.lseg;
    unsigned char* w = static_cast<unsigned char*>(workspace);
    a.ws_flag = reinterpret_cast<int32_t*>(w);
    w += (a.bounds * 4 + 15) / 16 * 16;
    a.ws_decay = reinterpret_cast<float*>(w);
    w += (a.bounds * n_heads * 4 + 15) / 16 * 16;
    a.ws_state = reinterpret_cast<float*>(w);
    if (a.bounds > 1) {
      int rc = by_type<true>(dtype, a, st);
      if (rc != TRACKFIT_OK) return rc;
      const int64_t n = (int64_t)n_heads * key_dim * value_dim;
      la_carry_kernel<<<(unsigned)((n + 127) / 128), 128, 0, st>>>(a);
      rc = launched();
      if (rc != TRACKFIT_OK) return rc;
    }
  } else {
    a.ws_flag = nullptr, a.ws_decay = a.ws_state = nullptr;
  }
  return by_type<false>(dtype, a, st);
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
  if (!log_decay || mis4(log_decay) || decay_stride < n_heads || decay_stride > (int64_t)1 << 40)
    return TRACKFIT_ERR_INVALID_ARG;
  if (mis4(slots) || !state_in || !state_out || mis16(state_in) || mis16(state_out)) return TRACKFIT_ERR_INVALID_ARG;
  StepArgs a;
  a.q = q, a.k = k, a.v = v, a.g = log_decay, a.out = out;
  a.qs = q_stride, a.ks = k_stride, a.vs = v_stride, a.gs = decay_stride, a.os = out_stride;
  a.slots = slots, a.state_in = state_in, a.state_out = state_out, a.n = n_seq, a.n_slots = n_slots;
  a.H = n_heads, a.K = key_dim, a.V = value_dim, a.slices = (value_dim + COLS - 1) / COLS, a.scale = scale;
  const int64_t units = n_seq * n_heads * a.slices;
  if ((units + NW - 1) / NW > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((units + NW - 1) / NW);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (dtype == TRACKFIT_FP32) la_step_kernel<float><<<grid, NW * 32, 0, st>>>(a);
  else if (dtype == TRACKFIT_BF16_PROJ) la_step_kernel<__nv_bfloat16><<<grid, NW * 32, 0, st>>>(a);
  else la_step_kernel<__half><<<grid, NW * 32, 0, st>>>(a);
  return launched();
}
