// Linear attention of the 16-bit types on the tensor cores.
//
// A warp takes a unit (linear_units.cuh) of one head and 16 or 32 channels of v, with the
// state's columns of these channels in registers, and goes through its sequences in chunks of
// up to 16 rows.  With G_i the sum of g over a chunk's rows up to i and S the state before it:
//   O   = diag(exp G) Q S + (Q K^T o L) V,    L_ij = exp(G_i - G_j) for j <= i, else 0
//   S'  = exp(G_end) S + K^T diag(exp(G_end - G)) V
// as m16n8k16 products.  The state stands transposed (value channels x key channels): its
// accumulators are then the B operand of Q S as they are, and V's fragments both the B operand
// of the second product and, scaled, the A operand of S'.
//
// Why 16 rows: a chunk of C rows costs C (K + V) products a row for the part within it and
// 2 K V for the state whatever C, and tracks have 8 to 20 rows.  Why mma.sync and not
// tcgen05: the products are 16 rows high (a track), the traffic of a row and head is
// 4 (K + V) bytes and its products at K = V = 64 take 17 of the 22 clocks that an SM's share
// of the memory bandwidth gives it.
//
// Every warp runs by itself, with a ring of chunks in shared memory that it fills by
// asynchronous copies; rows beyond a chunk's are zeros, so that nothing of another sequence
// enters a product.
//
// Roundings: the products' operands are 16 bits.  Q K^T o L is split into two bf16 parts, the
// decayed V into two, or three where the state is asked for (bf16: 8, 16, 24 bits), so that
// the states keep fp32; the state's operand of Q S is rounded once, which the output's own
// rounding exceeds.  fp16 has the bits but not the range for Q K^T and S: these go through
// tf32 products (11 bits, fp32's range), the decayed V, no larger than V, is split in two.
#include "linear_units.cuh"
#include "mma_sync.cuh"

namespace {
using namespace seqops;

constexpr int NST = 3;           // chunks in the ring
constexpr int C = 16;            // rows of a chunk

template <int DK, int NV>
struct __align__(16) Slot {
  static constexpr int PK = DK * 2 + 16, PV = NV * 16 + 16;   // bytes of a row: 16 more, for the banks
  unsigned char q[C * PK], k[C * PK], v[C * PV];
  float g[C];
  int64_t row;                   // the chunk: its first row in the direction of the recurrence
  int32_t seq, flags;
};
enum { LEN = 0xff, FIRST = 0x100, LAST = 0x200, GOES_ON = 0x400, ENDS = 0x800, NONE = 0x1000 };

__device__ __forceinline__ uint32_t zero_if_finite(uint32_t u, uint32_t sum, __nv_bfloat16) {
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u), "r"(0u));
  return sum;
}
__device__ __forceinline__ uint32_t zero_if_finite(uint32_t u, uint32_t sum, __half) {
  asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u), "r"(0u));
  return sum;
}

// o += the product of the chunk's weights with V, by mul(d, b0, b1) for 8 channels.  A
// weight of zero does not keep an infinity or a NaN of a later row out of an earlier one's
// sum: where V has any, each row by itself takes the rows up to its own.
template <class T, int NV, class Mul>
__device__ __forceinline__ void add_rows(T, Mul mul, float (&o)[NV][4], const uint32_t (&vb)[NV][2], int len, int g, int t) {
  uint32_t sum = 0u;
#pragma unroll
  for (int n = 0; n < NV; ++n) sum = zero_if_finite(vb[n][0], zero_if_finite(vb[n][1], sum, T()), T());
  if (!__any_sync(FULL, (sum & 0x7fff7fffu) != 0u)) {
#pragma unroll
    for (int n = 0; n < NV; ++n) mul(o[n], vb[n][0], vb[n][1]);
    return;
  }
  for (int r = 0; r < len; ++r) {
    const uint32_t m0 = (2 * t <= r ? 0xffffu : 0u) | (2 * t + 1 <= r ? 0xffff0000u : 0u);
    const uint32_t m1 = (2 * t + 8 <= r ? 0xffffu : 0u) | (2 * t + 9 <= r ? 0xffff0000u : 0u);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      mul(d, vb[n][0] & m0, vb[n][1] & m1);
      if (g == r) o[n][0] += d[0], o[n][1] += d[1];
      if (g + 8 == r) o[n][2] += d[2], o[n][3] += d[3];
    }
  }
}

template <class T, int DK, int NV, bool STATE_ONLY, bool EXACT>
__global__ void __launch_bounds__(NW * 32) la_mma_kernel(const __grid_constant__ LaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  using S = Slot<DK, NV>;
  constexpr bool BF = sizeof(T) == 2 && !__is_same(T, __half);
  constexpr int MT = NV / 2, KT = DK / 8;             // tiles of the state: MT x 16 by KT x 8
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = (int64_t)blockIdx.x * NW + warp;
  const int sl = (int)(unit % a.slices), h = (int)(unit / a.slices % a.H);
  const int64_t tile = unit / a.slices / a.H;
  if (tile >= (STATE_ONLY ? a.bounds - 1 : a.u.tiles)) return;
  S* slots = reinterpret_cast<S*>(smem) + warp * NST;
  const int c0 = sl * NV * 8, width = a.V - c0 < NV * 8 ? a.V - c0 : NV * 8;
  const int dir = a.u.reverse ? -1 : 1;
  const int g = lane >> 2, t = lane & 3;
  // channels beyond K and V are zeros from here on: the copies leave them alone
  if (a.K < DK || width < NV * 8) {
    for (uint32_t* p = reinterpret_cast<uint32_t*>(slots) + lane; p < reinterpret_cast<uint32_t*>(slots + NST); p += 32) *p = 0;
    __syncwarp();
  }
  const T* q = (const T*)a.q + h * a.K;
  const T* k = (const T*)a.k + h * a.K;
  const T* v = (const T*)a.v + h * a.V + c0;
  TilePieces pieces(a.u, tile, lane, STATE_ONLY);
  Piece p;
  bool more;
  if (STATE_ONLY) {
    more = boundary_piece(a.u, tile + 1, lane, p);
    if (sl == 0 && h == 0 && lane == 0) a.ws_flag[tile + 1] = !more ? 0 : p.from < 0 ? 1 : 2;
  } else {
    more = pieces.next(p);
  }
  int64_t done = 0;

  auto issue = [&](S& w) {
    if (more) {
      const int64_t left = p.hi - p.lo - done;
      const int len = (int)(left < C ? left : C);
      const int64_t row = a.u.reverse ? p.hi - 1 - done : p.lo + done;
      if (lane == 0) {
        w.row = row, w.seq = (int32_t)p.seq;
        w.flags = len | (done == 0 ? FIRST : 0) | (left <= C ? LAST : 0) | (p.from >= 0 ? GOES_ON : 0) | (p.ends ? ENDS : 0);
      }
      constexpr int VK = DK / 8;                       // 16-byte pieces of a row
#pragma unroll
      for (int i = 0; i < C * VK / 32; ++i) {
        const int r = (lane + 32 * i) / VK, e = (lane + 32 * i) % VK * 8;
        if (e < a.K) {
          const bool on = r < len;
          const int64_t at = on ? row + dir * r : 0;
          if (!STATE_ONLY) copy16(smem_addr(w.q + r * S::PK + e * 2), q + at * a.qs + e, on);
          copy16(smem_addr(w.k + r * S::PK + e * 2), k + at * a.ks + e, on);
        }
      }
#pragma unroll
      for (int i = 0; i < C * NV / 32; ++i) {
        const int r = (lane + 32 * i) / NV, e = (lane + 32 * i) % NV * 8;
        if (e < width) {
          const bool on = r < len;
          copy16(smem_addr(w.v + r * S::PV + e * 2), v + (on ? row + dir * r : 0) * a.vs + e, on);
        }
      }
      if (lane < C) copy4(smem_addr(&w.g[lane]), a.g + (lane < len ? row + dir * lane : 0) * a.gs + h, lane < len);
      done += len;
      if (left <= C) {
        done = 0;
        more = STATE_ONLY ? false : pieces.next(p);
      }
    } else if (lane == 0) {
      w.flags = NONE;
    }
    copy_commit();
  };

  for (int s = 0; s < NST; ++s) issue(slots[s]);
  float st[MT][KT][4];
  bool zero = true;                                    // the state before the chunk is zero
  float total = 0.0f;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) st[m][j][i] = 0.0f;
  const int64_t KV = (int64_t)a.K * a.V;
  // of this lane in operands of 8 x 8 matrices: rows by lane, columns by the matrix
  const int q_row = lane & 15, q_col = (lane >> 4) * 8;
  const int n_row = (lane >> 4) * 8 + (lane & 7), n_col = (lane >> 3 & 1) * 8;
  const int k_row = (lane >> 3 & 1) * 8 + (lane & 7), k_col = (lane >> 4) * 8;
  int s = 0;
  for (;;) {
    S& w = slots[s];
    copy_wait<NST - 1>();
    __syncwarp();
    const int flags = w.flags;
    if (flags & NONE) break;
    const int64_t row = w.row;
    const int64_t seq = w.seq;
    const int len = flags & LEN;

    if (flags & FIRST) {
      const float* src = nullptr;
      if (flags & GOES_ON)
        src = STATE_ONLY ? nullptr : a.ws_state + ((a.u.reverse ? row + 1 : row) / a.u.lseg * a.H + h) * KV;
      else if (a.state_in)
        src = a.state_in + (seq * a.H + h) * KV;
      zero = src == nullptr;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int kk = j * 8 + 2 * t + (i & 1), c = m * 16 + g + (i >> 1) * 8;
            st[m][j][i] = src && kk < a.K && c < width ? src[(int64_t)kk * a.V + c0 + c] : 0.0f;
          }
    }

    // sums of the logarithms (base 2): P up to a row, R behind it.  Below 2^-150 a decay is 0
    // in fp32; held there, so that the differences of sums stay finite and fine
    float x = w.g[lane & 15] * LOG2E;
    x = x < -150.0f ? -150.0f : x;
    if (STATE_ONLY) total += x;                        // summed over lanes at the end
    float P = x, R = __shfl_down_sync(FULL, x, 1, 16);
    if ((lane & 15) == 15) R = 0.0f;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const float y = __shfl_up_sync(FULL, P, o, 16), z = __shfl_down_sync(FULL, R, o, 16);
      if ((lane & 15) >= o) P += y;
      if ((lane & 15) + o < 16) R += z;
    }
    const bool update = STATE_ONLY || !(flags & LAST) || ((flags & ENDS) && a.state_out);

    uint32_t vb[NV][2];                                // V as 16 x 8 tiles, two rows a word
#pragma unroll
    for (int n = 0; n < NV; n += 2) {
      uint32_t r[4];
      ldsm4t(r, smem_addr(w.v + k_row * S::PV + (n * 8 + k_col) * 2));
      vb[n][0] = r[0], vb[n][1] = r[1], vb[n + 1][0] = r[2], vb[n + 1][1] = r[3];
    }

    if (!STATE_ONLY) {
      float o[NV][4];
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
      float s0[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s1[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kk = 0; kk < DK / 16; ++kk) {
        uint32_t qa[4], kb[4];
        ldsm4(qa, smem_addr(w.q + q_row * S::PK + (kk * 16 + q_col) * 2));
        ldsm4(kb, smem_addr(w.k + n_row * S::PK + (kk * 16 + n_col) * 2));
        mma16(s0, qa, kb[0], kb[1], T());
        mma16(s1, qa, kb[2], kb[3], T());
        if (!zero) {
          if (BF) {
#pragma unroll
            for (int n = 0; n < NV; ++n) {
              const float(&u0)[4] = st[n / 2][2 * kk], (&u1)[4] = st[n / 2][2 * kk + 1];
              const int i = (n & 1) * 2;
              mma16(o[n], qa, pack2(u0[i], u0[i + 1], T()), pack2(u1[i], u1[i + 1], T()), T());
            }
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {              // 8 channels of the key a time
              const float2 x0 = halves(qa[2 * e], T()), x1 = halves(qa[2 * e + 1], T());
#pragma unroll
              for (int n = 0; n < NV; ++n) {
                const float(&u)[4] = st[n / 2][2 * kk + e];
                const int i = (n & 1) * 2;
                mma8(o[n], __float_as_uint(x0.x), __float_as_uint(x1.x), __float_as_uint(x0.y), __float_as_uint(x1.y),
                     tf32(u[i]), tf32(u[i + 1]));
              }
            }
          }
        }
      }
      const float pg = __shfl_sync(FULL, P, g), pg8 = __shfl_sync(FULL, P, g + 8);
      if (!zero) {
        const float e0 = ex2(pg), e1 = ex2(pg8);
#pragma unroll
        for (int n = 0; n < NV; ++n) o[n][0] *= e0, o[n][1] *= e0, o[n][2] *= e1, o[n][3] *= e1;
      }
      // the decays between rows, and none to a later row
      const float p0 = __shfl_sync(FULL, P, 2 * t), p1 = __shfl_sync(FULL, P, 2 * t + 1);
      const float p8 = __shfl_sync(FULL, P, 2 * t + 8), p9 = __shfl_sync(FULL, P, 2 * t + 9);
      s0[0] = 2 * t <= g ? s0[0] * ex2(pg - p0) : 0.0f;
      s0[1] = 2 * t + 1 <= g ? s0[1] * ex2(pg - p1) : 0.0f;
      s0[2] *= ex2(pg8 - p0);
      s0[3] *= ex2(pg8 - p1);
      s1[2] = 2 * t <= g ? s1[2] * ex2(pg8 - p8) : 0.0f;
      s1[3] = 2 * t + 1 <= g ? s1[3] * ex2(pg8 - p9) : 0.0f;
      if (BF) {
        uint32_t hi[4] = {pack2(s0[0], s0[1], T()), pack2(s0[2], s0[3], T()), 0u, pack2(s1[2], s1[3], T())};
        uint32_t lo[4];
        const float2 h0 = halves(hi[0], T()), h1 = halves(hi[1], T()), h3 = halves(hi[3], T());
        lo[0] = pack2(s0[0] - h0.x, s0[1] - h0.y, T()), lo[1] = pack2(s0[2] - h1.x, s0[3] - h1.y, T());
        lo[2] = 0u, lo[3] = pack2(s1[2] - h3.x, s1[3] - h3.y, T());
        add_rows(
            T(),
            [&](float(&d)[4], uint32_t b0, uint32_t b1) {
              mma16(d, hi, b0, b1, T());
              mma16(d, lo, b0, b1, T());
            },
            o, vb, len, g, t);
      } else {
        const uint32_t f0 = tf32(s0[0]), f1 = tf32(s0[1]), f2 = tf32(s0[2]), f3 = tf32(s0[3]);
        const uint32_t f6 = tf32(s1[2]), f7 = tf32(s1[3]);
        add_rows(
            T(),
            [&](float(&d)[4], uint32_t b0, uint32_t b1) {
              const float2 v0 = halves(b0, T()), v1 = halves(b1, T());
              mma8(d, f0, f2, f1, f3, __float_as_uint(v0.x), __float_as_uint(v0.y));
              mma8(d, 0u, f6, 0u, f7, __float_as_uint(v1.x), __float_as_uint(v1.y));
            },
            o, vb, len, g, t);
      }
      // out through V's place in the slot: 16 bytes a lane
      __syncwarp();
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        *reinterpret_cast<uint32_t*>(w.v + g * S::PV + (n * 8 + 2 * t) * 2) = pack2(a.scale * o[n][0], a.scale * o[n][1], T());
        *reinterpret_cast<uint32_t*>(w.v + (g + 8) * S::PV + (n * 8 + 2 * t) * 2) = pack2(a.scale * o[n][2], a.scale * o[n][3], T());
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < C * NV / 32; ++i) {
        const int r = (lane + 32 * i) / NV, e = (lane + 32 * i) % NV * 8;
        if (r < len && e < width)
          *reinterpret_cast<uint4*>((T*)a.out + (row + dir * r) * a.os + h * a.V + c0 + e) =
              *reinterpret_cast<const uint4*>(w.v + r * S::PV + e * 2);
      }
    }

    if (update) {
      const float f = ex2(__shfl_sync(FULL, P, 15));
      if (!zero) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) st[m][j][i] *= f;
      }
      zero = false;
      R = ex2(R);
      const float w0 = __shfl_sync(FULL, R, 2 * t), w1 = __shfl_sync(FULL, R, 2 * t + 1);
      const float w8 = __shfl_sync(FULL, R, 2 * t + 8), w9 = __shfl_sync(FULL, R, 2 * t + 9);
      constexpr int TERMS = BF && EXACT ? 3 : 2;
      uint32_t va[TERMS][MT][4];
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float2 y = halves(vb[n][i], T());
          y.x *= i ? w8 : w0, y.y *= i ? w9 : w1;
#pragma unroll
          for (int e = 0; e < TERMS; ++e) {
            const uint32_t u = pack2(y.x, y.y, T());
            va[e][n / 2][2 * i + (n & 1)] = u;
            if (e + 1 < TERMS) {
              const float2 z = halves(u, T());
              y.x -= z.x, y.y -= z.y;
            }
          }
        }
#pragma unroll
      for (int kk = 0; kk < DK / 16; ++kk) {
        uint32_t kb[4];
        ldsm4t(kb, smem_addr(w.k + k_row * S::PK + (kk * 16 + k_col) * 2));
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int e = 0; e < TERMS; ++e) {
            mma16(st[m][2 * kk], va[e][m], kb[0], kb[1], T());
            mma16(st[m][2 * kk + 1], va[e][m], kb[2], kb[3], T());
          }
      }
      if ((flags & LAST) && (STATE_ONLY || (flags & ENDS))) {
        float* dst = STATE_ONLY ? a.ws_state + ((tile + 1) * a.H + h) * KV : a.state_out + (seq * a.H + h) * KV;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int kk = j * 8 + 2 * t + (i & 1), c = m * 16 + g + (i >> 1) * 8;
              if (kk < a.K && c < width) dst[(int64_t)kk * a.V + c0 + c] = st[m][j][i];
            }
        if (STATE_ONLY) {
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) total += __shfl_xor_sync(FULL, total, o, 16);
          if (sl == 0 && lane == 0) a.ws_decay[(tile + 1) * a.H + h] = total / LOG2E;
        }
      }
    }
    __syncwarp();
    issue(w);
    s = s + 1 == NST ? 0 : s + 1;
  }
}

template <class T, int DK, int NV, bool STATE_ONLY, bool EXACT>
int launch(const LaArgs& a, cudaStream_t st) {
  auto kern = la_mma_kernel<T, DK, NV, STATE_ONLY, EXACT>;
  const cudaError_t e = tf_allow_smem(kern);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  const int64_t units = (STATE_ONLY ? a.bounds - 1 : a.u.tiles) * a.H * a.slices;
  if ((units + NW - 1) / NW > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  kern<<<(unsigned)((units + NW - 1) / NW), NW * 32, sizeof(Slot<DK, NV>) * NST * NW, st>>>(a);
  return launched();
}
template <class T, int DK, int NV>
int by_use(const LaArgs& a, bool state_only, cudaStream_t st) {
  // fp16 splits into two parts either way
  if constexpr (!__is_same(T, __half)) {
    if (a.state_out && state_only) return launch<T, DK, NV, true, true>(a, st);
    if (a.state_out) return launch<T, DK, NV, false, true>(a, st);
  }
  return state_only ? launch<T, DK, NV, true, false>(a, st) : launch<T, DK, NV, false, false>(a, st);
}
template <class T>
int by_width(const LaArgs& a, bool state_only, cudaStream_t st) {
  const bool wide = linear_mma_cols(a.K, a.V) == 32;
  if (a.K <= 16) return wide ? by_use<T, 16, 4>(a, state_only, st) : by_use<T, 16, 2>(a, state_only, st);
  if (a.K <= 32) return wide ? by_use<T, 32, 4>(a, state_only, st) : by_use<T, 32, 2>(a, state_only, st);
  if (a.K <= 64) return wide ? by_use<T, 64, 4>(a, state_only, st) : by_use<T, 64, 2>(a, state_only, st);
  return by_use<T, 128, 2>(a, state_only, st);
}

}  // namespace

int seqops::linear_mma(int32_t dtype, const LaArgs& a, bool state_only, cudaStream_t st) {
  if (dtype == TRACKFIT_BF16_PROJ) return by_width<__nv_bfloat16>(a, state_only, st);
  return by_width<__half>(a, state_only, st);
}
