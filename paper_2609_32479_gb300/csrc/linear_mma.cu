// Linear attention of the 16-bit types on the tensor cores.
//
// A warp takes a unit (linear_units.cuh) of one head and 32 or 16 channels of v, with the
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
// Operands without a layout in shared memory: lane (g, t) = (l / 4, l % 4) reads 16 bytes,
// channels 8t .. 8t+7 of each 32, of rows g and g + 8.  A product's k index may be permuted,
// so these are the operands of Q K^T as they stand (slots 2t, 2t+1 of step i are channels
// 8t + 4i, + 1, slots 2t+8, 2t+9 the two after); movmatrix turns the words of V (and of K,
// for the state) to pairs of rows, and the products' columns come out with channels
// 8t .. 8t+7 in lane t again: 16 bytes to write.  Shared memory is a queue of each lane's own
// words, filled by asynchronous copies three chunks ahead.  Instructions bound the short
// chunks: staged through rows in shared memory with ldmatrix and 64-bit row addresses,
// 131,072 tracks took 700 us.
//
// Rows beyond a chunk's are zeros, so that nothing of another sequence enters a product.
//
// Roundings: the products' operands are 16 bits, and what is not a row as it came is split.
// bf16: Q K^T o L, the state as the operand of Q S, and the decayed V into two parts (16 bits), V
// into three where the state is asked for (24 bits; its chunks' sums are then added outside the
// products too).  fp16 has the bits but not the range for any of them (a lower part of V would fall
// below its smallest step, as V itself may lie next to that): all go through tf32 products (fp32's
// range) in two parts of 11 bits.  Outputs are off by their own rounding and by 2^-16 (bf16) or
// 2^-22 of what is added up; states asked for keep fp32.  With one part each for S and the fp16
// weights it was 2^-8 and 2^-11 of it, for 7 % (tracks, bf16) to 20 % (fp16) less time.
//
// Measured: 131,072 tracks, 4 heads of 32, bf16: 425 us a call, 4.5 TB/s of the 6.8 that a copy
// moves (412 the kernel; the rest two launches that find no sequence to cut); issued instructions
// bound it (71 % of the slots with 16 warps an SM, the rest waits for their results).  Four sequences
// of 20,000-40,000 rows, 8 heads of 64, states in and out: 363 us a call, 119 for the parts' own
// states, 15 for what they pass on, 232 for the outputs, against 84 for one reading of everything;
// latency with 8 warps an SM bounds it.
#include "linear_units.cuh"
#include "mma_sync.cuh"

namespace {
using namespace seqops;

constexpr int NST = 3;           // chunks in the queue
constexpr int C = 16;            // rows of a chunk

struct Chunk {
  int row, seq, flags;           // its first row in the direction of the recurrence, from the unit's base
};
enum { LEN = 0x1f, FIRST = 0x100, LAST = 0x200, GOES_ON = 0x400, ENDS = 0x800, NONE = 0x1000 };

// Bytes of a chunk's place in the queue: q and k, 4 x 16 bytes a lane and group of 32 channels,
// V, 2 x NV words a lane, and g, a word a lane.
__host__ __device__ constexpr int slot_bytes(int groups, int nv) { return 32 * (groups * 4 * 16 + 2 * nv * 4 + 4); }

// Words of a lane's 16 (NV = 4) or 8 (NV = 2) bytes of V.
template <int NV>
struct Vec {
  uint32_t w[NV];
};
template <int BYTES>
__device__ __forceinline__ void copy_v(uint32_t dst, const void* src, bool there) {
  if constexpr (BYTES == 16) copy16(dst, src, there);
  else copy8(dst, src, there);
}

// o += the product of the chunk's weights with V (zero: o is not set yet), by
// mul(d, b0, b1, anew) for 8 channels.  A weight of zero does not keep an infinity or a NaN of a
// later row out of an earlier one's sum: where V has any, each row by itself takes the rows up
// to its own.
template <class T, int NV, class Mul>
__device__ __forceinline__ void add_rows(T, Mul mul, bool zero, float (&o)[NV][4], const uint32_t (&vb)[NV][2], int len, int g,
                                         int t) {
  uint32_t sum = 0u;
#pragma unroll
  for (int n = 0; n < NV; ++n) sum = zero_if_finite(vb[n][0], zero_if_finite(vb[n][1], sum, T()), T());
  if (!__any_sync(FULL, (sum & 0x7fff7fffu) != 0u)) {
    if (zero) {
#pragma unroll
      for (int n = 0; n < NV; ++n) mul(o[n], vb[n][0], vb[n][1], true);
    } else {
#pragma unroll
      for (int n = 0; n < NV; ++n) mul(o[n], vb[n][0], vb[n][1], false);
    }
    return;
  }
  if (zero) {
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
  }
  for (int r = 0; r < len; ++r) {
    const uint32_t m0 = (2 * t <= r ? 0xffffu : 0u) | (2 * t + 1 <= r ? 0xffff0000u : 0u);
    const uint32_t m1 = (2 * t + 8 <= r ? 0xffffu : 0u) | (2 * t + 9 <= r ? 0xffff0000u : 0u);
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      float d[4];
      mul(d, vb[n][0] & m0, vb[n][1] & m1, true);
      if (g == r) o[n][0] += d[0], o[n][1] += d[1];
      if (g + 8 == r) o[n][2] += d[2], o[n][3] += d[3];
    }
  }
}

template <class T, int NG, int NV, bool STATE_ONLY, bool EXACT>
__global__ void __launch_bounds__(32, NG > 1 ? 8 : EXACT || __is_same(T, __half) ? 12 : 16) la_mma_kernel(const __grid_constant__ LaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr bool BF = !__is_same(T, __half);
  constexpr int MT = NV / 2, KT = NG * 4;             // tiles of the state: MT x 16 by KT x 8
  // With 128 registers a thread (16 warps an SM) q and k are read where they are used; with 255
  // (8 warps) early, and their place filled again: 221 instead of 305 us at K = 64, when both were tried
  constexpr bool EARLY = NG == 2;
  // A chunk's own sum first, added to the state outside the products: their accumulation cuts bits
  // off, and on the state itself that would shrink it a little with every chunk (2^-24: nothing that
  // bf16 outputs show)
  constexpr bool APART = EXACT || !BF;
  constexpr int VC = NV * 2;                           // channels of V a lane
  constexpr int SLOT = slot_bytes(NG, NV);
  const int lane = threadIdx.x;
  const unsigned unit = blockIdx.x;
  const int sl = (int)(unit % a.slices), h = (int)(unit / a.slices % a.H);
  const int64_t tile = unit / a.slices / a.H;
  const int c0 = sl * NV * 8, width = a.V - c0 < NV * 8 ? a.V - c0 : NV * 8;
  const int dir = a.u.reverse ? -1 : 1;
  const int g = lane >> 2, t = lane & 3;
  const int64_t base = STATE_ONLY ? (tile + 1) * a.u.lseg : tile * a.u.seg;
  // this lane's place in the queue: 16 bytes of each of q [group][row half], k likewise, its V
  // [row half], g
  const uint32_t mine = smem_addr(smem) + lane * 16;
  const uint32_t mine_v = smem_addr(smem) + NG * 4 * 512 + lane * VC * 2;
  const uint32_t mine_g = smem_addr(smem) + NG * 4 * 512 + 2 * 32 * VC * 2 + lane * 4;
  // channels beyond K and V are zeros from here on: the copies leave them alone
  for (int s = 0; s < NST; ++s) {
#pragma unroll
    for (int i = 0; i < NG * 4; ++i)
      asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(mine + s * SLOT + i * 512), "r"(0) : "memory");
#pragma unroll
    for (int i = 0; i < VC; ++i)
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(mine_v + s * SLOT + i / NV * 32 * VC * 2 + i % NV * 4), "r"(0) : "memory");
  }
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
  // bytes from a row to the next in the direction of the recurrence, and this lane's bytes of
  // the base row: a row's address is one 32 x 32 + 64 bit multiply-add
  const int qb = dir * (int)a.qs * 2, kb = dir * (int)a.ks * 2, vs = dir * (int)a.vs * 2, gs = dir * (int)a.gs * 4;
  const int ob = dir * (int)a.os * 2;
  const char* q0 = reinterpret_cast<const char*>((const T*)a.q + base * a.qs + h * a.K + 8 * t);
  const char* k0 = reinterpret_cast<const char*>((const T*)a.k + base * a.ks + h * a.K + 8 * t);
  const char* v0 = reinterpret_cast<const char*>((const T*)a.v + base * a.vs + h * a.V + c0 + VC * t);
  const char* g0 = reinterpret_cast<const char*>(a.g + base * a.gs + h);
  char* o0 = reinterpret_cast<char*>((T*)a.out + base * a.os + h * a.V + c0 + VC * t);
  const bool v_on = VC * t < width;
  const int block = STATE_ONLY ? 0 : block_of(a.u, tile);
  const int64_t KV = (int64_t)a.K * a.V;

  auto issue = [&](int s) {
    Chunk c;
    c.flags = NONE;
    if (more) {
      const int left = p.hi - p.lo - done;
      const int len = left < C ? left : C;
      c.row = a.u.reverse ? p.hi - 1 - done : p.lo + done;
      c.seq = p.seq;
      c.flags = len | (done == 0 ? FIRST : 0) | (left <= C ? LAST : 0) | (p.goes_on ? GOES_ON : 0) | (p.ends ? ENDS : 0);
      const int r0 = dir * c.row + g, r1 = r0 + 8;     // rows along the direction
      const bool on0 = g < len, on1 = g + 8 < len;
      const uint32_t m = mine + s * SLOT;
      const char* kk0 = k0 + (int64_t)r0 * kb;
      const char* kk1 = k0 + (int64_t)r1 * kb;
      const char* qq0 = q0 + (int64_t)r0 * qb;
      const char* qq1 = q0 + (int64_t)r1 * qb;
#pragma unroll
      for (int i = 0; i < NG; ++i)
        if (32 * i + 8 * t < a.K) {
          if (!STATE_ONLY) {
            copy16(m + (2 * i) * 512, qq0 + 64 * i, on0);
            copy16(m + (2 * i + 1) * 512, qq1 + 64 * i, on1);
          }
          copy16(m + (2 * NG + 2 * i) * 512, kk0 + 64 * i, on0);
          copy16(m + (2 * NG + 2 * i + 1) * 512, kk1 + 64 * i, on1);
        }
      if (v_on) {
        copy_v<VC * 2>(mine_v + s * SLOT, v0 + (int64_t)r0 * vs, on0);
        copy_v<VC * 2>(mine_v + s * SLOT + 32 * VC * 2, v0 + (int64_t)r1 * vs, on1);
      }
      if (EXACT && done == 0 && a.state_in && !p.goes_on) {   // the state that it begins with, on its way to L2
        const float* src = a.state_in + ((int64_t)c.seq * a.H + h) * KV + c0;
        for (int i = lane; i < a.K; i += 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + i * a.V));
      }
      const int lr = lane & 15;
      copy4(mine_g + s * SLOT, g0 + (int64_t)(dir * c.row + lr) * gs, lr < len);
      done += len;
      if (left <= C) {
        done = 0;
        more = STATE_ONLY ? false : pieces.next(p);
      }
    }
    copy_commit();
    return c;
  };

  float st[MT][KT][4];
  bool zero = true;                                    // the state before the chunk is zero, and st not set
  float total = 0.0f;
  // st[m][j][i] is key channel 32 (j/4) + 8t + 2 (j%4) + (i&1), value channel
  // VC (g/2) + 2 (2m + i/2) + (g&1) of the slice.  Lanes g and g^1 trade halves, so that each
  // has NV channels side by side
  const bool odd = g & 1;
  const int64_t mine_st = (int64_t)(8 * t) * a.V + c0 + VC * (g >> 1) + (odd ? NV : 0);
  const bool st_on = VC * (g >> 1) < width;
  auto load_state = [&](const float* src) {
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x[NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) x[n] = 0.0f;
        if (st_on && 32 * (j / 4) + 8 * t < a.K) {
          const float* s = src + mine_st + (32 * (j / 4) + 2 * (j % 4) + i) * a.V;
          if constexpr (NV == 4) *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(s);
          else *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(s);
        }
        // an even lane has the channels of the lower tiles, its own and its neighbour's by turns
#pragma unroll
        for (int n = 0; n < NV / 2; ++n) {
          const float y = __shfl_xor_sync(FULL, odd ? x[2 * n] : x[2 * n + 1], 4);
          const float own = odd ? x[2 * n + 1] : x[2 * n];
          const int lo = n, hi = n + NV / 2;           // tiles
          st[lo / 2][j][(lo & 1) * 2 + i] = odd ? y : own;
          st[hi / 2][j][(hi & 1) * 2 + i] = odd ? own : y;
        }
      }
  };
  auto store_state = [&](float* dst) {
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x[NV];
#pragma unroll
        for (int n = 0; n < NV / 2; ++n) {
          const int lo = n, hi = n + NV / 2;
          const float u = st[lo / 2][j][(lo & 1) * 2 + i], v = st[hi / 2][j][(hi & 1) * 2 + i];
          const float y = __shfl_xor_sync(FULL, odd ? u : v, 4);
          x[2 * n] = odd ? y : u;
          x[2 * n + 1] = odd ? v : y;
        }
        if (st_on && 32 * (j / 4) + 8 * t < a.K) {
          float* s = dst + mine_st + (32 * (j / 4) + 2 * (j % 4) + i) * a.V;
          if constexpr (NV == 4) *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(x);
          else *reinterpret_cast<float2*>(s) = *reinterpret_cast<const float2*>(x);
        }
      }
  };

  Chunk next[NST];
#pragma unroll
  for (int s = 0; s < NST; ++s) next[s] = issue(s);
  for (int s = 0;; s = s + 1 == NST ? 0 : s + 1) {
    const Chunk ch = next[0];
#pragma unroll
    for (int i = 0; i + 1 < NST; ++i) next[i] = next[i + 1];
    const int flags = ch.flags, row = ch.row, len = flags & LEN;
    if (flags & NONE) break;
    copy_wait<NST - 1>();
    const uint32_t slot = mine + s * SLOT;
    uint32_t q[NG][2][4], k[NG][2][4], vb[NV][2];
    if (EARLY) {
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (!STATE_ONLY) load_shared(q[i][e], slot + (2 * i + e) * 512);
          load_shared(k[i][e], slot + (2 * NG + 2 * i + e) * 512);
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {                      // V as 16 x 8 tiles, two rows a word
      Vec<NV> v;
      load_shared(v.w, mine_v + s * SLOT + e * 32 * VC * 2);
#pragma unroll
      for (int n = 0; n < NV; ++n) vb[n][e] = turned(v.w[n]);
    }
    // sums of the logarithms (base 2): P up to a row, later Z behind it.  Below 2^-150 a decay is
    // 0 in fp32; held there, so that the differences of sums stay finite and fine
    const int lr = lane & 15;
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(mine_g + s * SLOT) : "memory");
    if (EARLY) {
      __syncwarp();                                    // read: the place is free
      next[NST - 1] = issue(s);
    }
    x *= LOG2E;
    x = x < -150.0f ? -150.0f : x;
    if (flags & FIRST) {
      zero = true;
      if ((flags & GOES_ON) || a.state_in) {
        const float* src = STATE_ONLY ? boundary_begins_with(a, ch.seq, h, flags & GOES_ON)
                                      : piece_begins_with(a, block, ch.seq, h, flags & GOES_ON, flags & ENDS);
        zero = src == nullptr;
        if (!zero) load_state(src);
        if (STATE_ONLY && a.ws_begin && !(flags & GOES_ON)) store_state(a.ws_begin + ((tile + 1) * a.H + h) * KV);
      }
    }
    if (STATE_ONLY) total += x;                        // summed over lanes at the end
    float P = x;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const float y = __shfl_up_sync(FULL, P, o, 16);
      if (lr >= o) P += y;
    }
    const bool update = STATE_ONLY || !(flags & LAST) || ((flags & ENDS) && a.state_out);

    if (!STATE_ONLY) {
      float o[NV][4], s0[4], s1[4];
      if (!zero) {
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
      }
#pragma unroll
      for (int kk = 0; kk < 2 * NG; ++kk) {
        const int i0 = kk / 2, w = kk % 2 * 2;
        if (!EARLY && w == 0) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            load_shared(q[i0][e], slot + (2 * i0 + e) * 512);
            load_shared(k[i0][e], slot + (2 * NG + 2 * i0 + e) * 512);
          }
        }
        const uint32_t qa[4] = {q[i0][0][w], q[i0][1][w], q[i0][0][w + 1], q[i0][1][w + 1]};
        if (kk == 0) {
          mma16_new(s0, qa, k[i0][0][w], k[i0][0][w + 1], T());
          mma16_new(s1, qa, k[i0][1][w], k[i0][1][w + 1], T());
        } else {
          mma16(s0, qa, k[i0][0][w], k[i0][0][w + 1], T());
          mma16(s1, qa, k[i0][1][w], k[i0][1][w + 1], T());
        }
        if (!zero) {                                   // S in two parts
          if (BF) {
#pragma unroll
            for (int n = 0; n < NV; ++n) {
              const float(&u0)[4] = st[n / 2][2 * kk], (&u1)[4] = st[n / 2][2 * kk + 1];
              const int i = (n & 1) * 2;
              const uint32_t b0 = pack2(u0[i], u0[i + 1], T()), b1 = pack2(u1[i], u1[i + 1], T());
              const float2 h0 = halves(b0, T()), h1 = halves(b1, T());
              mma16(o[n], qa, pack2(u0[i] - h0.x, u0[i + 1] - h0.y, T()), pack2(u1[i] - h1.x, u1[i + 1] - h1.y, T()), T());
              mma16(o[n], qa, b0, b1, T());
            }
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {              // 8 channels of the key a time
              const float2 x0 = halves(qa[2 * e], T()), x1 = halves(qa[2 * e + 1], T());
              const uint32_t a0 = __float_as_uint(x0.x), a1 = __float_as_uint(x1.x);
              const uint32_t a2 = __float_as_uint(x0.y), a3 = __float_as_uint(x1.y);
#pragma unroll
              for (int n = 0; n < NV; ++n) {
                const float(&u)[4] = st[n / 2][2 * kk + e];
                const int i = (n & 1) * 2;
                const Parts b0 = tf32_split(u[i]), b1 = tf32_split(u[i + 1]);
                mma8(o[n], a0, a1, a2, a3, b0.lo, b1.lo);
                mma8(o[n], a0, a1, a2, a3, b0.hi, b1.hi);
              }
            }
          }
        }
      }
      const float pg = __shfl_sync(FULL, P, g), pg8 = __shfl_sync(FULL, P, g + 8);
      if (!zero) {
        const float e0 = a.scale * ex2(pg), e1 = a.scale * ex2(pg8);
#pragma unroll
        for (int n = 0; n < NV; ++n) o[n][0] *= e0, o[n][1] *= e0, o[n][2] *= e1, o[n][3] *= e1;
      }
      // the decays between rows, and none to a later row
      const float p0 = __shfl_sync(FULL, P, 2 * t), p1 = __shfl_sync(FULL, P, 2 * t + 1);
      const float p8 = __shfl_sync(FULL, P, 2 * t + 8), p9 = __shfl_sync(FULL, P, 2 * t + 9);
      s0[0] = 2 * t <= g ? s0[0] * (a.scale * ex2(pg - p0)) : 0.0f;
      s0[1] = 2 * t + 1 <= g ? s0[1] * (a.scale * ex2(pg - p1)) : 0.0f;
      s0[2] *= a.scale * ex2(pg8 - p0);
      s0[3] *= a.scale * ex2(pg8 - p1);
      s1[2] = 2 * t <= g ? s1[2] * (a.scale * ex2(pg8 - p8)) : 0.0f;
      s1[3] = 2 * t + 1 <= g ? s1[3] * (a.scale * ex2(pg8 - p9)) : 0.0f;
      if (BF) {
        uint32_t hi[4] = {pack2(s0[0], s0[1], T()), pack2(s0[2], s0[3], T()), 0u, pack2(s1[2], s1[3], T())};
        uint32_t lo[4];
        const float2 h0 = halves(hi[0], T()), h1 = halves(hi[1], T()), h3 = halves(hi[3], T());
        lo[0] = pack2(s0[0] - h0.x, s0[1] - h0.y, T()), lo[1] = pack2(s0[2] - h1.x, s0[3] - h1.y, T());
        lo[2] = 0u, lo[3] = pack2(s1[2] - h3.x, s1[3] - h3.y, T());
        add_rows(
            T(),
            [&](float(&d)[4], uint32_t b0, uint32_t b1, bool anew) {
              if (anew) mma16_new(d, hi, b0, b1, T());
              else mma16(d, hi, b0, b1, T());
              mma16(d, lo, b0, b1, T());
            },
            zero, o, vb, len, g, t);
      } else {
        const Parts f0 = tf32_split(s0[0]), f1 = tf32_split(s0[1]), f2 = tf32_split(s0[2]), f3 = tf32_split(s0[3]);
        const Parts f6 = tf32_split(s1[2]), f7 = tf32_split(s1[3]);
        add_rows(
            T(),
            [&](float(&d)[4], uint32_t b0, uint32_t b1, bool anew) {
              if (anew) d[0] = d[1] = d[2] = d[3] = 0.0f;
              const float2 v0 = halves(b0, T()), v1 = halves(b1, T());
              const uint32_t x0 = __float_as_uint(v0.x), y0 = __float_as_uint(v0.y);
              const uint32_t x1 = __float_as_uint(v1.x), y1 = __float_as_uint(v1.y);
              mma8(d, f0.lo, f2.lo, f1.lo, f3.lo, x0, y0);
              mma8(d, 0u, f6.lo, 0u, f7.lo, x1, y1);
              mma8(d, f0.hi, f2.hi, f1.hi, f3.hi, x0, y0);
              mma8(d, 0u, f6.hi, 0u, f7.hi, x1, y1);
            },
            zero, o, vb, len, g, t);
      }
      if (v_on) {
        const int along = dir * row + g;
        uint32_t w0[NV], w1[NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) w0[n] = pack2(o[n][0], o[n][1], T()), w1[n] = pack2(o[n][2], o[n][3], T());
        if (g < len) write_out(o0 + (int64_t)along * ob, w0);
        if (g + 8 < len) write_out(o0 + (int64_t)(along + 8) * ob, w1);
      }
    }

    if (update) {
      const float f = ex2(__shfl_sync(FULL, P, 15));
      if (zero) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) st[m][j][i] = 0.0f;
      } else if (!APART) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) st[m][j][i] *= f;
      }
      zero = false;
      float Z = __shfl_down_sync(FULL, x, 1, 16);
      if (lr == 15) Z = 0.0f;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        const float z = __shfl_down_sync(FULL, Z, o, 16);
        if (lr + o < 16) Z += z;
      }
      Z = ex2(Z);
      const float w0 = __shfl_sync(FULL, Z, 2 * t), w1 = __shfl_sync(FULL, Z, 2 * t + 1);
      const float w8 = __shfl_sync(FULL, Z, 2 * t + 8), w9 = __shfl_sync(FULL, Z, 2 * t + 9);
      // the decayed values in parts; fp16 has the bits but not the range for lower parts: tf32
      constexpr int TERMS = BF ? (EXACT ? 3 : 2) : 4;  // (fp16: of both parts the even and the odd rows)
      uint32_t va[TERMS][MT][4];
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float2 y = halves(vb[n][i], T());
          y.x *= i ? w8 : w0, y.y *= i ? w9 : w1;
          if (BF) {
#pragma unroll
            for (int e = 0; e < TERMS; ++e) {
              const uint32_t u = pack2(y.x, y.y, T());
              va[e][n / 2][2 * i + (n & 1)] = u;
              if (e + 1 < TERMS) {
                const float2 z = halves(u, T());
                y.x -= z.x, y.y -= z.y;
              }
            }
          } else {
            const Parts px = tf32_split(y.x), py = tf32_split(y.y);
            va[0][n / 2][2 * i + (n & 1)] = px.hi, va[1][n / 2][2 * i + (n & 1)] = py.hi;
            va[2][n / 2][2 * i + (n & 1)] = px.lo, va[3][n / 2][2 * i + (n & 1)] = py.lo;
          }
        }
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        const int i0 = j / 4;
        if (!EARLY && j % 4 == 0) {
          load_shared(k[i0][0], slot + (2 * NG + 2 * i0) * 512);
          load_shared(k[i0][1], slot + (2 * NG + 2 * i0 + 1) * 512);
        }
        const uint32_t b0 = turned(k[i0][0][j % 4]), b1 = turned(k[i0][1][j % 4]);
        const float2 k0 = halves(b0, T()), k1 = halves(b1, T());
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          float d[4];
          if (!APART) {
#pragma unroll
            for (int e = 0; e < TERMS; ++e) mma16(st[m][j], va[e][m], b0, b1, T());
            continue;
          }
          if (BF) {
            mma16_new(d, va[0][m], b0, b1, T());
#pragma unroll
            for (int e = 1; e < TERMS; ++e) mma16(d, va[e][m], b0, b1, T());
          } else {
            d[0] = d[1] = d[2] = d[3] = 0.0f;
#pragma unroll
            for (int e = TERMS - 2; e >= 0; e -= 2) {
              mma8(d, va[e][m][0], va[e][m][1], va[e + 1][m][0], va[e + 1][m][1], __float_as_uint(k0.x), __float_as_uint(k0.y));
              mma8(d, va[e][m][2], va[e][m][3], va[e + 1][m][2], va[e + 1][m][3], __float_as_uint(k1.x), __float_as_uint(k1.y));
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) st[m][j][i] = fmaf(st[m][j][i], f, d[i]);
        }
      }
      if ((flags & LAST) && (STATE_ONLY || (flags & ENDS))) {
        store_state(STATE_ONLY ? a.ws_state + ((tile + 1) * a.H + h) * KV : a.state_out + ((int64_t)ch.seq * a.H + h) * KV);
        if (STATE_ONLY) {
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) total += __shfl_xor_sync(FULL, total, o, 16);
          if (sl == 0 && lane == 0) a.ws_decay[(tile + 1) * a.H + h] = total / LOG2E;
        }
      }
    }
    if (!EARLY) {
      __syncwarp();
      next[NST - 1] = issue(s);
    }
  }
}

template <class T, int NG, int NV, bool STATE_ONLY, bool EXACT>
int launch(const LaArgs& a, cudaStream_t st) {
  auto kern = la_mma_kernel<T, NG, NV, STATE_ONLY, EXACT>;
  static_assert(NST * slot_bytes(NG, NV) <= 48 * 1024, "needs no leave");
  kern<<<linear_grid(a, STATE_ONLY), 32, NST * slot_bytes(NG, NV), st>>>(a);
  return launched();
}
template <class T, int NG, int NV>
int by_use(const LaArgs& a, bool state_only, cudaStream_t st) {
  if (state_only) return a.state_out ? launch<T, NG, NV, true, true>(a, st) : launch<T, NG, NV, true, false>(a, st);
  return a.state_out ? launch<T, NG, NV, false, true>(a, st) : launch<T, NG, NV, false, false>(a, st);
}
template <class T>
int by_width(const LaArgs& a, bool state_only, cudaStream_t st) {
  if (a.K <= 32) return by_use<T, 1, 4>(a, state_only, st);
  if (a.K <= 64) return by_use<T, 2, 4>(a, state_only, st);
  return by_use<T, 4, 2>(a, state_only, st);
}

}  // namespace

int seqops::linear_mma(int32_t dtype, const LaArgs& a, bool state_only, cudaStream_t st) {
  if (dtype == TRACKFIT_BF16_PROJ) return by_width<__nv_bfloat16>(a, state_only, st);
  return by_width<__half>(a, state_only, st);
}
