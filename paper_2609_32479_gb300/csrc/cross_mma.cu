// Attention to packed states, 16-bit types, on the tensor cores: tiles of 16 rows, a warp each.
//
// A warp goes through the states that any of its rows reads, 32 at a time: S = Q K^T, the
// running maximum m and sum l of each row, P = 2^(S - m), O = O 2^(m_before - m) + P V, as
// m16n8k16 products.  The rows' ranges need not be the same: a tile of five-query tracks
// reads three tracks' states, and what is not a row's own is masked.  A row's range is never
// left: a weight of zero times an infinity of another sequence would be NaN, so where V is
// not finite and ranges differ each row takes its own states by itself.
//
// Operands as in linear_mma.cu: 16 bytes a lane, channels 8t .. 8t+7 of each 32, rows g, g + 8,
// ..., through a queue of each lane's own words in shared memory; movmatrix turns V.
//
// What bounds it: for tracks the instructions (131,072 tracks of five queries, 4 heads of 32, bf16:
// 350 us a call, 3.7 TB/s of the 6.8 that a copy moves), for single queries memory (a state's K and V
// are read once for the G heads that share them: 61 queries over 1-16,384 states, 4 heads of 128: 212
// us a call, 4.3 TB/s; 173 the kernel, with five warps an SM).  P is the sum of two 16-bit parts as an operand of P V: with
// one, rounded to 2^-8 (fp16 2^-11), the readout took 320 us instead of 355 and outputs were off by
// as much again as by their own rounding.
#include "cross_units.cuh"
#include "mma_sync.cuh"

namespace {
using namespace seqops;

constexpr int KC = 32;           // states of a chunk

template <int NG>
constexpr __host__ __device__ int queue() { return NG == 4 ? 2 : 3; }

template <class T, int NG>
__global__ void __launch_bounds__(32, NG == 1 ? 16 : 8) ca_mma_kernel(const __grid_constant__ CaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NST = queue<NG>();
  constexpr int SLOT = NG * 8 * 512;                   // K, then V: [group][8 rows] of 32 x 16 bytes
  const int lane = threadIdx.x, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % a.splits;
  const unsigned unit = blockIdx.x / a.splits;
  // a warp takes `each` heads of the states, one after the other: the sequences of the tile's rows
  // are looked for once
  const int sets = a.Hk / a.each, first_head = unit % sets * a.each;
  const int tile = unit / sets;
  const int rows = (int)a.nq * a.G;
  const uint32_t mine = smem_addr(smem) + lane * 16;
  if (a.D < NG * 32) {                                 // channels beyond D stay zero: the copies leave them alone
    for (int i = 0; i < NST * NG * 8; ++i)
      asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(mine + i * 512), "r"(0) : "memory");
  }

  bool in;
  int lo_l, hi_l, most;
  find_rows(a, tile, split, lane, in, lo_l, hi_l, most);
  const int lo0 = __shfl_sync(FULL, lo_l, g), hi0 = __shfl_sync(FULL, hi_l, g);
  const int lo1 = __shfl_sync(FULL, lo_l, g + 8), hi1 = __shfl_sync(FULL, hi_l, g + 8);
  const bool in0 = __shfl_sync(FULL, (int)in, g), in1 = __shfl_sync(FULL, (int)in, g + 8);
  const int row0 = tile * a.tr + g, row1 = row0 + 8;
  const float up = weight_up<T>(most);
  const int end = __reduce_max_sync(FULL, hi0 > hi1 ? hi0 : hi1);
  auto wanted = [&](int pos) { return first_wanted(pos, lo0, hi0, lo1, hi1); };

  for (int hk = first_head; hk < first_head + a.each; ++hk) {
    uint32_t q[NG][2][4];
    {
      const T* p0 = (const T*)a.q + (int64_t)(in0 ? row0 / a.G : 0) * a.qs + (hk * a.G + row0 % a.G) * a.D + 8 * t;
      const T* p1 = (const T*)a.q + (int64_t)(in1 ? row1 / a.G : 0) * a.qs + (hk * a.G + row1 % a.G) * a.D + 8 * t;
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint4 u = make_uint4(0, 0, 0, 0);
          if ((e ? in1 : in0) && 32 * i + 8 * t < a.D) u = *reinterpret_cast<const uint4*>((e ? p1 : p0) + 32 * i);
          q[i][e][0] = (u.x & a.q_and) ^ a.q_xor, q[i][e][1] = (u.y & a.q_and) ^ a.q_xor;
          q[i][e][2] = (u.z & a.q_and) ^ a.q_xor, q[i][e][3] = (u.w & a.q_and) ^ a.q_xor;
        }
    }
    const int kb = (int)a.ks * 2, vb = (int)a.vs * 2;
    const char* k0 = reinterpret_cast<const char*>((const T*)a.k + hk * a.D + 8 * t);
    const char* v0 = reinterpret_cast<const char*>((const T*)a.v + hk * a.D + 8 * t);
    int ahead = wanted(0);                               // the next chunk to fetch
    int at[NST];                                         // first states of the chunks in the queue
    auto issue = [&](int s) {
      const int pos = ahead;
      if (pos != FARTHEST) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = pos + 8 * r + g;
          const bool on = row < end;
          const char* kp = k0 + (int64_t)row * kb;
          const char* vp = v0 + (int64_t)row * vb;
#pragma unroll
          for (int i = 0; i < NG; ++i)
            if (32 * i + 8 * t < a.D) {
              copy16(mine + s * SLOT + (4 * i + r) * 512, kp + 64 * i, on);
              copy16(mine + s * SLOT + (4 * NG + 4 * i + r) * 512, vp + 64 * i, on);
            }
        }
        ahead = wanted(pos + KC);
      }
      copy_commit();
      return pos;
    };
#pragma unroll
    for (int s = 0; s < NST; ++s) at[s] = issue(s);

    float o[NG * 4][4];
#pragma unroll
    for (int n = 0; n < NG * 4; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;   // m: score * scale2
    for (int s = 0;; s = s + 1 == NST ? 0 : s + 1) {
      const int pos = at[0];
#pragma unroll
      for (int i = 0; i + 1 < NST; ++i) at[i] = at[i + 1];
      if (pos == FARTHEST) break;
      copy_wait<NST - 1>();
      const uint32_t slot = mine + s * SLOT;
      // nothing in the chunk's upper half (looked at for narrow heads, whose chunks of a track are
      // short; the branches cost the wide ones a fifth)
      const bool lower = NG == 1 && pos + 16 >= end;
      float x[4][4];
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          if (n >= 2 && lower) {
            if (i == 0) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.0f;
            continue;
          }
          uint32_t k[4];
          load_shared(k, slot + (4 * i + n) * 512);
#pragma unroll
          for (int w = 0; w < 4; w += 2) {
            const uint32_t qa[4] = {q[i][0][w], q[i][1][w], q[i][0][w + 1], q[i][1][w + 1]};
            if (i == 0 && w == 0) mma16_new(x[n], qa, k[w], k[w + 1], T());
            else mma16(x[n], qa, k[w], k[w + 1], T());
          }
        }
      // states that are not a row's own count nothing
      const bool whole0 = lo0 <= pos && pos + KC <= hi0, whole1 = lo1 <= pos && pos + KC <= hi1;
      const bool whole = __all_sync(FULL, whole0 && whole1);
      if (!whole) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int j = pos + 8 * n + 2 * t + e;
            if (j < lo0 || j >= hi0) x[n][e] = -INFINITY;
            if (j < lo1 || j >= hi1) x[n][2 + e] = -INFINITY;
          }
      }
      float t0 = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1])), fmaxf(fmaxf(x[2][0], x[2][1]), fmaxf(x[3][0], x[3][1])));
      float t1 = fmaxf(fmaxf(fmaxf(x[0][2], x[0][3]), fmaxf(x[1][2], x[1][3])), fmaxf(fmaxf(x[2][2], x[2][3]), fmaxf(x[3][2], x[3][3])));
#pragma unroll
      for (int y = 1; y <= 2; y <<= 1) {
        t0 = fmaxf(t0, __shfl_xor_sync(FULL, t0, y));
        t1 = fmaxf(t1, __shfl_xor_sync(FULL, t1, y));
      }
      t0 = fmaxf(m0, t0 * a.scale2), t1 = fmaxf(m1, t1 * a.scale2);
      const float n0 = t0 == -INFINITY ? 0.0f : t0, n1 = t1 == -INFINITY ? 0.0f : t1;
      const float f0 = ex2(m0 - n0), f1 = ex2(m1 - n1);
      m0 = t0, m1 = t1;
      const float b0 = up - n0, b1 = up - n1;
      float c0 = 0.0f, c1 = 0.0f;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        x[n][0] = ex2(fmaf(x[n][0], a.scale2, b0)), x[n][1] = ex2(fmaf(x[n][1], a.scale2, b0));
        x[n][2] = ex2(fmaf(x[n][2], a.scale2, b1)), x[n][3] = ex2(fmaf(x[n][3], a.scale2, b1));
        c0 += x[n][0] + x[n][1], c1 += x[n][2] + x[n][3];
      }
      l0 = fmaf(l0, f0, c0), l1 = fmaf(l1, f1, c1);
      uint32_t pa[2][4], pl[2][4];                       // the weights in two parts
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float p0 = x[2 * e + w / 2][w % 2 * 2], p1 = x[2 * e + w / 2][w % 2 * 2 + 1];
          pa[e][w] = pack2(p0, p1, T());
          const float2 h = halves(pa[e][w], T());
          pl[e][w] = pack2(p0 - h.x, p1 - h.y, T());
        }
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        uint32_t v[4][4], sum = 0u;
#pragma unroll
        for (int r = 0; r < 4; ++r) load_shared(v[r], slot + (4 * NG + 4 * i + r) * 512);
        bool mixed = false;
        if (!whole) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int w = 0; w < 4; ++w) sum = zero_if_finite(v[r][w], sum, T());
          mixed = __any_sync(FULL, (sum & 0x7fff7fffu) != 0u);
        }
        // a chunk's own sum first, added to O outside the products: their accumulation cuts bits off, and
        // over a long range would draw sums of one sign towards zero
        if (!mixed) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            float sum[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if (e == 1 && lower) continue;
              const uint32_t u0 = turned(v[2 * e][w]), u1 = turned(v[2 * e + 1][w]);
              if (e == 0) mma16_new(sum, pl[e], u0, u1, T());
              else mma16(sum, pl[e], u0, u1, T());
              mma16(sum, pa[e], u0, u1, T());
            }
            float(&on)[4] = o[4 * i + w];
            on[0] = fmaf(on[0], f0, sum[0]), on[1] = fmaf(on[1], f0, sum[1]);
            on[2] = fmaf(on[2], f1, sum[2]), on[3] = fmaf(on[3], f1, sum[3]);
          }
        } else {
#pragma unroll
          for (int w = 0; w < 4; ++w) o[4 * i + w][0] *= f0, o[4 * i + w][1] *= f0, o[4 * i + w][2] *= f1, o[4 * i + w][3] *= f1;
          for (int r = 0; r < 16; ++r) {
            const int rl = __shfl_sync(FULL, lo_l, r) - pos, rh = __shfl_sync(FULL, hi_l, r) - pos;
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                uint32_t u[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  const int j = 16 * e + 8 * c + 2 * t;
                  u[c] = turned(v[2 * e + c][w]) & ((j >= rl && j < rh ? 0xffffu : 0u) | (j + 1 >= rl && j + 1 < rh ? 0xffff0000u : 0u));
                }
                float d[4];
                mma16_new(d, pl[e], u[0], u[1], T());
                mma16(d, pa[e], u[0], u[1], T());
                if (g == r) o[4 * i + w][0] += d[0], o[4 * i + w][1] += d[1];
                if (g + 8 == r) o[4 * i + w][2] += d[2], o[4 * i + w][3] += d[3];
              }
          }
        }
      }
      __syncwarp();                                      // read: the place is free
      at[NST - 1] = issue(s);
    }
#pragma unroll
    for (int y = 1; y <= 2; y <<= 1) {
      l0 += __shfl_xor_sync(FULL, l0, y);
      l1 += __shfl_xor_sync(FULL, l1, y);
    }
    if (a.splits == 1) {
      const float f0 = l0 == 0.0f ? 0.0f : 1.0f / l0, f1 = l1 == 0.0f ? 0.0f : 1.0f / l1;
      T* p0 = (T*)a.out + (int64_t)(row0 / a.G) * a.os + (hk * a.G + row0 % a.G) * a.D + 8 * t;
      T* p1 = (T*)a.out + (int64_t)(row1 / a.G) * a.os + (hk * a.G + row1 % a.G) * a.D + 8 * t;
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        if (32 * i + 8 * t >= a.D) continue;
        uint32_t w0[4], w1[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          w0[w] = pack2(o[4 * i + w][0] * f0, o[4 * i + w][1] * f0, T());
          w1[w] = pack2(o[4 * i + w][2] * f1, o[4 * i + w][3] * f1, T());
        }
        if (in0) write_out(p0 + 32 * i, w0);
        if (in1) write_out(p1 + 32 * i, w1);
      }
      continue;
    }
    const int64_t part = (int64_t)split * rows;
    const int64_t r0 = (part + row0) * a.Hk + hk, r1 = (part + row1) * a.Hk + hk;
    if (t == 0) {
      if (in0) a.ws_ml[r0] = make_float2(m0, l0);
      if (in1) a.ws_ml[r1] = make_float2(m1, l1);
    }
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      if (32 * i + 8 * t >= a.D) continue;
#pragma unroll
      for (int w = 0; w < 4; w += 2) {
        const int c = 32 * i + 8 * t + 2 * w;
        if (in0) *reinterpret_cast<float4*>(a.ws_o + r0 * a.D + c) = make_float4(o[4 * i + w][0], o[4 * i + w][1], o[4 * i + w + 1][0], o[4 * i + w + 1][1]);
        if (in1) *reinterpret_cast<float4*>(a.ws_o + r1 * a.D + c) = make_float4(o[4 * i + w][2], o[4 * i + w][3], o[4 * i + w + 1][2], o[4 * i + w + 1][3]);
      }
    }
  }
}

template <class T, int NG>
int launch(const CaArgs& a, cudaStream_t st) {
  constexpr auto kern = ca_mma_kernel<T, NG>;
  const size_t smem = queue<NG>() * NG * 8 * 512;
  const cudaError_t e = allow_smem<kern>(smem);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  const int64_t units = (a.nq * a.G + a.tr - 1) / a.tr * (a.Hk / a.each) * a.splits;
  if (units > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  kern<<<(unsigned)units, 32, smem, st>>>(a);
  return launched();
}
template <class T>
int by_width(const CaArgs& a, cudaStream_t st) {
  if (a.D <= 32) return launch<T, 1>(a, st);
  if (a.D <= 64) return launch<T, 2>(a, st);
  return launch<T, 4>(a, st);
}

}  // namespace

int seqops::cross_mma(int32_t dtype, const CaArgs& a, cudaStream_t st) {
  return dtype == TRACKFIT_BF16_PROJ ? by_width<__nv_bfloat16>(a, st) : by_width<__half>(a, st);
}
