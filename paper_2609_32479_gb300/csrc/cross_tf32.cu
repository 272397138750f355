// Attention to packed states, fp32, on the tensor cores: tiles of 16 rows, a warp each, as
// cross_mma.cu has them for the 16-bit types, with 16 states a chunk.
//
// Every operand is the sum of two tf32 values of 11 bits, and of the four products of a pair
// of operands the three largest are taken (m16n8k8): what is left out is 2^-22 of a product, of
// the order of fp32's own rounding.  Three products of half the rate each leave 100 TFLOP/s of
// mma.sync's 604, against the 75 of the CUDA cores, whose operands would come from shared
// memory value by value.  Measured: 2,000 queries over 16,000 states, 4 heads of 64: 1603 us, 20
// TFLOP/s; the instructions that form the parts bound it, each warp for its own 16 rows.
//
// Lane (g, t) reads 16 bytes, channels 4t .. 4t+3 of each 16, of rows g and g + 8: with the k
// index permuted alike on both sides these are operands of Q K^T as they stand (slots t and
// t + 4 of step i are channels 4t + 2i, + 1).  The values stand in rows of shared memory, 4
// floats longer than their channels, so that the lanes' words (row 2t or 2t + 1, channel g)
// lie in 32 banks.
#include "cross_units.cuh"
#include "mma_sync.cuh"

namespace {
using namespace seqops;

constexpr int KC = 16;           // states of a chunk

template <int NG>                // groups of 16 channels
constexpr __host__ __device__ int queue() { return NG == 8 ? 2 : 3; }
template <int NG>
constexpr __host__ __device__ int pitch() { return NG * 16 + 4; }
template <int NG>
constexpr __host__ __device__ int slot_bytes() { return NG * 2 * 512 + KC * pitch<NG>() * 4; }

template <int NG>
__global__ void __launch_bounds__(32, NG <= 4 ? 12 : 8) ca_tf32_kernel(const __grid_constant__ CaArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int NST = queue<NG>(), SLOT = slot_bytes<NG>(), PV = pitch<NG>();
  const int lane = threadIdx.x, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % a.splits;
  const unsigned unit = blockIdx.x / a.splits;
  const int hk = unit % a.Hk, tile = unit / a.Hk;
  const int rows = (int)a.nq * a.G;
  const uint32_t base = smem_addr(smem), mine = base + lane * 16, mine_q = mine + NST * SLOT;
  if (a.D < NG * 16) {                                 // channels beyond D stay zero: the copies leave them alone
    for (int i = lane * 4; i < NST * SLOT + NG * 4 * 512; i += 128)
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + i), "r"(0) : "memory");
    __syncwarp();
  }
  bool in;
  int lo_l, hi_l, most;
  find_rows(a, tile, split, lane, in, lo_l, hi_l, most);
  const int lo0 = __shfl_sync(FULL, lo_l, g), hi0 = __shfl_sync(FULL, hi_l, g);
  const int lo1 = __shfl_sync(FULL, lo_l, g + 8), hi1 = __shfl_sync(FULL, hi_l, g + 8);
  const bool in0 = __shfl_sync(FULL, (int)in, g), in1 = __shfl_sync(FULL, (int)in, g + 8);
  const int row0 = tile * a.tr + g, row1 = row0 + 8;
  const float up = exp2f(weight_up<float>(most));
  const int end = __reduce_max_sync(FULL, hi0 > hi1 ? hi0 : hi1);

  // the queries' parts wait in shared memory (they would take 16 registers a group): the upper
  // ones [group][8 rows], then the lower
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const bool on = e ? in1 : in0;
    const int row = e ? row1 : row0;
    const float* p = (const float*)a.q + (int64_t)(on ? row / a.G : 0) * a.qs + (hk * a.G + row % a.G) * a.D + 4 * t;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (on && 16 * i + 4 * t < a.D) u = *reinterpret_cast<const uint4*>(p + 16 * i);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      Parts x[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) x[n] = tf32_parts(__uint_as_float((w[n] & a.q_and) ^ a.q_xor));
      const uint32_t to = mine_q + (2 * i + e) * 512;
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(x[0].hi), "r"(x[1].hi), "r"(x[2].hi), "r"(x[3].hi)
                   : "memory");
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + NG * 2 * 512), "r"(x[0].lo), "r"(x[1].lo), "r"(x[2].lo),
                   "r"(x[3].lo)
                   : "memory");
    }
  }
  const int64_t kb = a.ks * 4, vb = a.vs * 4;
  const char* k0 = reinterpret_cast<const char*>((const float*)a.k + hk * a.D + 4 * t);
  const char* v0 = reinterpret_cast<const char*>((const float*)a.v + hk * a.D);
  int ahead = first_wanted(0, lo0, hi0, lo1, hi1);
  int at[NST];
  auto issue = [&](int s) {
    const int pos = ahead;
    if (pos != FARTHEST) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = pos + 8 * r + g;
        const char* kp = k0 + row * kb;
#pragma unroll
        for (int i = 0; i < NG; ++i)
          if (16 * i + 4 * t < a.D) copy16(mine + s * SLOT + (2 * i + r) * 512, kp + 64 * i, row < end);
      }
#pragma unroll
      for (int i = 0; i < KC * NG * 4 / 32; ++i) {     // 16-byte pieces of the values' rows
        const int r = (lane + 32 * i) / (NG * 4), e = (lane + 32 * i) % (NG * 4);
        if (4 * e < a.D)
          copy16(base + s * SLOT + NG * 2 * 512 + (r * PV + 4 * e) * 4, v0 + (pos + r) * vb + 16 * e, pos + r < end);
      }
      ahead = first_wanted(pos + KC, lo0, hi0, lo1, hi1);
    }
    copy_commit();
    return pos;
  };
#pragma unroll
  for (int s = 0; s < NST; ++s) at[s] = issue(s);

  float o[NG * 2][4];
#pragma unroll
  for (int n = 0; n < NG * 2; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
  float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;   // m: score * scale2
  for (int s = 0;; s = s + 1 == NST ? 0 : s + 1) {
    const int pos = at[0];
#pragma unroll
    for (int i = 0; i + 1 < NST; ++i) at[i] = at[i + 1];
    if (pos == FARTHEST) break;
    copy_wait<NST - 1>();
    __syncwarp();
    float x[2][4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[n][i] = 0.0f;
#pragma unroll 2
    for (int i = 0; i < NG; ++i) {
      uint32_t h0[4], h1[4], g0[4], g1[4];
      load_shared(h0, mine_q + (2 * i) * 512);
      load_shared(h1, mine_q + (2 * i + 1) * 512);
      load_shared(g0, mine_q + (2 * NG + 2 * i) * 512);
      load_shared(g1, mine_q + (2 * NG + 2 * i + 1) * 512);
      uint32_t k[2][4];
      load_shared(k[0], mine + s * SLOT + (2 * i) * 512);
      load_shared(k[1], mine + s * SLOT + (2 * i + 1) * 512);
      float d[2][4];                                   // these channels' sum, added outside the products
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) d[n][c] = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; w += 2) {
        const uint32_t ah[4] = {h0[w], h1[w], h0[w + 1], h1[w + 1]}, al[4] = {g0[w], g1[w], g0[w + 1], g1[w + 1]};
#pragma unroll
        for (int n = 0; n < 2; ++n)
          mma8_parts(d[n], ah, al, tf32_bparts(__uint_as_float(k[n][w])), tf32_bparts(__uint_as_float(k[n][w + 1])));
      }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[n][c] += d[n][c];
    }
    // states that are not a row's own count nothing
    const bool whole = __all_sync(FULL, lo0 <= pos && pos + KC <= hi0 && lo1 <= pos && pos + KC <= hi1);
    if (!whole) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int j = pos + 8 * n + 2 * t + e;
          if (j < lo0 || j >= hi0) x[n][e] = -INFINITY;
          if (j < lo1 || j >= hi1) x[n][2 + e] = -INFINITY;
        }
    }
    float t0 = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1])), t1 = fmaxf(fmaxf(x[0][2], x[0][3]), fmaxf(x[1][2], x[1][3]));
#pragma unroll
    for (int y = 1; y <= 2; y <<= 1) {
      t0 = fmaxf(t0, __shfl_xor_sync(FULL, t0, y));
      t1 = fmaxf(t1, __shfl_xor_sync(FULL, t1, y));
    }
    t0 = fmaxf(m0, t0 * a.scale2), t1 = fmaxf(m1, t1 * a.scale2);
    const float n0 = t0 == -INFINITY ? 0.0f : t0, n1 = t1 == -INFINITY ? 0.0f : t1;
    const float f0 = ex2(m0 - n0), f1 = ex2(m1 - n1);
    m0 = t0, m1 = t1;
    float c0 = 0.0f, c1 = 0.0f;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      // (the factor in the exponent would cost the argument five bits)
      x[n][0] = up * ex2(fmaf(x[n][0], a.scale2, -n0)), x[n][1] = up * ex2(fmaf(x[n][1], a.scale2, -n0));
      x[n][2] = up * ex2(fmaf(x[n][2], a.scale2, -n1)), x[n][3] = up * ex2(fmaf(x[n][3], a.scale2, -n1));
      c0 += x[n][0] + x[n][1], c1 += x[n][2] + x[n][3];
    }
    l0 = fmaf(l0, f0, c0), l1 = fmaf(l1, f1, c1);
    uint32_t ph[2][4], pl[2][4];                       // rows g, g + 8 by slots t, t + 4: states 2t, 2t + 1
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Parts p = tf32_parts(x[n][(i & 1) * 2 + (i >> 1)]);
        ph[n][i] = p.hi, pl[n][i] = p.lo;
      }
    const float* sv = reinterpret_cast<const float*>(smem + s * SLOT + NG * 2 * 512) + 2 * t * PV + g;
    bool mixed = false;
    if (!whole) {
      float sum = 0.0f;
#pragma unroll
      for (int n = 0; n < NG * 2; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          sum = fmaf(sv[8 * e * PV + 8 * n], 0.0f, sum);
          sum = fmaf(sv[(8 * e + 1) * PV + 8 * n], 0.0f, sum);
        }
      mixed = __any_sync(FULL, !(sum == 0.0f));
    }
    // a chunk's own sum first, added to O outside the products: their accumulation cuts bits off, and
    // over a long range would draw sums of one sign towards zero (16,000 states: 5e-6, 60,000: 2e-5)
#pragma unroll
    for (int n = 0; n < NG * 2; ++n) {
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float v0 = sv[8 * e * PV + 8 * n], v1 = sv[(8 * e + 1) * PV + 8 * n];
        const BParts b0 = tf32_bparts_of_weighted(v0), b1 = tf32_bparts_of_weighted(v1), none = {0u, 0u, 0u};
        if (!mixed) {
          mma8_parts(sum, ph[e], pl[e], b0, b1);
        } else {
          // a value that is not finite stays out of the rows that do not read it: each row by itself
          for (int r = 0; r < 16; ++r) {
            const int j = pos + 8 * e + 2 * t, rl = __shfl_sync(FULL, lo_l, r), rh = __shfl_sync(FULL, hi_l, r);
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            mma8_parts(d, ph[e], pl[e], j >= rl && j < rh ? b0 : none, j + 1 >= rl && j + 1 < rh ? b1 : none);
            if (g == r) sum[0] += d[0], sum[1] += d[1];
            if (g + 8 == r) sum[2] += d[2], sum[3] += d[3];
          }
        }
      }
      o[n][0] = fmaf(o[n][0], f0, sum[0]), o[n][1] = fmaf(o[n][1], f0, sum[1]);
      o[n][2] = fmaf(o[n][2], f1, sum[2]), o[n][3] = fmaf(o[n][3], f1, sum[3]);
    }
    __syncwarp();                                      // read: the place is free
    at[NST - 1] = issue(s);
  }
#pragma unroll
  for (int y = 1; y <= 2; y <<= 1) {
    l0 += __shfl_xor_sync(FULL, l0, y);
    l1 += __shfl_xor_sync(FULL, l1, y);
  }
  const int64_t r0 = ((int64_t)split * rows + row0) * a.Hk + hk, r1 = ((int64_t)split * rows + row1) * a.Hk + hk;
  const bool joined = a.splits > 1;
  const float f0 = joined ? 1.0f : l0 == 0.0f ? 0.0f : 1.0f / l0, f1 = joined ? 1.0f : l1 == 0.0f ? 0.0f : 1.0f / l1;
  if (joined && t == 0) {
    if (in0) a.ws_ml[r0] = make_float2(m0, l0);
    if (in1) a.ws_ml[r1] = make_float2(m1, l1);
  }
  float* p0 = joined ? a.ws_o + r0 * a.D : (float*)a.out + (int64_t)(row0 / a.G) * a.os + (hk * a.G + row0 % a.G) * a.D;
  float* p1 = joined ? a.ws_o + r1 * a.D : (float*)a.out + (int64_t)(row1 / a.G) * a.os + (hk * a.G + row1 % a.G) * a.D;
#pragma unroll
  for (int n = 0; n < NG * 2; ++n) {
    const int c = 8 * n + 2 * t;
    if (c >= a.D) continue;
    if (in0) *reinterpret_cast<float2*>(p0 + c) = make_float2(average(o[n][0], f0), average(o[n][1], f0));
    if (in1) *reinterpret_cast<float2*>(p1 + c) = make_float2(average(o[n][2], f1), average(o[n][3], f1));
  }
}

template <int NG>
int launch(const CaArgs& a, cudaStream_t st) {
  constexpr auto kern = ca_tf32_kernel<NG>;
  const size_t smem = queue<NG>() * slot_bytes<NG>() + NG * 4 * 512;
  const cudaError_t e = allow_smem<kern>(smem);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  const int64_t units = (a.nq * a.G + a.tr - 1) / a.tr * a.Hk * a.splits;
  if (units > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  kern<<<(unsigned)units, 32, smem, st>>>(a);
  return launched();
}

}  // namespace

int seqops::cross_tf32(const CaArgs& a, cudaStream_t st) {
  if (a.D <= 32) return launch<2>(a, st);
  if (a.D <= 64) return launch<4>(a, st);
  return launch<8>(a, st);
}
