// Attention of many queries to many packed states, 16-bit types, on the tcgen05 tensor cores:
// tiles of 128 rows of one head of the states, blocks of 64 states.
//
//   S = Q K^T (tensor memory), P = 2^(S - m), O = O 2^(m_before - m) + P V (tensor memory)
//
// A CTA goes through the sequences that its rows belong to, one after the other (a pass each);
// rows of other sequences take part in the products and are not written.  Sequences of fewer
// than 64 states are left to the 16-row kernel.  The last block of a sequence ends at its last
// state and takes the first ones twice, the second time with weight zero: no state of another
// sequence is ever in a product.
//   warps 0-3  a thread a row: the maximum of S, the weights (two 16-bit parts each, put in the
//              place of the scores, which P V reads as its A operand), the sum; at a pass's end
//              O / l
//   warp 4     TMA loads of K and V
//   warp 5     the tcgen05.mma issuer and owner of the tensor memory
// S has two places: the scores of the next block are formed while the weights of this one are, and
// P V runs behind.  (In one place, with blocks of 128 states, the chain of
// product, weights and product left the tensor cores idle most of the time: 448 us for 4,099
// queries and 30,011 states of 8 heads of 64.)  A thread holds a block's 64 scores in registers:
// one read of the tensor memory.
// The maximum that the weights are taken against moves only when a row's grows by more than 2^LAG:
// O is hardly ever read back and scaled.
// With heads up to 64 channels two CTAs share an SM (80 KB and 256 columns each), one's products
// beside the other's exponentials.
//
// With one part a weight, rounded to 2^-8 (fp16 2^-11), outputs were off by as much again as by
// their own rounding; it was stored in shared memory and took 327 (bf16) and 351 us (fp16) instead of
// 388 and 421 for the case below.
// Bound: a block takes an SM 985 clocks, of which its twelve products of 128 x 64 x 16 (four for the
// scores, eight for both parts of the weights) need 384, its 8,192 exponentials 256, and the 504
// instructions of each of its four warps as many of a scheduler; the rest is the chain of a block,
// which two CTAs an SM do not hide.
// Measured: 4,099 queries over 30,011 states, 8 heads of 64, fp16: 421 us a call, 600 TFLOP/s of the
// 1,969 that a large library product reaches (the lower parts' products not counted).
//
// Every wait has a limit; where one expires, the CTA gives up, the call's outputs are not valid,
// and trackfit_operator_errors() says so.
#include <cuda.h>
#include <cudaTypedefs.h>

#include "cross_units.cuh"
#include "mma_sync.cuh"
#include "sm100_ptx.cuh"

namespace {
using namespace seqops;
using namespace sm100;

constexpr int TILE = 128;                    // rows of a tile
constexpr int BLOCK = CROSS_TC_FROM;         // states of a block
constexpr uint32_t ATOM_Q = TILE * 128;      // 128 rows of 64 channels
constexpr uint32_t ATOM = BLOCK * 128;       // 64 states of 64 channels
constexpr uint64_t LIMIT_NS = 2000000000ull;   // of a wait; a test hook shortens it
constexpr int STAGES = 4;
static_assert(BLOCK == 64, "a block's weights, in two parts, take the place of its scores");
// The maximum that the weights are taken against may be 2^LAG behind.  Not further in fp16: the
// weights lie as much lower in the type's range (2^-38 of the largest is what one may be off).
template <class T>
constexpr float LAG = __is_same(T, __half) ? 2.0f : 8.0f;

// Blocks whose products are added up in O before the row's thread puts it aside: the accumulation
// cuts bits off, up to 2^-23 of O a step of 16 states, which draws sums of one sign towards zero
// (32 blocks: 1.4e-5, a 35th of an fp16 output's rounding, whatever the range; in one sum it would
// be that rounding for a range of 100,000 states).
constexpr int ASIDE = 32;

struct TcArgs {
  CaArgs a;
  int tiles;
  uint32_t idesc_s, idesc_o;
  uint64_t limit_ns;
  int hold;                                  // test hook: the first CTA's loader holds its first block back
};

struct Bars {
  uint64_t k_full[STAGES], k_free[STAGES], v_full[STAGES], v_free[STAGES];
  uint64_t s_full[2], p_full[2], p_free[2], o_done, drained;
  uint32_t tmem;
  int abort_flag;
};

template <int NA>
constexpr __host__ __device__ uint32_t smem_bytes() {
  return NA * ATOM_Q + 2 * STAGES * NA * ATOM + 256;
}
// Of tensor memory: two places of S, O and what of it is put aside.
template <int NA>
constexpr __host__ __device__ uint32_t columns() {
  return NA == 1 ? 256 : 512;
}
static_assert(sizeof(Bars) <= 256, "the barriers' place");

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::
          "r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}

// The passes of a tile, alike for every warp.
struct Pass {
  int lo, len;          // the sequence's states
  int first, last;      // rows of the tile that are its queries: [first, last)
  int j0, j1;           // this part's blocks
};
class Passes {
 public:
  __device__ __forceinline__ Passes(const CaArgs& a, int row0, int split, int lane) : a_(a), row0_(row0), split_(split) {
    b_ = first_at_least(a.qo, a.n_seq, (int64_t)row0 / a.G + 1, lane) - 1;
    if (b_ < 0) b_ = 0;
  }
  __device__ __forceinline__ bool next(Pass& p) {
    const int64_t rows = a_.nq * a_.G, top = row0_ + TILE < rows ? row0_ + TILE : rows;
    for (; b_ < a_.n_seq; ) {
      const int64_t qlo = clamp64(a_.qo[b_], 0, a_.nq) * a_.G, qhi = clamp64(a_.qo[b_ + 1], 0, a_.nq) * a_.G;
      if (qlo >= top) return false;
      const int64_t b = b_++;
      if (qhi <= row0_ || qhi <= qlo) continue;
      const int64_t lo = clamp64(a_.ko[b], 0, a_.nk), hi = clamp64(a_.ko[b + 1], lo, a_.nk);
      if (hi - lo < BLOCK) continue;
      p.lo = (int)lo, p.len = (int)(hi - lo);
      p.first = (int)(qlo > row0_ ? qlo - row0_ : 0), p.last = (int)((qhi < top ? qhi : top) - row0_);
      const int64_t nb = (p.len + BLOCK - 1) / BLOCK;
      p.j0 = (int)(nb * split_ / a_.splits), p.j1 = (int)(nb * (split_ + 1) / a_.splits);
      return true;
    }
    return false;
  }

 private:
  const CaArgs& a_;
  int row0_, split_;
  int64_t b_;
};
// The first state of a block.
__device__ __forceinline__ int block_at(const Pass& p, int j) {
  return p.lo + ((int64_t)(j + 1) * BLOCK > p.len ? p.len - BLOCK : j * BLOCK);
}

__device__ unsigned long long g_expired;   // CTAs that gave up; it only grows

__device__ __forceinline__ void give_up(Bars* s) {
  if (atomicExch(&s->abort_flag, 1) == 0) atomicAdd(&g_expired, 1ull);
}

template <class T, int NA>
__global__ void __launch_bounds__(192, NA == 1 ? 2 : 1)
    ca_tc_kernel(const __grid_constant__ TcArgs p, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const CaArgs& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned unit = blockIdx.x;
  const int tile = unit % p.tiles, hk = unit / p.tiles % a.Hk, split = unit / p.tiles / a.Hk;
  const int row0 = tile * TILE;
  const int rows = (int)(a.nq * a.G);
  const uint32_t base = smem_u32(smem);
  if (base & 1023u) {                                  // the swizzled tiles' alignment, asked for above
    if (threadIdx.x == 0) atomicAdd(&g_expired, 1ull);
    return;
  }
  const uint32_t q_s = base, k_s = q_s + NA * ATOM_Q, v_s = k_s + STAGES * NA * ATOM;
  Bars* bars = reinterpret_cast<Bars*>(smem + smem_bytes<NA>() - 256);
  const uint32_t s_full = smem_u32(bars->s_full), p_full = smem_u32(bars->p_full), p_free = smem_u32(bars->p_free);
  const uint32_t o_done = smem_u32(&bars->o_done);
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&bars->k_full[i]), 1);
      mbar_init(smem_u32(&bars->k_free[i]), 1);
      mbar_init(smem_u32(&bars->v_full[i]), 1);
      mbar_init(smem_u32(&bars->v_free[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 8 * i, 128);
      mbar_init(p_free + 8 * i, 1);
    }
    mbar_init(o_done, 1);
    mbar_init(smem_u32(&bars->drained), 1);
    bars->abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 5) {
    tmem_alloc(smem_u32(&bars->tmem), columns<NA>());
    tmem_relinquish();
  }
  // the tile's queries: rows of 128 bytes, 16-byte pieces swizzled as the K-major operand wants
  for (int i = threadIdx.x; i < TILE * NA * 8; i += 192) {
    const int r = i / (NA * 8), e = i % (NA * 8), row = row0 + r;
    uint4 u = make_uint4(0, 0, 0, 0);
    if (row < rows && e * 8 < a.D)
      u = *reinterpret_cast<const uint4*>((const T*)a.q + (int64_t)(row / a.G) * a.qs + (hk * a.G + row % a.G) * a.D + e * 8);
    const uint32_t at = q_s + (e >> 3) * ATOM_Q + r * 128 + (((e & 7) ^ (r & 7)) << 4);
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"((u.x & a.q_and) ^ a.q_xor),
                 "r"((u.y & a.q_and) ^ a.q_xor), "r"((u.z & a.q_and) ^ a.q_xor), "r"((u.w & a.q_and) ^ a.q_xor)
                 : "memory");
  }
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem, tmem_o = tmem + 2 * BLOCK, tmem_aside = tmem_o + 64 * NA;
  volatile int* abort = &bars->abort_flag;
  Passes passes(a, row0, split, lane);
  Pass ps;

  if (warp == 4) {
    // ---- loads
    if (elect_one()) {
      prefetch_tmap(&tk);
      prefetch_tmap(&tv);
      uint32_t n = 0;                                  // blocks loaded
      bool ok = true;
      while (ok && passes.next(ps)) {
        for (int j = ps.j0; j < ps.j1 && ok; ++j, ++n) {
          const int s = n % STAGES, row = block_at(ps, j);
          const uint32_t ph = (n / STAGES & 1) ^ 1;
          const uint32_t kf = smem_u32(&bars->k_full[s]), vf = smem_u32(&bars->v_full[s]);
          if (p.hold && unit == 0 && n == 0) {
            const uint64_t t0 = globaltimer();
            while (!*abort && globaltimer() - t0 < 2 * p.limit_ns) __nanosleep(1000);
            ok = !*abort;
            if (!ok) break;
          }
          ok = mbar_wait(smem_u32(&bars->k_free[s]), ph, abort, p.limit_ns);
          if (!ok) break;
          mbar_arrive_expect_tx(kf, NA * ATOM);
          for (int c = 0; c < NA; ++c) tma_load_3d(k_s + (s * NA + c) * ATOM, &tk, kf, 64 * c, hk, row);
          ok = mbar_wait(smem_u32(&bars->v_free[s]), ph, abort, p.limit_ns);
          if (!ok) {
            // the keys just asked for land before the CTA may exit
            volatile int never = 0;
            mbar_wait(kf, n / STAGES & 1, &never, LIMIT_NS);
            break;
          }
          mbar_arrive_expect_tx(vf, NA * ATOM);
          for (int c = 0; c < NA; ++c) tma_load_3d(v_s + (s * NA + c) * ATOM, &tv, vf, 64 * c, hk, row);
        }
      }
      if (!ok) give_up(bars);
      // copies still under way land before the CTA exits (after a failure nobody else waits for them)
      volatile int never = 0;
      for (uint32_t i = n < STAGES ? 0 : n - STAGES; i < n; ++i) {
        mbar_wait(smem_u32(&bars->k_full[i % STAGES]), i / STAGES & 1, &never, LIMIT_NS);
        mbar_wait(smem_u32(&bars->v_full[i % STAGES]), i / STAGES & 1, &never, LIMIT_NS);
      }
    }
    __syncwarp();
  } else if (warp == 5) {
    // ---- products
    if (elect_one()) {
      uint32_t n = 0;                                  // blocks of the passes before
      bool ok = true;
      // the scores of block m of all, in place m & 1, where the weights of the block before the last
      // were: their product has ended
      auto scores = [&](uint32_t m) {
        const int s = m % STAGES;
        ok = (m < 2 || mbar_wait(p_free + 8 * (m & 1), (m >> 1 & 1) ^ 1, abort, p.limit_ns)) &&
             mbar_wait(smem_u32(&bars->k_full[s]), m / STAGES & 1, abort, p.limit_ns);
        if (!ok) return;
        tc_fence_after();
        const uint32_t ks = k_s + s * NA * ATOM;
        for (int c = 0; c < NA; ++c)
          for (int k = 0; k < 4; ++k)
            umma_f16(tmem + (m & 1) * BLOCK, sdesc_sw128(q_s + c * ATOM_Q + 32 * k, 16, 1024),
                     sdesc_sw128(ks + c * ATOM + 32 * k, 16, 1024), p.idesc_s, c | k);
        umma_commit(s_full + 8 * (m & 1));
        umma_commit(smem_u32(&bars->k_free[s]));
      };
      while (ok && passes.next(ps)) {
        const uint32_t blocks = ps.j1 - ps.j0;
        if (blocks > 0) scores(n);
        for (uint32_t j = 0; j < blocks && ok; ++j) {
          const uint32_t m = n + j;
          const int s = m % STAGES;
          if (j + 1 < blocks) scores(m + 1);
          ok = ok && mbar_wait(p_full + 8 * (m & 1), m >> 1 & 1, abort, p.limit_ns) &&
               mbar_wait(smem_u32(&bars->v_full[s]), m / STAGES & 1, abort, p.limit_ns);
          if (!ok) break;
          tc_fence_after();
          // both parts of the weights, 8 columns for 16 states; V as it lies, [state][channel]: groups
          // of 8 states 1024 bytes apart, 64 channels ATOM
          for (int k = 0; k < BLOCK / 8; ++k)
            umma_f16_ts(tmem_o, tmem + (m & 1) * BLOCK + 8 * k, sdesc_sw128(v_s + s * NA * ATOM + k % 4 * 2048, ATOM, 1024),
                        p.idesc_o, ((j % ASIDE) > 0) | (k > 0));
          umma_commit(p_free + 8 * (m & 1));
          umma_commit(smem_u32(&bars->v_free[s]));
          if (j + 1 == blocks) umma_commit(o_done);
        }
        n += blocks;
      }
      if (!ok) give_up(bars);
      // products still under way end before their memory is given back
      volatile int never = 0;
      umma_commit(smem_u32(&bars->drained));
      mbar_wait(smem_u32(&bars->drained), 0, &never, LIMIT_NS);
    }
    __syncwarp();
  } else {
    // ---- a thread a row
    const int r = threadIdx.x, row = row0 + r;
    const uint32_t lanes = (uint32_t)(32 * warp) << 16;
    uint32_t n = 0, done = 0;
    bool ok = true;
    while (ok && passes.next(ps)) {
      float m = -INFINITY, l = 0.0f;                   // m: score * scale2 that the weights are taken against
      float m_aside = -INFINITY;                       // .. that those of what is put aside were
      const float up = weight_up<T>(ps.len) - LAG<T>;
      for (int j = ps.j0; j < ps.j1; ++j, ++n) {
        const uint32_t place = n & 1, phase = n >> 1 & 1;
        ok = __all_sync(FULL, mbar_wait(s_full + 8 * place, phase, abort, p.limit_ns));
        if (!ok) break;
        tc_fence_after();
        float v[2][32];
        tmem_ld32(tmem + lanes + place * BLOCK, v[0]);
        tmem_ld32(tmem + lanes + place * BLOCK + 32, v[1]);
        tmem_ld_wait();
        if ((int64_t)(j + 1) * BLOCK > ps.len) {       // the last block: states that the one before had
          const int twice = (int)((int64_t)(j + 1) * BLOCK - ps.len);
#pragma unroll
          for (int i = 0; i < BLOCK; ++i)
            if (i < twice) v[i / 32][i % 32] = -INFINITY;
        }
        float t0 = v[0][0], t1 = v[0][1], t2 = v[0][2], t3 = v[0][3];
#pragma unroll
        for (int i = 4; i < BLOCK - 4; i += 8) {
          t0 = max3(t0, v[i / 32][i % 32], v[(i + 1) / 32][(i + 1) % 32]);
          t1 = max3(t1, v[(i + 2) / 32][(i + 2) % 32], v[(i + 3) / 32][(i + 3) % 32]);
          t2 = max3(t2, v[(i + 4) / 32][(i + 4) % 32], v[(i + 5) / 32][(i + 5) % 32]);
          t3 = max3(t3, v[(i + 6) / 32][(i + 6) % 32], v[(i + 7) / 32][(i + 7) % 32]);
        }
        t0 = max3(t0, v[1][28], v[1][29]), t1 = max3(t1, v[1][30], v[1][31]);
        const float top = fmaxf(max3(t0, t1, t2), t3) * a.scale2;
        const bool aside = j > ps.j0 && (j - ps.j0) % ASIDE == 0;
        const bool moves = j > ps.j0 && __any_sync(FULL, top > m + LAG<T>);
        if (j == ps.j0) m = top;
        if (aside || moves) {
          // the product before this block adds to O until then
          ok = __all_sync(FULL, mbar_wait(p_free + 8 * (place ^ 1), (n - 1) >> 1 & 1, abort, p.limit_ns));
          if (!ok) break;
          tc_fence_after();
          // put aside as it is, or scaled to the new maximum (with one row of the warp all that have grown)
          const float f = aside ? m_aside == -INFINITY ? 0.0f : ex2(m_aside - m) : top > m ? ex2(m - top) : 1.0f;
          const bool first = j - ps.j0 == ASIDE;
          const uint32_t to = lanes + (aside ? tmem_aside : tmem_o);
#pragma unroll 1
          for (int c = 0; c < NA * 4; ++c) {
            float o[16];
            tmem_ld16(to + 16 * c, o);
            if (aside) {
              float x[16];
              tmem_ld16(tmem_o + lanes + 16 * c, x);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = first ? x[i] : fmaf(o[i], f, x[i]);
            } else {
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] *= f;
            }
            tmem_st16(to + 16 * c, o);
          }
          tmem_st_wait();
          if (aside) m_aside = m;
          if (moves && top > m) {
            l *= ex2(m - top);
            m = top;
          }
        }
        const float mm = m == -INFINITY ? 0.0f : m;
        const uint64_t scale = both(a.scale2, a.scale2), minus = both(up - mm, up - mm), back = both(-1.0f, -1.0f);
        uint64_t s0 = 0, s1 = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {                  // 16 states: 8 columns of the upper parts, 8 of the lower
          float hi[8], lo[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = 16 * c + 2 * i;
            const float2 x = parts(fma2(both(v[e / 32][e % 32], v[(e + 1) / 32][(e + 1) % 32]), scale, minus));
            const uint64_t w = both(ex2(x.x), ex2(x.y));
            if (i & 1) s1 = add2(s1, w);
            else s0 = add2(s0, w);
            const float2 y = parts(w);
            const uint32_t u = pack2(y.x, y.y, T());
            const float2 h = halves(u, T());
            const float2 z = parts(fma2(both(h.x, h.y), back, w));
            hi[i] = __uint_as_float(u), lo[i] = __uint_as_float(pack2(z.x, z.y, T()));
          }
          tmem_st8(tmem + lanes + place * BLOCK + 8 * c, hi);
          tmem_st8(tmem + lanes + place * BLOCK + 32 + 8 * c, lo);
        }
        const float2 sum = parts(add2(s0, s1));
        l += sum.x + sum.y;
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(p_full + 8 * place);
      }
      if (!ok) break;
      const bool mine = r >= ps.first && r < ps.last, any = ps.j1 > ps.j0;
      if (any) {
        ok = __all_sync(FULL, mbar_wait(o_done, done++ & 1, abort, p.limit_ns));
        if (!ok) break;
        tc_fence_after();
      }
      const int64_t at = ((int64_t)split * rows + row) * a.Hk + hk;
      const float f = a.splits > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
      if (a.splits > 1 && mine) a.ws_ml[at] = make_float2(m, l);
      const float f_aside = m_aside == -INFINITY ? 0.0f : ex2(m_aside - m);
      T* out = mine ? (T*)a.out + (int64_t)(row / a.G) * a.os + (hk * a.G + row % a.G) * a.D : nullptr;
      float* part = mine ? a.ws_o + at * a.D : nullptr;
#pragma unroll 1
      for (int c = 0; c < NA * 2; ++c) {
        float v[32];
        __syncwarp();
        if (any) {
          tmem_ld32(tmem_o + lanes + 32 * c, v);
          tmem_ld_wait();
          if (ps.j1 - ps.j0 > ASIDE) {
            float x[32];
            tmem_ld32(tmem_aside + lanes + 32 * c, x);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = fmaf(x[i], f_aside, v[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = 0.0f;
        }
        if (!mine) continue;
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          if (32 * c + i >= a.D) continue;
          if (a.splits > 1) {
            *reinterpret_cast<float4*>(part + 32 * c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            *reinterpret_cast<float4*>(part + 32 * c + i + 4) = make_float4(v[i + 4], v[i + 5], v[i + 6], v[i + 7]);
          } else {
            *reinterpret_cast<uint4*>(out + 32 * c + i) =
                make_uint4(pack2(v[i] * f, v[i + 1] * f, T()), pack2(v[i + 2] * f, v[i + 3] * f, T()),
                           pack2(v[i + 4] * f, v[i + 5] * f, T()), pack2(v[i + 6] * f, v[i + 7] * f, T()));
          }
        }
      }
    }
    if (!ok) give_up(bars);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 5) tmem_dealloc(tmem, columns<NA>());
}

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

// [rows][heads][D] with a row stride, boxes of 64 channels of a head and 64 rows, 128-byte swizzle;
// channels from D on and rows beyond the array read as zero.
bool make_map(CUtensorMap* m, const void* p, int64_t rows, int64_t stride, int heads, int D, bool fp16) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)rows};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, 1, BLOCK}, step[3] = {1, 1, 1};
  return fn(m, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims,
            strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

std::atomic<uint64_t> g_limit_ns{LIMIT_NS};
std::atomic<int> g_hold{0};

template <class T, int NA>
int launch(const CaArgs& a, bool fp16, cudaStream_t st) {
  TcArgs p;
  p.a = a;
  p.tiles = (int)((a.nq * a.G + TILE - 1) / TILE);
  p.idesc_s = idesc_f16(128, BLOCK, fp16 ? 0u : 1u, false, false);
  p.idesc_o = idesc_f16(128, NA * 64, fp16 ? 0u : 1u, false, true);
  p.limit_ns = g_limit_ns.load(), p.hold = g_hold.load();
  CUtensorMap tk, tv;
  if (!make_map(&tk, a.k, a.nk, a.ks, a.Hk, a.D, fp16) || !make_map(&tv, a.v, a.nk, a.vs, a.Hk, a.D, fp16))
    return TRACKFIT_ERR_CUDA;
  constexpr auto kern = ca_tc_kernel<T, NA>;
  const cudaError_t e = allow_smem<kern>(smem_bytes<NA>());
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  const int64_t units = (int64_t)p.tiles * a.Hk * a.splits;
  if (units > 0x7fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  kern<<<(unsigned)units, 192, smem_bytes<NA>(), st>>>(p, tk, tv);
  return launched();
}

}  // namespace

int seqops::cross_tc(int32_t dtype, const CaArgs& a, cudaStream_t st) {
  if (dtype == TRACKFIT_BF16_PROJ)
    return a.D <= 64 ? launch<__nv_bfloat16, 1>(a, false, st) : launch<__nv_bfloat16, 2>(a, false, st);
  return a.D <= 64 ? launch<__half, 1>(a, true, st) : launch<__half, 2>(a, true, st);
}

uint64_t seqops::operator_limit_ns() { return g_limit_ns.load(); }

unsigned long long* seqops::operator_expired() {
  static std::atomic<unsigned long long*> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  unsigned long long* p = dev < 64 ? known[dev].load() : nullptr;
  if (!p) {
    const cudaError_t e = cudaGetSymbolAddress(reinterpret_cast<void**>(&p), g_expired);
    if (e != cudaSuccess) {
      tf_note_cuda(e, "cudaGetSymbolAddress");
      return nullptr;
    }
    if (dev < 64) known[dev].store(p);
  }
  return p;
}

extern "C" int trackfit_debug_operator_wait(int64_t limit_ns, int32_t hold) {
  if (limit_ns < 0 || limit_ns > (int64_t)LIMIT_NS || hold < 0 || hold > 1) return TRACKFIT_ERR_INVALID_ARG;
  g_limit_ns.store(limit_ns > 0 ? (uint64_t)limit_ns : LIMIT_NS);
  g_hold.store(hold);
  return TRACKFIT_OK;
}

namespace {
// What a thread was told of last, for each stream that it asked with: one that asks takes nothing
// away from another.  A pair that finds no place any more, or had to give it up, is told of all.
struct Told {
  int dev;
  void* stream;
  unsigned long long n;
};
constexpr int TOLD = 64;
thread_local Told t_told[TOLD];
thread_local int t_pairs = 0;      // ever, of which the last TOLD have a place
}  // namespace

extern "C" int trackfit_operator_errors(void* stream) {
  tf_nvtx_range nvtx_range("trackfit_operator_errors");
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  void* p = nullptr;
  unsigned long long n = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaGetSymbolAddress(&p, g_expired);
  if (e == cudaSuccess) e = cudaMemcpyAsync(&n, p, sizeof(n), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  Told* told = nullptr;
  for (int i = 0; i < t_pairs && i < TOLD && !told; ++i)
    if (t_told[i].dev == dev && t_told[i].stream == stream) told = &t_told[i];
  if (!told) {
    told = &t_told[t_pairs % TOLD];
    t_pairs = t_pairs + 1 < 2 * TOLD ? t_pairs + 1 : TOLD;
    *told = {dev, stream, 0};
  }
  const bool more = n > told->n;
  told->n = n;
  return more ? TRACKFIT_ERR_TIMEOUT : TRACKFIT_OK;
}
