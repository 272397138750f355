// Rows times a weight matrix with its epilogue on the tensor cores, 16-bit and 8-bit operands.
//
// Tiles of 128 rows x BN outputs a CTA or, in pairs of CTAs on two neighbouring SMs, 256 x BN,
// where each CTA brings its 128 rows of x and half of the tile's rows of W, and the one product
// instruction of the first reads both halves: half as many bytes of W go into each SM.  A CTA
// (pair) takes tile after tile; two accumulators in tensor memory, so that the epilogue of one
// tile runs beside the products of the next.
//
//   warp 0      TMA loads of 128 bytes of K of x and W into a ring of stages
//   warp 1      products, by one lane (of the first CTA of a pair)
//   warp 2      TMA loads of gate and residual, 128 bytes x 128 rows at a time, into slots
//   warp 3      tensor memory
//   warps 4-11  epilogue: two sets of four warps take pieces of 128 bytes of outputs by turns; a
//               thread has a row of the piece, puts it into the piece's slot and a warp stores its
//               32 rows by TMA.  (Stores and loads a row a thread would touch 32 lines each.)
//
// Measured: 8011 x 4096 x 4096 in bf16 166 us, 1,618 TFLOP/s (the library's product alone 171), with gelu in
// fp16 177 to 195 as the card's power lets it, in 8 bits 95 to 102, 2,700 TFLOP/s; bound by the operands' way
// into the SM (256 rows of 128 bytes a step) and the power.  1,310,003 x 256 x 128, gated onto a residual: 244 us,
// the bytes at the rate of a copy.  With K small and an activation the epilogue's eight warps bound it:
// 100,000 x 256 x 896 with silu 119 us of 34.
//
// Every wait is limited; one that expires sets the CTA's flag, on which all others give up too,
// and is counted for trackfit_operator_errors().
#include "product_units.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>

namespace {
using namespace seqops;
using namespace sm100;

constexpr int THREADS = 384;
constexpr int EPI_WARPS = 8;
constexpr int MAX_STAGES = 12;
constexpr int SLOTS = 4;
constexpr int PIECE = 128 * 128;               // bytes of a piece: 128 rows x 128 bytes
constexpr int SMEM = 227 * 1024;
constexpr int RESERVED = 2048;                 // alignment, barriers
constexpr uint64_t DRAIN_NS = 200000000ull;

struct TcArgs {
  CUtensorMap tx, tw, tg, tr, to;
  ProductArgs a;
  int tiles_m, tiles_n, kblocks, bn, stages, slot_bytes, group;
  uint32_t idesc;
  uint64_t limit_ns;
  unsigned long long* expired;
};

struct Bars {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], acc_full[2], acc_empty[2], slot_full[SLOTS], slot_empty[SLOTS], drain;
  uint32_t tmem;
  int abort, never;
};

__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of the same shared memory in the first CTA of the pair.
__device__ __forceinline__ uint32_t in_first(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void load_2d_pair(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, "
      "%4}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
template <int CG, bool EIGHT>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t onto) {
#define TF_MMA(group, kind)                                                                                            \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::" group ".kind::" kind            \
               " [%0], %1, %2, %3, p;\n\t}" ::"r"(d),                                                                   \
               "l"(a), "l"(b), "r"(idesc), "r"(onto)                                                                    \
               : "memory")
  if constexpr (CG == 1 && !EIGHT) TF_MMA("1", "f16");
  if constexpr (CG == 1 && EIGHT) TF_MMA("1", "f8f6f4");
  if constexpr (CG == 2 && !EIGHT) TF_MMA("2", "f16");
  if constexpr (CG == 2 && EIGHT) TF_MMA("2", "f8f6f4");
#undef TF_MMA
}
// An arrival on `bar` of the CTA (of both CTAs of the pair) when the products so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (CG == 1)
    umma_commit(bar);
  else
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}

// Tiles in an order in which those that run together share rows of x and of W: `group` tiles of
// rows by all tiles of outputs, the rows first.
__device__ __forceinline__ void place(const TcArgs& p, int t, int& tm, int& tn) {
  const int per = p.group * p.tiles_n, g = t / per, in = t - g * per;
  const int rows = p.tiles_m - g * p.group < p.group ? p.tiles_m - g * p.group : p.group;
  tn = in / rows, tm = g * p.group + in - tn * rows;
}

__device__ __forceinline__ void lds4(uint32_t addr, uint32_t (&v)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void sts4(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

template <class T, int CG, bool EIGHT>
__global__ void __launch_bounds__(THREADS, 1) product_tc_kernel(const __grid_constant__ TcArgs p) {
  constexpr int VE = 16 / sizeof(T), PC = 128 / sizeof(T);   // outputs of 16 bytes, of a piece
  constexpr int KB = EIGHT ? 128 : 64;                       // channels of a stage
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const int stage_bytes = (128 + p.bn / CG) * 128;
  const uint32_t slots = base + (uint32_t)(p.stages * stage_bytes);
  Bars* bars = reinterpret_cast<Bars*>(smem_raw + (base - raw) + p.stages * stage_bytes + SLOTS * p.slot_bytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cta_rank() : 0u;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) mbar_init(smem_u32(&bars->full[s]), 1), mbar_init(smem_u32(&bars->empty[s]), 1);
    for (int b = 0; b < 2; ++b) mbar_init(smem_u32(&bars->acc_full[b]), 1), mbar_init(smem_u32(&bars->acc_empty[b]), EPI_WARPS * CG);
    for (int s = 0; s < SLOTS; ++s) mbar_init(smem_u32(&bars->slot_full[s]), 1), mbar_init(smem_u32(&bars->slot_empty[s]), 4);
    mbar_init(smem_u32(&bars->drain), 1);
    bars->abort = bars->never = 0;
    fence_mbar_init();
  }
  if (warp == 3) {
    if constexpr (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&bars->tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tmem_alloc(smem_u32(&bars->tmem), 512);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync();
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  volatile int *abort = &bars->abort, *never = &bars->never;
  const int total = p.tiles_m * p.tiles_n, first = blockIdx.x / CG, step = gridDim.x / CG;
  const int pieces = (p.bn + PC - 1) / PC;
  const bool operands = p.a.gate || p.a.res;
  auto fail = [&] {
    if (atomicExch(&bars->abort, 1) == 0) atomicAdd(p.expired, 1ull);
  };

  if (warp == 0 && lane == 0) {
    prefetch_tmap(&p.tx);
    prefetch_tmap(&p.tw);
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (int t = first; t < total && !*abort; t += step) {
      int tm, tn;
      place(p, t, tm, tn);
      const int m0 = (tm * CG + (int)rank) * 128, n0 = tn * p.bn + (int)rank * (p.bn / CG);
      for (int k = 0; k < p.kblocks; ++k) {
        if (!mbar_wait(smem_u32(&bars->empty[s]), ph ^ 1u, abort, p.limit_ns)) {
          fail();
          break;
        }
        const uint32_t at = base + (uint32_t)(s * stage_bytes), full = smem_u32(&bars->full[s]);
        if constexpr (CG == 2) {
          // both CTAs' copies count on the first one's barrier
          if (rank == 0) mbar_arrive_expect_tx(full, 2u * (uint32_t)stage_bytes);
          const uint32_t bar = in_first(full);
          load_2d_pair(at, &p.tx, bar, k * KB, m0);
          load_2d_pair(at + 128 * 128, &p.tw, bar, k * KB, n0);
        } else {
          mbar_arrive_expect_tx(full, (uint32_t)stage_bytes);
          tma_load_2d(at, &p.tx, full, k * KB, m0);
          tma_load_2d(at + 128 * 128, &p.tw, full, k * KB, n0);
        }
        ++issued;
        if (++s == p.stages) s = 0, ph ^= 1u;
      }
    }
    if (*abort) {
      // copies in flight land before the CTA may go; the second of a pair has no barrier of its own
      // for them and gives them the limit's time
      if (CG == 2) {
        const uint64_t t0 = globaltimer();
        while (globaltimer() - t0 < DRAIN_NS) {
        }
      } else {
        for (int i = issued < p.stages ? 0 : issued - p.stages; i < issued; ++i)
          mbar_wait(smem_u32(&bars->full[i % p.stages]), (uint32_t)(i / p.stages) & 1u, never, DRAIN_NS);
      }
    }
  } else if (warp == 1 && lane == 0 && rank == 0) {
    int s = 0, n = 0;
    uint32_t ph = 0;
    bool issued = false, ok = true;
    for (int t = first; t < total && ok; t += step, ++n) {
      const int buf = n & 1;
      if (!mbar_wait(smem_u32(&bars->acc_empty[buf]), ((n >> 1) & 1) ^ 1u, abort, p.limit_ns)) {
        fail();
        break;
      }
      tc_fence_after();
      for (int k = 0; k < p.kblocks; ++k) {
        if (!mbar_wait(smem_u32(&bars->full[s]), ph, abort, p.limit_ns)) {
          fail();
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t at = base + (uint32_t)(s * stage_bytes);
        const uint64_t da = sdesc_sw128(at, 16, 1024), db = sdesc_sw128(at + 128 * 128, 16, 1024);
#pragma unroll
        for (int i = 0; i < 4; ++i) mma<CG, EIGHT>(tmem + buf * 256, da + 2 * i, db + 2 * i, p.idesc, k | i ? 1u : 0u);
        issued = true;
        commit<CG>(smem_u32(&bars->empty[s]));
        if (++s == p.stages) s = 0, ph ^= 1u;
      }
      if (ok) commit<CG>(smem_u32(&bars->acc_full[buf]));
    }
    if (issued) {   // every product done before the tensor memory goes
      commit<CG>(smem_u32(&bars->drain));
      if (!mbar_wait(smem_u32(&bars->drain), 0, never, DRAIN_NS)) fail();
    }
  } else if (warp == 2 && lane == 0 && operands) {
    int c = 0;
    bool ok = true;
    for (int t = first; t < total && ok; t += step) {
      int tm, tn;
      place(p, t, tm, tn);
      const int m0 = (tm * CG + (int)rank) * 128;
      for (int j = 0; j < pieces; ++j, ++c) {
        const int slot = c % SLOTS;
        if (!mbar_wait(smem_u32(&bars->slot_empty[slot]), ((c / SLOTS) & 1) ^ 1u, abort, p.limit_ns)) {
          fail();
          ok = false;
          break;
        }
        const uint32_t full = smem_u32(&bars->slot_full[slot]), at = slots + (uint32_t)(slot * p.slot_bytes);
        const int n0 = tn * p.bn + j * PC;
        mbar_arrive_expect_tx(full, PIECE * ((p.a.gate ? 1 : 0) + (p.a.res ? 1 : 0)));
        if (p.a.res) tma_load_2d(at, &p.tr, full, n0, m0);
        if (p.a.gate) tma_load_2d(at + p.slot_bytes - PIECE, &p.tg, full, n0, m0);
      }
    }
    if (*abort)
      for (int i = c < SLOTS ? 0 : c - SLOTS; i < c; ++i)
        mbar_wait(smem_u32(&bars->slot_full[i % SLOTS]), (uint32_t)(i / SLOTS) & 1u, never, DRAIN_NS);
  } else if (warp >= 4) {
    const int q = warp & 3, set = (warp - 4) >> 2, r = 32 * q + lane;
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    int c = 0, last = -1, n = 0;
    bool ok = true;
    for (int t = first; t < total && ok; t += step, ++n) {
      int tm, tn;
      place(p, t, tm, tn);
      const int64_t row0 = (int64_t)(tm * CG + (int)rank) * 128 + 32 * q;
      const float xs = EIGHT && row0 + lane < p.a.n ? p.a.x_scales[row0 + lane] : 0.0f;
      const int buf = n & 1;
      const uint32_t acc = tmem + lanes + buf * 256;
      ok = __all_sync(FULL, mbar_wait(smem_u32(&bars->acc_full[buf]), (n >> 1) & 1, abort, p.limit_ns));
      if (!ok) break;
      tc_fence_after();
      for (int j = 0; j < pieces; ++j, ++c) {
        if ((c & 1) != set) continue;
        const int slot = c % SLOTS, n0 = tn * p.bn + j * PC;
        const uint32_t mine = slots + (uint32_t)(slot * p.slot_bytes + r * 128), its = mine + p.slot_bytes - PIECE;
        if (operands) {
          // the piece before is on its way: its slot is free for the loads of the piece after this one
          if (lane == 0 && last >= 0) {
            bulk_wait_read_keep(0);
            mbar_arrive(smem_u32(&bars->slot_empty[last]));
          }
          ok = __all_sync(FULL, mbar_wait(smem_u32(&bars->slot_full[slot]), (uint32_t)(c / SLOTS) & 1u, abort, p.limit_ns));
          if (!ok) break;
        } else {
          if (lane == 0) bulk_wait_read_keep(1);   // of this warp's pieces, the one before the last was in this slot
          __syncwarp();
        }
        // 32 outputs at a time (16 bits: the second 32 are on their way with the first)
        float v[PC / 32][32];
#pragma unroll
        for (int h = 0; h < PC / 32; ++h) tmem_ld32(acc + j * PC + h * 32, v[h]);
        tmem_ld_wait();
#pragma unroll
        for (int h = 0; h < PC / 32; ++h) {
          const int col = n0 + h * 32, left = p.a.M - col;
          auto put = [&](int i) {
            const uint32_t piece = (uint32_t)(((h * 32 + i) * (int)sizeof(T) >> 4) ^ (r & 7)) << 4;
            float y[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) y[e] = v[h][i + e];
            uint32_t g[4] = {}, x[4] = {};
            if (p.a.gate) lds4(its + piece, g);
            if (p.a.res) lds4(mine + piece, x);
            gated<T>(p.a, y, make_uint4(g[0], g[1], g[2], g[3]), make_uint4(x[0], x[1], x[2], x[3]));
            sts4(mine + piece, pack(y, T()));
          };
          if (left >= 32) {
            activated<EIGHT>(p.a, v[h], xs, col);
#pragma unroll
            for (int i = 0; i < 32; i += VE) put(i);
          } else {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {         // (outputs are a multiple of 8)
              if (i >= left) break;
              float y[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = v[h][i + e];
              activated<EIGHT>(p.a, y, xs, col + i);
#pragma unroll
              for (int e = 0; e < 8; ++e) v[h][i + e] = y[e];
#pragma unroll
              for (int e = 0; e < 8; e += VE) put(i + e);
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0 && row0 < p.a.n && n0 < p.a.M) {
          tma_store_2d(&p.to, slots + (uint32_t)(slot * p.slot_bytes + 32 * q * 128), n0, (int)row0);
          bulk_commit();
        }
        last = slot;
      }
      if (!ok) break;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) arrive_cluster(in_first(smem_u32(&bars->acc_empty[buf])));
        else mbar_arrive(smem_u32(&bars->acc_empty[buf]));
      }
    }
    if (!ok && lane == 0) fail();
    if (lane == 0) bulk_wait_all();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync();
  tc_fence_after();
  if (warp == 3) {
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else
      tmem_dealloc(tmem, 512);
  }
}

// ---------------------------------------------------------------- few tiles

// A tile of 128 x BN by a cluster of CTAs, each with a part of K: their sums go to shared memory, and each
// CTA finishes a part of the tile out of all of them, in their order.
//   warp 0      TMA loads
//   warp 1      products, tensor memory
//   warps 2-5   the sums from tensor memory; all: the epilogue
constexpr int SPLIT_THREADS = 192;

struct SplitBars {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], done;
  uint32_t tmem;
  int abort, never;
};

__device__ __forceinline__ float from_cta(uint32_t at, int rank) {
  uint32_t u;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(u) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(u) : "memory");
  return v;
}

template <class T, bool EIGHT>
__global__ void __launch_bounds__(SPLIT_THREADS, 1) product_split_kernel(const __grid_constant__ TcArgs p, int split) {
  constexpr int VE = 16 / sizeof(T), KB = EIGHT ? 128 : 64;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const int stage_bytes = (128 + p.bn) * 128;
  float* sums = reinterpret_cast<float*>(smem_raw + (base - raw) + p.stages * stage_bytes);   // [BN][128 rows]
  SplitBars* bars = reinterpret_cast<SplitBars*>(sums + p.bn * 128);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) mbar_init(smem_u32(&bars->full[s]), 1), mbar_init(smem_u32(&bars->empty[s]), 1);
    mbar_init(smem_u32(&bars->done), 1);
    bars->abort = bars->never = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&bars->tmem), 128);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem;
  volatile int *abort = &bars->abort, *never = &bars->never;
  const int part = blockIdx.x % split, tile = blockIdx.x / split;
  const int tm = tile / p.tiles_n, tn = tile % p.tiles_n, m0 = tm * 128, n0 = tn * p.bn;
  const int k_lo = p.kblocks * part / split, k_hi = p.kblocks * (part + 1) / split;
  auto fail = [&] {
    if (atomicExch(&bars->abort, 1) == 0) atomicAdd(p.expired, 1ull);
  };
  if (warp == 0 && lane == 0) {
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (int k = k_lo; k < k_hi; ++k) {
      if (!mbar_wait(smem_u32(&bars->empty[s]), ph ^ 1u, abort, p.limit_ns)) {
        fail();
        break;
      }
      const uint32_t at = base + (uint32_t)(s * stage_bytes), full = smem_u32(&bars->full[s]);
      mbar_arrive_expect_tx(full, (uint32_t)stage_bytes);
      tma_load_2d(at, &p.tx, full, k * KB, m0);
      tma_load_2d(at + 128 * 128, &p.tw, full, k * KB, n0);
      ++issued;
      if (++s == p.stages) s = 0, ph ^= 1u;
    }
    if (*abort)
      for (int i = issued < p.stages ? 0 : issued - p.stages; i < issued; ++i)
        mbar_wait(smem_u32(&bars->full[i % p.stages]), (uint32_t)(i / p.stages) & 1u, never, DRAIN_NS);
  } else if (warp == 1 && lane == 0) {
    int s = 0;
    uint32_t ph = 0;
    for (int k = k_lo; k < k_hi; ++k) {
      if (!mbar_wait(smem_u32(&bars->full[s]), ph, abort, p.limit_ns)) {
        fail();
        break;
      }
      tc_fence_after();
      const uint32_t at = base + (uint32_t)(s * stage_bytes);
      const uint64_t da = sdesc_sw128(at, 16, 1024), db = sdesc_sw128(at + 128 * 128, 16, 1024);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma<1, EIGHT>(tmem, da + 2 * i, db + 2 * i, p.idesc, k > k_lo || i ? 1u : 0u);
      commit<1>(smem_u32(&bars->empty[s]));
      if (++s == p.stages) s = 0, ph ^= 1u;
    }
    commit<1>(smem_u32(&bars->done));
    if (!mbar_wait(smem_u32(&bars->done), 0, never, DRAIN_NS)) fail();   // (before the tensor memory goes)
  } else if (warp >= 2) {
    const bool ok = __all_sync(FULL, mbar_wait(smem_u32(&bars->done), 0, abort, p.limit_ns));
    if (!ok && lane == 0) fail();
    tc_fence_after();
    const int r = 32 * (warp & 3) + lane;
    for (int c = 0; c < p.bn; c += 16) {
      float v[16];
      tmem_ld16(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + c, v);
      tmem_ld_wait();
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[(c + i) * 128 + r] = v[i];
    }
    tc_fence_before();
  }
  __syncwarp();
  cluster_sync();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 128);
  const int items = p.bn / VE * 128, lo = items * part / split, hi = items * (part + 1) / split;
  for (int i = lo + (int)threadIdx.x; i < hi; i += SPLIT_THREADS) {
    const int r = i & 127, c = (i >> 7) * VE;
    const int64_t row = (int64_t)m0 + r;
    if (row >= p.a.n || n0 + c >= p.a.M) continue;
    float y[VE] = {};
    for (int u = 0; u < split; ++u)
#pragma unroll
      for (int e = 0; e < VE; ++e) y[e] += from_cta(smem_u32(sums + (c + e) * 128 + r), u);
    const int64_t col = n0 + c;
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 gate = p.a.gate ? *reinterpret_cast<const uint4*>((const T*)p.a.gate + row * p.a.gs + col) : none;
    const uint4 res = p.a.res ? *reinterpret_cast<const uint4*>((const T*)p.a.res + row * p.a.rs + col) : none;
    finish<T, EIGHT>(p.a, y, EIGHT ? p.a.x_scales[row] : 1.0f, (int)col, gate, res);
    *reinterpret_cast<uint4*>((T*)p.a.out + row * p.a.os + col) = pack(y, T());
  }
  cluster_sync();   // no CTA goes while another reads its sums
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

// [rows][width] with a row stride, boxes of 128 bytes x `high` rows, 128-byte swizzle; beyond the
// array loads give zeros and stores nothing.
bool make_map(CUtensorMap* m, const void* p, int64_t rows, int64_t width, int64_t stride, int size, CUtensorMapDataType type,
              int high) {
  const auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * size};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)high}, step[2] = {1, 1};
  return fn(m, type, 2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T>
CUtensorMapDataType map_type() {
  return sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
         : __is_same(T, __half) ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
}

// CTA pairs that are resident together (the SMs of an odd group have no partner).
template <auto kern>
int resident_pairs() {
  static std::atomic<int> known{0};
  int n = known.load();
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 2, at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.gridDim = dim3(152), cfg.blockDim = dim3(THREADS), cfg.dynamicSmemBytes = SMEM, cfg.attrs = &at, cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = 64;
  }
  known.store(n);
  return n;
}

template <class T, int CG, bool EIGHT>
int launch(const ProductArgs& a, int bn, cudaStream_t st) {
  TcArgs p;
  p.a = a;
  const int size = EIGHT ? 1 : (int)sizeof(T);
  const CUtensorMapDataType in = EIGHT ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : map_type<T>();
  bool ok = make_map(&p.tx, a.x, a.n, a.K, a.xs, size, in, 128) && make_map(&p.tw, a.w, a.M, a.K, a.ws, size, in, bn / CG) &&
            make_map(&p.to, a.out, a.n, a.M, a.os, sizeof(T), map_type<T>(), 32);
  if (a.gate) ok = ok && make_map(&p.tg, a.gate, a.n, a.M, a.gs, sizeof(T), map_type<T>(), 128);
  if (a.res) ok = ok && make_map(&p.tr, a.res, a.n, a.M, a.rs, sizeof(T), map_type<T>(), 128);
  if (!ok) return TRACKFIT_ERR_CUDA;
  p.tiles_m = (int)((a.n + 128 * CG - 1) / (128 * CG)), p.tiles_n = (a.M + bn - 1) / bn;
  p.kblocks = (a.K * size + 127) / 128, p.bn = bn, p.group = 8;
  p.slot_bytes = PIECE * (a.gate ? 2 : 1);
  const int stage_bytes = (128 + bn / CG) * 128;
  const int room = (SMEM - RESERVED - SLOTS * p.slot_bytes) / stage_bytes;
  p.stages = room < MAX_STAGES ? room : MAX_STAGES;
  // D fp32; operands of 16 bits: fp16 0, bf16 1; of 8 bits: e4m3 0
  p.idesc = idesc_f16(128 * CG, bn, !EIGHT && __is_same(T, __nv_bfloat16) ? 1u : 0u, false, false);
  p.limit_ns = operator_limit_ns(), p.expired = operator_expired();
  if (!p.expired) return TRACKFIT_ERR_CUDA;
  constexpr auto kern = product_tc_kernel<T, CG, EIGHT>;
  cudaError_t e = allow_smem<kern>(SMEM);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
  if (total > 0x3fffffff) return TRACKFIT_ERR_UNSUPPORTED;
  if constexpr (CG == 2) {
    const int pairs = resident_pairs<kern>();
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.gridDim = dim3(2 * (unsigned)(total < pairs ? total : pairs)), cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM, cfg.stream = st, cfg.attrs = &at, cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kern, p);
    if (e != cudaSuccess) return tf_status_from_cuda(e);
  } else {
    kern<<<(unsigned)(total < 152 ? total : 152), THREADS, SMEM, st>>>(p);
  }
  return launched();
}

template <class T, bool EIGHT>
int launch_split(const ProductArgs& a, int bn, int split, cudaStream_t st) {
  TcArgs p = {};
  p.a = a;
  const int size = EIGHT ? 1 : (int)sizeof(T);
  const CUtensorMapDataType in = EIGHT ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : map_type<T>();
  if (!make_map(&p.tx, a.x, a.n, a.K, a.xs, size, in, 128) || !make_map(&p.tw, a.w, a.M, a.K, a.ws, size, in, bn))
    return TRACKFIT_ERR_CUDA;
  p.tiles_m = (int)((a.n + 127) / 128), p.tiles_n = (a.M + bn - 1) / bn;
  p.kblocks = (a.K * size + 127) / 128, p.bn = bn;
  const int room = (SMEM - RESERVED - bn * 512) / ((128 + bn) * 128);
  p.stages = room < MAX_STAGES ? room : MAX_STAGES;
  p.idesc = idesc_f16(128, bn, !EIGHT && __is_same(T, __nv_bfloat16) ? 1u : 0u, false, false);
  p.limit_ns = operator_limit_ns(), p.expired = operator_expired();
  if (!p.expired) return TRACKFIT_ERR_CUDA;
  constexpr auto kern = product_split_kernel<T, EIGHT>;
  cudaError_t e = allow_smem<kern>(SMEM);
  if (e != cudaSuccess) return tf_status_from_cuda(e);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(p.tiles_m * p.tiles_n * split)), cfg.blockDim = dim3(SPLIT_THREADS);
  cfg.dynamicSmemBytes = SMEM, cfg.stream = st, cfg.attrs = &at, cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p, split);
  return e == cudaSuccess ? launched() : tf_status_from_cuda(e);
}

template <class T, bool EIGHT>
int by_tile(const ProductArgs& a, cudaStream_t st) {
  constexpr int PC = 128 / sizeof(T);
  auto tiles = [&](int rows, int bn) { return (a.n + rows - 1) / rows * ((a.M + bn - 1) / bn); };
  if (a.M > 128 && tiles(256, 256) >= 64) {
    // Pairs, where they fill the SMs.  A step of K takes as long as its rows of x and W take into the SM:
    // 128 + bn / 2 of them (8011 x 4096 x 4096: 201 us with 256 outputs, 248 with 192, whose 22 tiles do
    // little more).  The width with the least of that in all; where outputs are several tiles, of whole pieces.
    int bn = a.M <= 256 ? (a.M + 31) / 32 * 32 : 256;
    auto cost = [&](int b) { return (int64_t)((a.M + b - 1) / b) * (128 + b / 2); };
    for (int b = 192; a.M > 256 && b >= 128; b -= 64)
      if (b % PC == 0 && cost(b) < cost(bn)) bn = b;
    return launch<T, 2, EIGHT>(a, bn, st);
  }
  // Few tiles and a long K: tiles of up to 64 outputs, each by a cluster, with four steps of K a CTA at least
  // (100 x 4096 x 256: 13 us, 27 without).
  const int steps = (a.K * (EIGHT ? 1 : (int)sizeof(T)) + 127) / 128;
  const int sbn = a.M > 64 ? 64 : (a.M + 15) / 16 * 16;
  int split = 1;
  while (split < 8 && tiles(128, sbn) * split * 2 <= 152 && steps >= 8 * split) split *= 2;
  if (split > 1) return launch_split<T, EIGHT>(a, sbn, split, st);
  // a tile as wide as the outputs, up to 256; where tiles are too few for the SMs, narrower, as long as the
  // pieces of outputs stay whole
  int bn = a.M > 256 ? 256 : (a.M + 15) / 16 * 16;
  while (bn > PC && tiles(128, bn) < 152) bn = (bn / 2 + PC - 1) / PC * PC;
  return launch<T, 1, EIGHT>(a, bn, st);
}

}  // namespace

int seqops::product_tc(int32_t dtype, const ProductArgs& a, cudaStream_t st) {
  if (a.x_scales)
    return dtype == TRACKFIT_FP32 ? by_tile<float, true>(a, st)
           : dtype == TRACKFIT_BF16_PROJ ? by_tile<__nv_bfloat16, true>(a, st) : by_tile<__half, true>(a, st);
  return dtype == TRACKFIT_BF16_PROJ ? by_tile<__nv_bfloat16, false>(a, st) : by_tile<__half, false>(a, st);
}
