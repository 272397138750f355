// What the operators on packed sequences share: element types, 16-byte vectors,
// asynchronous copies of a warp's own, the search in the sequences' offsets, and the
// checks of a row array.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "trackfit_internal.h"

namespace seqops {

constexpr unsigned FULL = 0xffffffffu;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int MAX_DIM = 128;     // width of a head
constexpr int MAX_HEADS = 256;
constexpr int64_t MAX_STRIDE = (int64_t)1 << 28;   // elements: a row's bytes fit 32 bits

// ---------------------------------------------------------------- element types
__device__ __forceinline__ void unpack(const uint4& u, float (&x)[4], float) {
  x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack(const uint4& u, float (&x)[8], __nv_bfloat16) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ void unpack(const uint4& u, float (&x)[8], __half) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __half2 h;
    *reinterpret_cast<uint32_t*>(&h) = w[i];
    const float2 f = __half22float2(h);
    x[2 * i] = f.x, x[2 * i + 1] = f.y;
  }
}
// Two values rounded to nearest even; `lo` is the lower half.
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
  __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack(const float (&x)[4], float) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <class T>
__device__ __forceinline__ uint4 pack(const float (&x)[8], T t) {
  return make_uint4(pack2(x[0], x[1], t), pack2(x[2], x[3], t), pack2(x[4], x[5], t), pack2(x[6], x[7], t));
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }

// 2^x by the hardware exponential (2 ulp; results below the normal range are 0).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 values in one instruction.
__device__ __forceinline__ uint64_t both(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ float2 parts(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
// The largest of three (a NaN is passed over).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// ---------------------------------------------------------------- asynchronous copies
__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// 16 bytes global -> shared, zeros if !there (the address is not read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(there ? 8 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ---------------------------------------------------------------- offsets
__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// The first i in [0, n) with offs[i] >= row, or n: a whole warp searches, 33 parts a round.
__device__ __forceinline__ int64_t first_at_least(const int64_t* __restrict__ offs, int64_t n, int64_t row, int lane) {
  int64_t lo = 0, hi = n;   // the answer is in [lo, hi]
  while (hi > lo) {
    const int64_t step = (hi - lo + 32) / 33;
    const int64_t at = lo + (lane + 1) * step - 1;      // the last of this lane's part
    const bool below = at < hi && offs[at] < row;
    const int k = __popc(__ballot_sync(FULL, below));    // parts wholly below the row (offsets rise)
    const int64_t nlo = lo + k * step;
    const int64_t nhi = k == 32 ? hi : nlo + step - 1;
    lo = nlo < hi ? nlo : hi;
    hi = nhi < hi ? nhi : hi;
  }
  return lo;
}

// ---------------------------------------------------------------- checks of arguments
inline bool mis16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool mis4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
inline bool type_ok(int32_t dtype) {
  return dtype == TRACKFIT_FP32 || dtype == TRACKFIT_BF16_PROJ || dtype == TRACKFIT_FP16_PROJ;
}
inline int type_size(int32_t dtype) { return dtype == TRACKFIT_FP32 ? 4 : 2; }
inline bool dim_ok(int32_t d) { return d >= 8 && d <= MAX_DIM && d % 8 == 0; }
inline bool heads_ok(int32_t h) { return h >= 1 && h <= MAX_HEADS; }
// A row array [rows][stride] of `width` values a row: 16-byte aligned at every row.
inline bool rows_ok(const void* p, int64_t stride, int64_t width, int size) {
  return p && !mis16(p) && stride >= width && stride <= MAX_STRIDE && (stride * size) % 16 == 0;
}
// Dynamic shared memory beyond what any kernel may have needs leave, once a device and kernel
// (the kernel itself is the parameter: several have one type).
template <auto kernel>
inline cudaError_t allow_smem(size_t bytes) {
  static std::atomic<uint64_t> given{0};   // a bit a device
  if (bytes <= 48 * 1024) return cudaSuccess;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (given.load() & bit) return cudaSuccess;
  e = tf_allow_smem(kernel);
  if (e == cudaSuccess) given.fetch_or(bit);
  return e;
}
inline int launched() {
  const cudaError_t e = cudaPeekAtLastError();
  if (e == cudaSuccess) return TRACKFIT_OK;
  tf_note_cuda(e, "kernel launch");
  return TRACKFIT_ERR_CUDA;
}

}  // namespace seqops
