// Warp-level matrix products (mma.sync) and their operands, for the operators whose pieces of
// work are a few rows long.  Lane l holds, with g = l / 4 and
// t = l % 4, of an accumulator 16 x 8: (g, 2t), (g, 2t+1), (g+8, 2t), (g+8, 2t+1).
#pragma once

#include "seq_ops.cuh"

namespace seqops {

// d += a b, 16 x 8 x 16
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d = a b
__device__ __forceinline__ void mma16_new(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma16_new(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
// d += a b, 16 x 8 x 8, operands tf32 (fp32 words whose lower 13 bits do not count).  The
// k index is free to be permuted: slot t is taken as 2t and slot t + 4 as 2t + 1, so that an
// accumulator is an operand as it stands.
__device__ __forceinline__ void mma8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                     uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// x = hi + lo, 11 bits each: products of three of the four parts keep fp32's 2^-21.  An infinity is
// all in the lower part; of a B operand it is left out (fin) where it would meet the lower part of
// A, which may be zero.
struct Parts {
  uint32_t hi, lo;
};
// The parts of a number that is not next to the largest, 11 bits each of 24: off by 2^-22 at most.
__device__ __forceinline__ Parts tf32_split(float x) {
  const uint32_t hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  return {hi, __float_as_uint(x - __uint_as_float(hi))};
}
struct BParts {
  uint32_t hi, lo, fin;
};
// The upper part is rounded by integer arithmetic (the conversion takes several times the
// instructions).  The lower one then has 12 bits, of which the product takes 11: off by 2^-22 x at
// most, and as often to one side as to the other, for it has either sign.  The upper part stays finite
// where x is next to the largest; a NaN is all in the lower part.
__device__ __forceinline__ Parts tf32_parts(float x) {
  const uint32_t u = __float_as_uint(x), m = (u + 0x1000u) & 0x7fffe000u;
  const uint32_t hi = (m < 0x7f7fe000u ? m : 0x7f7fe000u) | (u & 0x80000000u);
  return {hi, __float_as_uint(x - __uint_as_float(hi))};
}
__device__ __forceinline__ BParts tf32_bparts(float x) {
  const Parts p = tf32_parts(x);
  return {p.hi, p.lo, fabsf(x) == INFINITY ? 0u : p.hi};
}
// Where A's values are one at most, their lower parts may meet any finite number.
__device__ __forceinline__ BParts tf32_bparts_of_weighted(float x) {
  const Parts p = tf32_parts(x);
  return {p.hi, p.lo, p.hi};
}
// d += a b without the product of the lower parts
__device__ __forceinline__ void mma8_parts(float (&d)[4], const uint32_t (&ah)[4], const uint32_t (&al)[4], const BParts& b0,
                                           const BParts& b1) {
  mma8(d, al[0], al[1], al[2], al[3], b0.fin, b1.fin);
  mma8(d, ah[0], ah[1], ah[2], ah[3], b0.lo, b1.lo);
  mma8(d, ah[0], ah[1], ah[2], ah[3], b0.hi, b1.hi);
}
__device__ __forceinline__ float2 halves(uint32_t u, __nv_bfloat16) {
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ float2 halves(uint32_t u, __half) {
  __half2 h;
  *reinterpret_cast<uint32_t*>(&h) = u;
  return __half22float2(h);
}

__device__ __forceinline__ void load_shared(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_shared(uint32_t (&r)[2], uint32_t addr) {
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}
// An 8 x 8 tile of 16-bit values with rows and columns exchanged.
__device__ __forceinline__ uint32_t turned(uint32_t u) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(u));
  return d;
}
__device__ __forceinline__ void write_out(void* p, const uint32_t (&w)[4]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void write_out(void* p, const uint32_t (&w)[2]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

// sum + 0 u, both halves: zero as long as all u were finite
__device__ __forceinline__ uint32_t zero_if_finite(uint32_t u, uint32_t sum, __nv_bfloat16) {
  asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u), "r"(0u));
  return sum;
}
__device__ __forceinline__ uint32_t zero_if_finite(uint32_t u, uint32_t sum, __half) {
  asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u), "r"(0u));
  return sum;
}

}  // namespace seqops
