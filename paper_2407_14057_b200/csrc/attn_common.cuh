// Pieces shared by the tensor-core attention kernels: instruction descriptor, the score by-product's
// layout, and the few arithmetic instructions the softmax threads are written around.
#pragma once
#include "tc_common.cuh"

namespace lazy {

// kind::f16 instruction descriptor: D fp32, A/B bf16; major bits: 0 = K-major, 1 = MN-major.
__device__ __forceinline__ uint32_t idesc_bf16(int m, int n, int a_mn, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// Optional by-product: the last row's softmax numerators, for the Eq. 1 score.
// p[(seq*H + h)*max_tiles*64 + j] receives 2^(s - m_tile) for key j of the sequence,
// mtile[(seq*H + h)*max_tiles + t] the reference exponent used in tile t, stats[(seq*H + h)*2 ..] the
// final (m, 1/l).
struct AttnScoreOut {
  float *p, *mtile, *stats;
  int max_tiles, seq_id;
};

// 2^x on the special-function unit; ex2(-inf) = 0.
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Softmax weights enter a bf16 product as the sum of two bf16 numbers, P = hi + lo.  hi is cut off, not rounded, and lo = p - (1 -
// 2^-20) hi, so that lo of a weight above zero is above zero too: times an infinite value both parts then give that infinity,
// where a rounded hi would leave lo = 0 or below it and the sum NaN.  hi + lo is p (1 + 2^-20) up to 2^-16 of it (lo's
// rounding), and the products' sums are multiplied by WEIGHT_UNLIFT.  A weight below 2^-100 may have lo = 0.
constexpr float WEIGHT_REST = 1.f - 0x1p-20f, WEIGHT_LIFT = 1.f + 0x1p-20f, WEIGHT_UNLIFT = 1.f / WEIGHT_LIFT;
__device__ __forceinline__ uint32_t bf16x2_pack_rz(float lo, float hi) {
  uint32_t d;
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// Three-input maximum and two-wide fp32 arithmetic (one instruction each on this architecture): the
// softmax threads are bound by instruction issue, so halving the count of the plain ALU work matters.
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ unsigned long long f32x2_pack(float lo, float hi) {
  unsigned long long p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ void f32x2_unpack(unsigned long long p, float &lo, float &hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ unsigned long long f32x2_fma(unsigned long long a, unsigned long long b,
                                                        unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long f32x2_add(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ unsigned long long f32x2_mul(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// 2^x of two numbers on the FMA pipe, for loops that the special-function unit bounds: x = n + f with n the nearest
// integer (found by adding 1.5 2^23, which leaves n + 127 in the low bits), 2^f by a polynomial of degree 5 on
// [-1/2, 1/2], 2^n as a float with that exponent.  The constant term is 1, so that whole powers are exact; the others make
// the largest relative error small (weighted least squares on Chebyshev nodes, weights raised where the error is largest, then
// single steps of the rounded coefficients): 9.9e-8 by themselves, 1.5e-7 with the arithmetic's rounding (ex2.approx: 2.4e-7),
// -1.8e-8 on average.  x below -126 counts as -126; NaN stays NaN; x must be below 127.
__device__ __forceinline__ unsigned long long ex2_poly_x2(unsigned long long x) {
  float a, b, t0, t1;
  f32x2_unpack(x, a, b);
  asm("max.NaN.f32 %0, %1, 0fC2FC0000;" : "=f"(a) : "f"(a));  // -126
  asm("max.NaN.f32 %0, %1, 0fC2FC0000;" : "=f"(b) : "f"(b));
  x = f32x2_pack(a, b);
  const float magic = 12582912.f + 127.f;
  const unsigned long long t = f32x2_add(x, f32x2_pack(magic, magic));
  const unsigned long long n = f32x2_add(t, f32x2_pack(-magic, -magic));
  const unsigned long long f = f32x2_fma(n, f32x2_pack(-1.f, -1.f), x);
  unsigned long long p = f32x2_pack(0x1.5bba1ep-10f, 0x1.5bba1ep-10f);
  p = f32x2_fma(p, f, f32x2_pack(0x1.3cea94p-7f, 0x1.3cea94p-7f));
  p = f32x2_fma(p, f, f32x2_pack(0x1.c6b72ep-5f, 0x1.c6b72ep-5f));
  p = f32x2_fma(p, f, f32x2_pack(0x1.ebf9bep-3f, 0x1.ebf9bep-3f));
  p = f32x2_fma(p, f, f32x2_pack(0x1.62e42ap-1f, 0x1.62e42ap-1f));
  p = f32x2_fma(p, f, f32x2_pack(0x1.000000p+0f, 0x1.000000p+0f));
  f32x2_unpack(t, t0, t1);
  return f32x2_mul(p, f32x2_pack(__uint_as_float(__float_as_uint(t0) << 23), __uint_as_float(__float_as_uint(t1) << 23)));
}
// 2^x of two numbers on the special-function unit.
__device__ __forceinline__ unsigned long long ex2_approx_x2(unsigned long long x) {
  float a, b;
  f32x2_unpack(x, a, b);
  return f32x2_pack(ex2_approx(a), ex2_approx(b));
}

}  // namespace lazy
