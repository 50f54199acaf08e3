// Whole-number weights of the draws: sums of them depend on no order.
#pragma once
#include "common.cuh"

typedef unsigned long long u64;

IPD_DEVINL u64 f2_add_rz(u64 a, u64 b) {
  u64 d;
  asm("add.rz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// w = floor(2^30 2^x + 1/2) of two x, -inf excluded (x >= -100 or so): 2^x = 2^i P(f),
// i = x rounded, f = x - i in [-1/2, 1/2], P by Horner's rule, every product and
// sum rounded to fp32 on its own; P is a least-squares fit of 2^f, relative to it, on Chebyshev
// nodes with constant term 1 (relative error below 1.9e-7 with its rounding).
// The factor 2^30 is in the coefficients (a power of two moves through the
// roundings), and the sum with 1/2 is rounded towards 0: whole numbers are fp32
// values up to 2^24 and all there is above, so that its floor is the exact sum's.
//
// The compiler contracts a packed product and sum, explicitly rounded ones too, into one
// operation.  So that every product keeps its own rounding, the sum is a product with `one`, a pair
// of 1 that the compiler does not know: there is nothing to contract.
IPD_DEVINL void pow2_weight2(u64 x, uint32_t &w0, uint32_t &w1, u64 one) {
  const float kMagic = 12582912.f;  // 1.5 * 2^23: x + kMagic rounds x to a whole number
  const u64 r = f2_fma(x, one, f2_pack(kMagic, kMagic));
  const u64 f = f2_fma(x, one, f2_sub(f2_pack(kMagic, kMagic), r));
  const float c1 = __uint_as_float(0x3f317213u) * 0x1p30f, c2 = __uint_as_float(0x3e75fcdbu) * 0x1p30f,
              c3 = __uint_as_float(0x3d635d55u) * 0x1p30f, c4 = __uint_as_float(0x3c1e760bu) * 0x1p30f,
              c5 = __uint_as_float(0x3aad4281u) * 0x1p30f;
  u64 p = f2_pack(c5, c5);
  p = f2_fma(f2_mul(p, f), one, f2_pack(c4, c4));
  p = f2_fma(f2_mul(p, f), one, f2_pack(c3, c3));
  p = f2_fma(f2_mul(p, f), one, f2_pack(c2, c2));
  p = f2_fma(f2_mul(p, f), one, f2_pack(c1, c1));
  p = f2_fma(f2_mul(p, f), one, f2_pack(0x1p30f, 0x1p30f));
  float r0, r1, p0, p1;
  f2_unpack(r, r0, r1);
  f2_unpack(p, p0, p1);
  // 2^x: i into the exponent
  const u64 y = f2_add_rz(f2_pack(__uint_as_float(__float_as_uint(p0) + (__float_as_uint(r0) << 23)),
                                  __uint_as_float(__float_as_uint(p1) + (__float_as_uint(r1) << 23))),
                          f2_pack(0.5f, 0.5f));
  float y0, y1;
  f2_unpack(y, y0, y1);
  w0 = __float2uint_rz(y0);
  w1 = __float2uint_rz(y1);
}
