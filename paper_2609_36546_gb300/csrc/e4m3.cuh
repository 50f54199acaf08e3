// 8-bit values (OCP FP8 E4M3) and power-of-two scales (E8M0) of the 8-bit cache.
#pragma once
#include "common.cuh"

// 2^n as fp32: exact from n = -149 on, 0 below, +inf from 128 on.
IPD_DEVINL float pow2i(int n) {
  if (n >= -126) return n > 127 ? __uint_as_float(0x7f800000u) : __uint_as_float((uint32_t)(n + 127) << 23);
  return n >= -149 ? __uint_as_float(1u << (n + 149)) : 0.f;
}

// What a scale byte stands for, times 2^n.
IPD_DEVINL float e8m0(uint32_t b, int n = 0) {
  return b == 255u ? __uint_as_float(0x7fc00000u) : pow2i((int)b - 127 + n);
}

// Two fp32 values as e4m3 (to nearest even; |x| over 448 becomes 448, NaN stays): lo in bits 0-7.
IPD_DEVINL uint32_t e4m3x2(float lo, float hi) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
  return d;
}
// Two e4m3 values (bits 0-15) as fp16: exact.
IPD_DEVINL uint32_t h2_from_e4m3x2(uint32_t v) {
  uint32_t d;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((uint16_t)v));
  return d;
}
IPD_DEVINL void h2_to_floats(uint32_t h2, float &lo, float &hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(lo), "=f"(hi)
      : "r"(h2));
}
// Four e4m3 values as fp32.
IPD_DEVINL void e4m3x4_to_floats(uint32_t v, float (&f)[4]) {
  h2_to_floats(h2_from_e4m3x2(v & 0xffffu), f[0], f[1]);
  h2_to_floats(h2_from_e4m3x2(v >> 16), f[2], f[3]);
}
