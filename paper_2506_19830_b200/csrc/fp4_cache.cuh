// The format of the 4-bit cache, as the kernels that write and read it share it: e2m1 codes with a power-of-two scale byte for every 32
// channels of a row (include/lr_verify.h, lr_fp4_cache).
#pragma once

#include "fp8_cache.cuh"

namespace lr {

constexpr int kFp4Group = 32;             // channels that share a scale
constexpr uint32_t kFp4NanScale = 255u;   // bytes of a row that stands for NaN
constexpr int kFp4LeastScale = 1;         // 2^-126: the smallest code is 2^-1, and a byte in the exponent of an fp32 number is its scale

// A word holds the codes of channels 0 .. 7 as nibbles 0, 2, 4, 6, 1, 3, 5, 7 from the bottom: the four bits of neighbouring channels lie 16 bits apart, as two bf16
// numbers in a register do.  Nibble J of each half moves to where bf16 has its sign, the last two bits of its exponent and the first of its fraction: the two codes times
// 2^-126 (the exponent's bias is 127, e2m1's 1; 1/2 is a subnormal number in either).  One product puts a copy of the nibble at bits 6 and 12 of its half; shifting and
// masking the sign and the rest apart would take four instructions, all for the same pipe.
template <int J>
__device__ __forceinline__ uint32_t fp4_place(uint32_t w) {
  const uint32_t x = J >= 2 ? w >> 8 : w;
  return ((J & 1) != 0 ? (x & 0x00F000F0u) * 260u : (x & 0x000F000Fu) * 4160u) & 0x81C081C0u;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t twice(uint32_t bf16) { return bf16 * 0x10001u; }
// 2^(byte - 127) as two bf16 numbers, NaN for 255
__device__ __forceinline__ uint32_t fp4_scale_bf16(uint32_t byte) { return twice(byte == kFp4NanScale ? 0x7FFFu : byte == 0u ? 0x0040u : byte << 7); }

// What eight codes and their scale byte stand for, as bf16: both products are exact (numbers of 2^128 are infinities).
__device__ __forceinline__ uint4 fp4_values(uint32_t w, uint32_t byte) {
  const uint32_t up = twice(0x7E80u), s = fp4_scale_bf16(byte);  // 2^126
  return make_uint4(mul_bf16x2(mul_bf16x2(fp4_place<0>(w), up), s), mul_bf16x2(mul_bf16x2(fp4_place<1>(w), up), s),
                    mul_bf16x2(mul_bf16x2(fp4_place<2>(w), up), s), mul_bf16x2(mul_bf16x2(fp4_place<3>(w), up), s));
}

// Eight codes as fp32, in the order of their channels: exact.
__device__ __forceinline__ void fp4_floats(uint32_t w, float (&x)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // bytes 0 .. 3: channels 0 and 2, 4 and 6, 1 and 3, 5 and 7
    __half2 t;
    memcpy(&t, &h[i], 4);
    const float2 f = __half22float2(t);
    x[(i & 1) * 4 + (i >> 1)] = f.x;
    x[(i & 1) * 4 + (i >> 1) + 2] = f.y;
  }
}

// Eight numbers times a power of two (products exact) as codes: one rounding, to nearest, ties to an even code.
__device__ __forceinline__ uint32_t fp4_codes(const float *x, float by) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %3, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %7, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %4, %2;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %6;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(x[0] * by), "f"(x[1] * by), "f"(x[2] * by), "f"(x[3] * by), "f"(x[4] * by), "f"(x[5] * by), "f"(x[6] * by), "f"(x[7] * by));
  return w;
}

// The scale byte of numbers whose largest magnitude has these fp32 bits: (1 + m) 2^E, E - 2 brings it below 8, one more where that is above 6 = 1.5 x 4.
__device__ __forceinline__ int fp4_byte(uint32_t top) { return max((int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x400000u ? 1 : 0), kFp4LeastScale); }

}  // namespace lr
