// The format of the 8-bit cache, as the kernels that write and read it share it: e4m3 codes with one power-of-two scale byte a row
// (include/lr_verify.h, lr_fp8_cache).
#pragma once

#include <cuda_fp16.h>

#include "lr_common.cuh"

namespace lr {

constexpr uint32_t kFp8NanScale = 255u;  // byte of a row that stands for NaN
constexpr int kFp8LeastScale = 3;        // 2^-124: the smallest code is 2^-9, and bf16 ends at 2^-133

// 2^(byte - 127), NaN for 255
__device__ __forceinline__ float fp8_scale(uint32_t byte) {
  return __uint_as_float(byte == kFp8NanScale ? 0x7FC00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// What a kernel reads of the cache it reads from L2 (this, __ldcg, copies that pass L1 by), whichever kernel it is.  Its blocks are there before the kernel in front of
// it has ended, which may be the one that writes the rows: the read-only path is for what does not change while a grid lives.  And 32 bytes of scales hold
// those of two heads, or of two pages, which may be another sequence's: a kernel on another stream may have brought them into this SM's L1 before they were written.
__device__ __forceinline__ uint32_t ld_scale(const uint8_t *p) {
  uint32_t v;
  asm volatile("ld.global.cg.u8 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}

// two e4m3 codes (low byte first) as halves: exact
__device__ __forceinline__ uint32_t fp8_half2(uint32_t two) {
  uint32_t h;
  asm("{\n\t.reg .b16 c;\n\tcvt.u16.u32 c, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, c;\n\t}" : "=r"(h) : "r"(two));
  return h;
}

__device__ __forceinline__ float2 fp8_float2(uint32_t two) {
  const uint32_t h = fp8_half2(two);
  __half2 t;
  memcpy(&t, &h, 4);
  return __half22float2(t);
}

}  // namespace lr
