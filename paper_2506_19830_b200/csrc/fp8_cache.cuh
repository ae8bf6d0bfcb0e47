// The format of the 8-bit cache, as the kernels that write and read it share it: e4m3 codes with one power-of-two scale byte a row
// (include/lr_verify.h, lr_fp8_cache); and the rows of a call between a projection and a cache of 8 or 4 bits.
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

// Four numbers times a power of two as e4m3 codes.
__device__ __forceinline__ uint32_t fp8_codes(const float *x, float by) {
  uint32_t w;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(w)
      : "f"(x[0] * by), "f"(x[1] * by), "f"(x[2] * by), "f"(x[3] * by));
  return w;
}

// The scale byte of numbers whose largest magnitude has these fp32 bits: (1 + m) 2^E, E - 8 brings it below 512, one more where that is above 448 = 1.75 x 256.
__device__ __forceinline__ int fp8_byte(uint32_t top) { return max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), kFp8LeastScale); }
// 2^(127 - byte), for bytes from 1 to 253: what a row is multiplied by
__device__ __forceinline__ float scale_down(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

static_assert(kPage == 16, "slots are taken apart by shifts");

// The rows of a call that moves K and V between a projection's output and the slots of a cache.
struct CacheRows {
  const int64_t *slots;
  int64_t n_rows;      // n_tokens * heads
  int64_t n_slots;     // of the cache
  int64_t k_stride, v_stride;
  int32_t heads;
  int32_t *status;
  // a thread's token and head; a division of 64 bits, which takes as long as the rest of a thread's work, only where rows are that many
  __device__ __forceinline__ void split(int64_t row, int64_t &token, int &head) const {
    if (n_rows <= 0x7FFFFFFF) {
      const uint32_t t = (uint32_t)row / (uint32_t)heads;
      token = t;
      head = (int)((uint32_t)row - t * (uint32_t)heads);
    } else {
      token = row / heads;
      head = (int)(row - token * heads);
    }
  }
};
// The number of a token's row in a pool, (page * heads + head) * 16 + place; -1: nothing to do.  A slot beyond the cache is reported.
__device__ __forceinline__ int64_t cache_row(int64_t slot, int64_t n_slots, int32_t heads, int32_t head, int64_t token, int32_t *status) {
  if (slot >= 0 && slot < n_slots) return ((slot >> 4) * heads + head) * kPage + (slot & 15);
  if (slot >= 0 && status != nullptr) {
    status[0] = LR_EBOUNDS;
    status[1] = (int32_t)token;
  }
  return -1;
}

}  // namespace lr
