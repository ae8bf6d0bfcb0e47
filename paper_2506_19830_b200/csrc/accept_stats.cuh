// What the sampling acceptances share: the streaming pass over a row of logits that leaves, for every chunk of it, the pair (raw maximum
// M_c, S_c = sum exp((x - M_c) / T)), and how rows are cut into chunks.
#pragma once

#include "lr_common.cuh"

namespace lr {

namespace {

constexpr int kVec = 8;                       // 16-byte vectors a lane loads at a time
constexpr int kStep = 32 * kVec * 8;          // logits a warp takes at a time
constexpr int kMaxChunks = 160;               // per row

__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ float ex2_approx(float x) {  // one MUFU operation; -inf gives 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float denan(float x) { return fmaxf(x, -INFINITY); }  // NaN counts as -inf (max drops a NaN operand)

// the logits of vector vi of a row (-inf past its end)
__device__ __forceinline__ void unpack(const uint4 &v, float *x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = denan(bf_lo(w[j]));
    x[2 * j + 1] = denan(bf_hi(w[j]));
  }
}
__device__ __forceinline__ void load_tail(const uint16_t *rp, int32_t vocab, int32_t vi, float *x) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {  // ragged end of the row (vocab not a multiple of 8), or beyond it
    const int32_t e = vi * 8 + j;
    x[j] = e < vocab ? denan(bf_lo((uint32_t)rp[e])) : -INFINITY;
  }
}

__device__ __forceinline__ uint32_t max_bf2(uint32_t x, uint32_t y) {  // a NaN operand loses
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}
__device__ __forceinline__ uint4 ld_stream(const uint4 *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Where m log2(e) / T is this large nothing but a row's largest logits has any weight: two bf16 numbers that differ do so by 2^-8 of the larger at least, an exponent of
// -2^22 there.  What `off` below is rounded by is all that is left of it, and passes the range of the exponential from 2^31 on: such logits are counted, in a second
// pass over the chunk that has them.  (As a branch in the first, 4 % of its time.)
constexpr float kCold = 0x1p30f;

// The pair of a chunk, by one warp: this lane starts at vector v0 of the row rp, and the warp takes `steps` steps.  worst: the largest magnitude that `off` had.
template <bool kCounts>
__device__ __forceinline__ float2 chunk_pair_as(const uint16_t *rp, int32_t vocab, int32_t v0, int steps, float k_log2, float &worst) {
  const int32_t n_vec = vocab >> 3, rem = vocab & 7;
  constexpr uint32_t kNegInf2 = 0xFF80FF80u;
  // Of this lane's share of the chunk: the maximum, an exponent near -m * k_log2 and the sum of 2^(x * k_log2 + off).  `off` is
  // rounded at its own magnitude, which for large logits or low temperatures is far above that of the differences:
  // whatever goes from one lane or step to another is scaled by what `off` really is, not by what it stands for.
  float m = -INFINITY, off = 0.f, sum = 0.f;
  for (int st = 0; st < steps; ++st, v0 += kStep / 8) {
    uint32_t x[kVec * 4];
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const int32_t vi = v0 + k * 32;
      uint4 v = make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2);
      if (vi < n_vec) v = ld_stream(reinterpret_cast<const uint4 *>(rp) + vi);
      x[4 * k] = v.x;
      x[4 * k + 1] = v.y;
      x[4 * k + 2] = v.z;
      x[4 * k + 3] = v.w;
    }
    if (rem != 0 && v0 <= n_vec && v0 + kStep / 8 > n_vec && ((n_vec - v0) & 31) == 0) {  // this lane has the ragged end of the row
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        if (v0 + k * 32 == n_vec)
#pragma unroll
          for (int j = 0; j < 7; ++j)
            if (j < rem) {
              const uint32_t h = rp[(int64_t)n_vec * 8 + j];
              x[4 * k + (j >> 1)] = (j & 1) ? ((x[4 * k + (j >> 1)] & 0xFFFFu) | (h << 16)) : ((x[4 * k + (j >> 1)] & 0xFFFF0000u) | h);
            }
    }
    uint32_t mx = kNegInf2;
#pragma unroll
    for (int i = 0; i < kVec * 4; ++i) {
      x[i] = max_bf2(x[i], kNegInf2);  // NaN counts as -inf
      mx = max_bf2(mx, x[i]);
    }
    const float mn = fmaxf(m, fmaxf(bf_lo(mx), bf_hi(mx)));
    const float off_before = off;
    off = mn > -INFINITY ? -mn * k_log2 : 0.f;
    if (!kCounts) worst = fmaxf(worst, fabsf(off));
    if (kCounts && fabsf(off) >= kCold) {
      if (m < mn) sum = 0.f;
      m = mn;
#pragma unroll
      for (int i = 0; i < kVec * 4; ++i) sum += (bf_lo(x[i]) == mn ? 1.f : 0.f) + (bf_hi(x[i]) == mn ? 1.f : 0.f);
      continue;
    }
    float a0 = 0.f, a1 = 0.f, a2 = 0.f, a3 = 0.f;
#pragma unroll
    for (int i = 0; i < kVec * 4; i += 2) {
      a0 += ex2_approx(fmaf(bf_lo(x[i]), k_log2, off));
      a1 += ex2_approx(fmaf(bf_hi(x[i]), k_log2, off));
      a2 += ex2_approx(fmaf(bf_lo(x[i + 1]), k_log2, off));
      a3 += ex2_approx(fmaf(bf_hi(x[i + 1]), k_log2, off));
    }
    sum = fmaf(sum, m > -INFINITY ? ex2_approx(off - off_before) : 0.f, (a0 + a1) + (a2 + a3));
    m = mn;
  }
  float M = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
  float S = m > -INFINITY ? sum * ex2_approx(-fmaf(M, k_log2, off)) : 0.f;
  if (kCounts && fabsf(off) >= kCold) S = m == M ? sum : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xFFFFFFFFu, S, o);
  return make_float2(M, S);
}
__device__ __noinline__ float2 chunk_pair_cold(const uint16_t *rp, int32_t vocab, int32_t v0, int steps, float k_log2) {
  float none = 0.f;
  return chunk_pair_as<true>(rp, vocab, v0, steps, k_log2, none);
}
__device__ __forceinline__ float2 chunk_pair(const uint16_t *rp, int32_t vocab, int32_t v0, int steps, float k_log2) {
  float worst = 0.f;
  const float2 pair = chunk_pair_as<false>(rp, vocab, v0, steps, k_log2, worst);
  return __any_sync(0xFFFFFFFFu, worst >= kCold) ? chunk_pair_cold(rp, vocab, v0, steps, k_log2) : pair;
}

// steps of kStep logits per chunk
inline int chunk_steps(int32_t vocab) {
  int steps = 1;
  while ((vocab + (int64_t)steps * kStep - 1) / ((int64_t)steps * kStep) > kMaxChunks) steps *= 2;
  return steps;
}

}  // namespace

}  // namespace lr
