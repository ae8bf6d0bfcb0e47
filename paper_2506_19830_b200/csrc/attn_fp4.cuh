// What the two tensor-core attention kernels of the 4-bit cache share (attn_fp4.cu, attn_fp4_few.cu): codes as halves, and the rows that have to be worked out without them.
//
// One instruction turns two codes into two halves, one more multiplies them by their scale (as bf16, which a product with the queries as they are would want, a pair takes
// twice as many).  A half holds a code times 2^(byte - 127) exactly for bytes from kLeastHalf to kMostHalf, channels from 4e-7 to 49,152; what has a byte of kZeroHalf at most, below
// 2^-114, counts as zero.  A piece that has a group of another size among its valid keys, or a row of K or V that stands for NaN, has its rows gone through again
// on the CUDA cores once it is done (exact_row): any input has its result, the ones that no model gives have it some hundred times more slowly.
#pragma once

#include "attn_mma.cuh"
#include "fp4_cache.cuh"

namespace lr {

struct Fp4Call {  // of the call, what exact_row needs
  const uint16_t *q;
  const uint8_t *k, *v, *k_scale, *v_scale;
  uint16_t *out;
  float *lse, *partial_o, *partial_ml;
  const TcPage *pages;
  const TcRow *rows;
  const TcPiece *pieces;
  const TcReq *reqs;
  int64_t n_pool_pages;
  int32_t *status;
  int32_t n_q_heads, n_kv_heads, group, tokens_per_mtile;
  float scale_log2;
};

// Of a plan whose tc_most_rows is kFp4FewRows at most; without the merge.  48 requests of so many rows over 2 to 32 K keys, here and with the tile kernel, which pads rows to 128: 8 rows 130 us and
// 265, 16 rows 189 and 267 (64-wide heads 87 and 208, 120 and 208).  A third set of eight has no registers left.  The largest request of a batch decides for all of it: 48 of 5 rows take 121 us,
// with one of 15 among them 179, with one of 20 255.
constexpr int kFp4FewRows = 16;
int launch_attn_fp4_few(lr_plan *p, const Fp4Call &in, cudaStream_t s);

namespace {

constexpr uint32_t kZeroHalf = 10, kLeastHalf = 104, kMostHalf = 140;

// 2^(byte - 127) as two halves; zeros far below their range, infinities above it
__device__ __forceinline__ uint32_t half_factor(uint32_t byte) {
  uint32_t r;
  const float f = __uint_as_float(byte << 23);
  asm("cvt.rn.f16x2.f32 %0, %1, %1;" : "=r"(r) : "f"(f));
  return r;
}
__device__ __forceinline__ uint32_t half_factors(uint32_t low, uint32_t high) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(__uint_as_float(low << 23)), "f"(__uint_as_float(high << 23)));
  return r;
}
// The four bytes of a word, two codes each, times a factor: of a row's word channels 0 and 2, 4 and 6, 1 and 3, 5 and 7.
__device__ __forceinline__ void halves8(uint32_t (&h)[4], uint32_t w, uint32_t by) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t.reg .b32 x, y, z, u;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 x, a;\n\tcvt.rn.f16x2.e2m1x2 y, b;\n\tcvt.rn.f16x2.e2m1x2 z, c;\n\tcvt.rn.f16x2.e2m1x2 u, d;\n\t"
      "mul.rn.f16x2 %0, x, %5;\n\tmul.rn.f16x2 %1, y, %5;\n\tmul.rn.f16x2 %2, z, %5;\n\tmul.rn.f16x2 %3, u, %5;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w), "r"(by));
}
// four neighbouring pairs of channels in that order
__device__ __forceinline__ uint4 as_halves8(uint4 w) {
  return make_uint4(__byte_perm(w.x, w.y, 0x5410), __byte_perm(w.z, w.w, 0x5410), __byte_perm(w.x, w.y, 0x7632), __byte_perm(w.z, w.w, 0x7632));
}
// Whether one of four bytes is outside kLeastHalf .. kMostHalf.  (Below the first one that is, nothing is carried or borrowed, and that one shows.)
__device__ __forceinline__ bool any_odd_scale(uint32_t w) {
  const uint32_t d = w - 0x01010101u * kLeastHalf;
  return ((d | (d + 0x01010101u * (127u - (kMostHalf - kLeastHalf)))) & 0x80808080u) != 0u;
}
__device__ __forceinline__ bool odd_scale(uint32_t byte) { return byte > kZeroHalf && byte - kLeastHalf > kMostHalf - kLeastHalf; }

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ int2 ld_pair(const void *p) {
  int2 v;
  asm volatile("ld.global.nc.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
// past L1, as everything that reads the cache (fp8_cache.cuh)
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// What a row of Q is multiplied by to become halves: the power of two that brings its largest magnitude (bits of a bf16 number) to 2^14 .. 2^15.  Channels are then exact down to
// 2^-17, 2^-31 of the largest; a row with a smaller one that is not 0 is gone through again.  (Powers of two beyond what fp32 has: such a row is, too.)
__device__ __forceinline__ int half_exponent(uint32_t top) { return 141 - (int)(top >> 7); }
constexpr uint32_t kQMostExponent = 126;
// What a score of such a row is worth, log2 units; NaN for a row that is not finite, negative for one to be gone through again.  Products are below 2^38 (2^15 of Q, 49,152 of K, 128 channels):
// with the least normal number in place of a smaller unit scores are below 2^-88, as they would be, and those of keys that the row does not see stay -infinity, which 0 would make NaN.
__device__ __forceinline__ float score_unit(float scale_log2, int e, uint32_t top, bool odd) {
  const float unit = fmaxf(scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23), 0x1p-126f);
  return top >= 0x7F80u ? __uint_as_float(0x7FC00000u) : odd || unit == INFINITY ? -unit : unit;
}

// Row r of the M-tile that stream s of piece pc has, by a whole warp on the CUDA cores: what the tensor cores would have left for it.  32 keys at a time: a lane scores
// one, the lanes then share the value rows.  alive: told the time now and then, as this may take longer than a wait.
template <int kD>
__device__ __noinline__ void exact_row(const Fp4Call &in, int pc, int s, int r, volatile uint64_t *alive) {
  constexpr int kEach = kD / 32;  // output channels of a lane
  const TcPiece pi = in.pieces[pc];
  const TcReq rq = in.reqs[pi.req];
  DevBatch d;
  d.group = in.group;
  d.n_q_heads = in.n_q_heads;
  DevTcPlan tc;
  tc.rows = in.rows;
  const RowInfo one = row_info(d, tc, rq, in.tokens_per_mtile, pi.n_mt == 2 ? pi.mtile0 + s : pi.mtile0, r, pi.kv_head);
  const int slot = pi.slot[pi.n_mt == 2 ? s : 0];
  const int lane = threadIdx.x & 31, n_tiles = pi.tile_end - pi.tile_begin, n_dense = rq.n_dense_tiles - pi.tile_begin;
  const TcPage *pages = in.pages + rq.page_off + pi.tile_begin * kPagesPerTile;
  const uint4 *qp = reinterpret_cast<const uint4 *>(in.q + one.q_index * kD);
  float m = -INFINITY, l = 0.f, acc[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int t = 0; t < 4 * n_tiles; ++t) {  // two pages
    if (lane == 0 && alive != nullptr && (t & 63) == 0) *alive = global_ns();
    const int2 e = ld_pair(pages + 2 * t + (lane >> 4));
    const int n_ok = (t >> 2) < n_dense ? kPage : page_n_ok((uint32_t)e.y, one);
    const bool valid = (lane & 15) < n_ok;
    const unsigned live = __ballot_sync(0xFFFFFFFFu, valid);
    if (live == 0u) continue;
    // (the page named, or page 0 in its place, as for the products, which report it)
    const int64_t page = e.x >= 0 && e.x < in.n_pool_pages ? e.x : 0, at = (page * in.n_kv_heads + pi.kv_head) * kPage + (lane & 15);
    float s = -INFINITY;
    if (valid) {
      s = 0.f;
#pragma unroll 1
      for (int g = 0; g < kD / kFp4Group; ++g) {
        const uint4 kk = __ldcg(reinterpret_cast<const uint4 *>(in.k + at * (kD / 2)) + g);
        const uint32_t w[4] = {kk.x, kk.y, kk.z, kk.w};
        float a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 qa = __ldcg(qp + g * 4 + j);
          float x[8];
          fp4_floats(w[j], x);
          a0 = fmaf(bits_f(qa.x << 16), x[0], a0);
          a1 = fmaf(bits_f(qa.x & 0xFFFF0000u), x[1], a1);
          a0 = fmaf(bits_f(qa.y << 16), x[2], a0);
          a1 = fmaf(bits_f(qa.y & 0xFFFF0000u), x[3], a1);
          a0 = fmaf(bits_f(qa.z << 16), x[4], a0);
          a1 = fmaf(bits_f(qa.z & 0xFFFF0000u), x[5], a1);
          a0 = fmaf(bits_f(qa.w << 16), x[6], a0);
          a1 = fmaf(bits_f(qa.w & 0xFFFF0000u), x[7], a1);
        }
        const uint32_t vb = ld_scale(in.v_scale + at * (kD / kFp4Group) + g);
        s = fmaf(a0 + a1, fp8_scale(vb == kFp4NanScale ? kFp4NanScale : ld_scale(in.k_scale + at * (kD / kFp4Group) + g)), s);
      }
      s *= in.scale_log2;
    }
    float m_new = s;  // (a score that is no number is not the largest: it comes back through the sum)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m_new = fmaxf(m_new, __shfl_xor_sync(0xFFFFFFFFu, m_new, o));
    m_new = fmaxf(m, m_new);
    const float ref = m_new > -INFINITY ? m_new : 0.f, down = m > -INFINITY ? exp2f(m - ref) : 0.f, p = valid ? exp2f(s - ref) : 0.f;
    float sum = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    l = fmaf(l, down, sum);
    m = m_new;
#pragma unroll
    for (int e2 = 0; e2 < kEach; ++e2) acc[e2] *= down;
#pragma unroll 1
    for (unsigned left = live; left != 0u; left &= left - 1u) {
      const int j = __ffs(left) - 1;
      const float pj = __shfl_sync(0xFFFFFFFFu, p, j);
      const int64_t aj = __shfl_sync(0xFFFFFFFFu, (long long)at, j);
      // the lane's channels lane * kEach .. + kEach - 1 of their word of eight
      const uint32_t vv = __ldcg(reinterpret_cast<const uint32_t *>(in.v + aj * (kD / 2)) + lane * kEach / 8);
      const float by = pj * fp8_scale(ld_scale(in.v_scale + aj * (kD / kFp4Group) + lane * kEach / kFp4Group));
      float x[8];
      fp4_floats(vv, x);
#pragma unroll
      for (int e2 = 0; e2 < kEach; ++e2) {
        float y = x[e2];
#pragma unroll
        for (int f = kEach; f < 8; f += kEach)
          if (lane * kEach % 8 == f) y = x[f + e2];
        acc[e2] = fmaf(by, y, acc[e2]);
      }
    }
  }
  if (slot < 0) {
    const float inv = 1.0f / l;
#pragma unroll
    for (int e = 0; e < kEach; e += 2) *reinterpret_cast<uint32_t *>(in.out + one.q_index * kD + lane * kEach + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
    if (lane == 0 && in.lse != nullptr) in.lse[one.q_index] = (m + log2f(l)) * 0.6931471805599453f;
  } else {
    float *dst = in.partial_o + (((int64_t)slot * (kD / 4) + lane * kEach / 4) * 128 + r) * 4 + (lane * kEach) % 4;
#pragma unroll
    for (int e = 0; e < kEach; e += 2) *reinterpret_cast<float2 *>(dst + e) = make_float2(acc[e], acc[e + 1]);
    // a sum that is not a number must not look like that of a row that saw nothing: the merge asks whether the sum is above 0
    if (lane == 0) *reinterpret_cast<float2 *>(in.partial_ml + ((int64_t)slot * 128 + r) * 2) = l != l ? make_float2(l, 1.0f) : make_float2(m, l);
  }
}

}  // namespace

}  // namespace lr
