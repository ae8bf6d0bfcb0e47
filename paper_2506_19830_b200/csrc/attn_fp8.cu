// Tensor-core nested-prefix attention over the 8-bit cache (head_dim 64 or 128).
//
// The plan -- page lists, tiles of 128 keys, M-tiles, pieces, partial results and their merge -- is that of attn_tc.cu, and so are the two
// streams of a CTA, the issuers and the score buffers in tensor memory.  What is different is how K and V get into shared memory and
// what the products are made of.
//
// Scores.  S = Q K^T is a product of 8-bit numbers: K goes from the cache into shared memory as it is, by TMA.  Q comes in two terms, hi = the e4m3
// numbers nearest to the row (scaled by a power of two to lie within 448) and lo = the e5m2 numbers nearest to what that leaves.  bf16 has eight bits: from 2^-6 on
// hi holds four of them and lo, whose three bits with a sign tell apart the 17 multiples of the last bit that may be left, the others, so there the two are Q itself.
// Below, they leave 2^-14 at most: 2^-21.8 of the row's largest number.  With a key's codes of 448 at most that bounds what a row's scores can be off by; a row
// where it is above kScoreTol, one with a channel a thousand times the others, is gone through again on the CUDA cores with Q as it is (exact_rows).  Both terms as
// e4m3 would leave 2^-10.  Two products at twice f16's rate take what one would.  A key's scale multiplies its column of S, before masks and maximum.
//
// Weights and V are f16.  One instruction turns two codes into two halves; a bf16 operand would take five.  Scales being powers of two, only differences
// of exponents go into a tile: with ref the largest scale byte of a half-tile's keys, a row of V enters as code * 2^(byte - ref).  That is exact for rows down to
// 2^-15 of ref's scale; below, the factor still is to 2^-24, the products are multiples of 2^-24 (of 448 at the most), and a row further down becomes zeros: 2^-24 of the
// largest number.  2^(ref - 127) itself goes into the exponent of the weights, P 2^(ref - base), where base is the stream's: the accumulator is in units of
// 2^(base - 127).  base is set one above the first ref; when a ref is more than kRise above it the accumulator is scaled down, as when the maximum
// grows; the row sums take the factor back out.  A half-tile more than kApart below base sums its weights apart, as keys whose values are all zeros
// may have any weight.  Weights lie 2^kHead above what they are; a row's reference is 2^kLift above its maximum, and a half-tile whose scores are more than 2^kGrow
// above the reference is done again: 2^15 at most, and eleven bits down to 2^-14.  Below, a weight is a multiple of 2^-24, off by 2^-25 at most.  In an output whose row
// sum is 2^-kLift, the least it can be, that is 2^(kLift - 25) x 448 x 2^(base - 127 - kHead); the largest number of V is above 224 x 2^(base - 1 - 127), so it is
// 2^(kLift - kHead - 23) of that.
//
// One CTA = 16 warps in four warpgroups, registers moved with setmaxnreg (168 x 256 + 88 x 256 = 128 x 512):
//   warps 8-11  converters, each with every fourth half-tile (64 keys): the codes of V by asynchronous copies into a buffer of the warp's own, the next
//                one's taking the place of each part as it is read; halves into the ring as the swizzled operand.  A warp has the half-tile's scale
//                bytes in one word a lane, so that ref is one reduction and a key's factor one shuffle.  Slots that hold no valid token become
//                zeros, whatever they held.  A warp also asks for K of its half-tiles, 4 boxes of a page each, and publishes the keys' scales and ref.
//   warps 13, 14  MMA issuers of stream 0 and 1 (not 12: with few queries the rows that live are those of the warps that share its quarter of the SM).
//   warps 0-3, 4-7  softmax of stream 0 and 1, one thread per query row; they also turn the rows of Q into their two terms.  A piece of one M-tile with at most
//                32 rows (single tokens, short drafts) has them in the lanes of all four warps of a stream, each of which takes 16 of a half-tile's keys;
//                their sums are joined at the end.
//
// What bounds it is neither bytes nor products but the chain of a half-tile (64 keys) through its softmax warp, 2,600 cycles where the exponentials of the two
// warps of a scheduler need 1,024: all roles share an SM's instruction cache, of which 2,048 instructions are fast, and code that runs once a
// half-tile comes at some eight cycles an instruction.  So loops are rolled, what is rare is in functions, and what runs once a piece is short.  A version
// with everything unrolled and in line, K converted to halves as well, took three times as long.
// Measured: 96 query tokens of 32 heads over 32 K keys 87 us (31 for the products), a serving batch of 16 requests 214 to 226 us (65), 8 trees of 64-wide heads 154 us (28),
// one token over 250 keys 11.7 us; 64 single tokens over 1024 keys each 84 us with head size 128 (93 without sharing the keys), 64 us with 64 (83).  Looking for rows that
// the terms of Q fall short of takes 1 to 2 % of it, 6 of the last; with every row gone through again the first takes 23 ms.
//
// A visible row that stands for NaN: K's has a scale of NaN, and with it the row's sum is.  V's becomes zeros, for a weight of 0 times NaN
// would reach rows that do not see it; the converter notes such keys per half-tile, and a row that sees one multiplies its result by NaN.
#include <cuda.h>

#include <algorithm>

#include "attn_mma.cuh"
#include "fp8_cache.cuh"

namespace lr {

namespace {

constexpr int kAtomBytes = 1024;   // 8 keys of V x 64 channels as halves, one 128-byte-swizzle atom
constexpr int kMaxK = 8, kMaxV = 8;
constexpr int kThreads = 512;
constexpr int kTeams = 4;          // converter warps, each with half-tiles of its own
// Half-tiles whose scales are published ahead of their products.  A converter writes those of half-tile x + kInfos once the stage of K that it takes is
// free, which half-tile x + kInfos - kKStages had; from x + 6 (three tiles) on, that tells that no softmax thread will look at x again: an issuer
// asks for or skips x + 6 behind the weights of its last half-tile up to x.
constexpr int kInfos = 16;
constexpr float kLift = 2.0f;      // log2: a row's reference exponent is set this much above its maximum so far,
constexpr float kGrow = 11.0f;     // log2: ... scores may rise this much above it,
constexpr float kHead = 2.0f;      // log2: ... weights are kept this much above what they are,
constexpr int kRise = 2;           // log2: ... and V's half-tiles may be this much above the accumulator's unit: 11 + 2 + 2 = 15, f16 ends at 16
constexpr int kApart = 24;         // log2: V this far below the unit has its weights summed apart
constexpr float kScoreTol = 0x1p-10f;  // log2: a row whose scores the terms of Q might put off by more is gone through again with Q as it is.  2^-10 is 7e-4 of a
                                       // weight or a log-sum, a third of what the framework's attention is held to
constexpr float kTermsLeave = 0x1p-14f;  // of a channel of Q, scaled to lie within 448: below 2^-6 at most, above nothing

template <int kD>
struct Shape {
  static_assert(kD == 64 || kD == 128, "head sizes of the tensor-core path");
  static constexpr int kHalves = kD / 64;                   // 64-channel halves of a row of V (one 128-byte swizzle line each)
  static constexpr int kTermBytes = 128 * kD;               // a term of an M-tile of Q: 128 rows of kD bytes
  static constexpr int kQBytes = 2 * kTermBytes;
  static constexpr int kCodeBytes = 64 * kD;                // a half-tile (64 keys) as it comes
  static constexpr int kGroupBytes = kHalves * kAtomBytes;  // the atoms of 8 keys of V
  static constexpr int kVBytes = 8 * kGroupBytes;           // a half-tile of V as halves: [8 groups][halves][8 keys][128 B]
  static constexpr int kKStages = kD == 128 ? 4 : 8, kVStages = kD == 128 ? 4 : 8;
  static constexpr int kCols = kD / 16;                     // lanes side by side in a row, 16 channels each
  static constexpr int kGroups = 32 / kCols;                // groups of four keys that a warp has at a time
  static constexpr int kRounds = 16 / kGroups;              // ... and how many times for a half-tile
};

struct Info {  // of a half-tile: the keys' scales, the largest scale bytes of V and of K, whether some valid row of V stands for NaN (and which: four keys a byte)
  float k_scale[64];
  int32_t v_ref, v_nan, k_ref, pad;
  uint8_t nan4[16];
};

struct Plain {  // what exact_rows needs of the call
  const uint16_t *q;
  const uint8_t *k, *v, *k_scale, *v_scale;
  uint16_t *out;
  float *lse, *partial_o, *partial_ml;
  const TcPage *pages;
  const TcRow *rows;
  const TcPiece *pieces;
  const TcReq *reqs;
  int64_t n_pool_pages;
  int32_t n_q_heads, n_kv_heads, group, tokens_per_mtile;
  float scale_log2;
};

struct __align__(16) Ctrl {
  TcCtaHead head;         // this CTA's record
  Info info[kInfos];
  uint64_t k_full[kMaxK], k_empty[kMaxK], v_full[kMaxV], v_empty[kMaxV];
  uint64_t q_full, q_empty;
  uint64_t s_full[2][2], p_full[2][2], o_done[2];  // [stream][half]
  uint64_t epi_done, drain[2];
  uint64_t join;          // stream 0's warps among each other, in pieces whose keys they share
  uint64_t xch;           // stream 1 -> stream 0: its sums are published and its accumulator is final
  uint64_t info_full[kInfos];
  uint32_t tmem_base;
  int abort_flag;
  uint64_t wait_limit_ns;
  uint64_t alive_ns;      // when a warp was last seen at work that may take longer than a wait (exact_rows)
  int32_t *status;        // the plan's
  Plain plain;
  int32_t xch_k;          // stream 1's largest scale byte of K
  float xch_m[128], xch_l[128], xch_unit[128];  // stream 1's rows, for the in-CTA combination
  // What the rows of Q were divided by and (in such units) what their terms may be off by, summed over the channels, of two pieces in turn: the queries of a piece are
  // written when both streams have asked for the last scores of the piece before, and a stream asks for its first behind the weights of the one before that, which its
  // threads had to know this for.
  float2 q_unit[2][2][128];
};
constexpr int kCtrlBytes = 11 << 10;
static_assert(sizeof(Ctrl) <= kCtrlBytes, "Ctrl must fit behind the tiles");
constexpr int kJoinRow = 36;  // floats: 32 channels of a row, and four so that rows start in different banks
constexpr int kJoinBytes = 4 * 32 * kJoinRow * 4;
template <int kD>
constexpr int kSmemBytes = 2 * Shape<kD>::kQBytes + Shape<kD>::kKStages * Shape<kD>::kCodeBytes + Shape<kD>::kVStages * Shape<kD>::kVBytes +
                           kTeams * Shape<kD>::kCodeBytes + kJoinBytes + kCtrlBytes;  // the base must be 1024-aligned
static_assert(kGrow + kHead + kRise <= 15.0f, "the largest weight as a half");
static_assert(kLift <= kHead, "what a key's part of an output may be off by, 2^-23 of the largest number of V: see above");
static_assert(kInfos - Shape<64>::kKStages >= 6 && kInfos - Shape<128>::kKStages >= 6, "see kInfos");
// A converter at position r of a ring has filled position r - kTeams, whose stage position r - kTeams - stages had been released from.  Releases are in
// order, so with no more teams than stages the release before the one it waits for has happened, and the parity of the barrier means what it
// looks for.
static_assert(kTeams <= Shape<64>::kVStages && kTeams <= Shape<128>::kVStages && kTeams <= Shape<64>::kKStages && kTeams <= Shape<128>::kKStages,
              "a converter must not be two phases of a stage ahead");
static_assert(kSmemBytes<64> <= 227 * 1024 && kSmemBytes<128> <= 227 * 1024, "shared memory per CTA");

// Instruction descriptors: D fp32, M = 128; QK: A e4m3 or e5m2 (formats 0 and 1 of kind::f8f6f4), B e4m3, N = 64 keys, both operands K-major; PV: A and B f16
// (format 0 of kind::f16), N = head size, B N-major.
constexpr uint32_t kIdescBase = (1u << 4) | (8u << 24);
constexpr uint32_t kIdescQK = kIdescBase | ((64u >> 3) << 17), kAIsE5M2 = 1u << 7;
template <int kD>
constexpr uint32_t kIdescPV = kIdescBase | (((uint32_t)kD >> 3) << 17) | (1u << 16);

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc)
      : "memory");
}
// Descriptor of a K-major operand of rows of kD bytes: the swizzle spans a row (128 or 64 bytes), groups of eight rows lie one after another.
template <int kD>
__device__ __forceinline__ uint64_t make_row_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(8 * kD >> 4) << 32) | (1ull << 46) |
         ((uint64_t)(kD == 128 ? 2 : 4) << 61);
}
// the place of 16-byte unit u of row r in such an operand
template <int kD>
__device__ __forceinline__ uint32_t row_unit(int r, int u) {
  return (uint32_t)(r * kD + ((u ^ (kD == 128 ? r & 7 : (r >> 1) & 3)) << 4));
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint64_t *bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map),
               "r"(smem_u32(bar)), "r"(x), "r"(y)
               : "memory");
}

// Five roles share an SM's instruction cache (2048 instructions of it are fast), and warps that wait for instructions are what bounds a version of this
// kernel that has everything in line: what is rare is in functions of its own, for each role (which have registers of different numbers) apart.
// The bounded wait of a whole warp (as wait_bar):
__device__ __forceinline__ bool test_bar(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0u;
}
extern __shared__ __align__(1024) unsigned char smem[];
template <int kD>
__device__ __forceinline__ Ctrl *ctrl_at() {
  return reinterpret_cast<Ctrl *>(smem + kSmemBytes<kD> - kCtrlBytes);
}
// Keeps the compiler from making a copy of a loop for each value of a condition that does not change in it.
__device__ __forceinline__ void opaque(int &x) { asm volatile("" : "+r"(x)); }

template <int kD>
__device__ __forceinline__ bool wait_long(uint32_t bar, uint32_t parity, int code) {
  Ctrl *ctrl = ctrl_at<kD>();
  uint64_t t0 = 0;
  for (uint32_t i = 0;; ++i) {
    uint32_t got;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(got)
                 : "r"(bar), "r"(parity), "r"(20000u)  // suspend for at most 20 us per try
                 : "memory");
    if (__all_sync(0xFFFFFFFFu, got != 0u)) return true;
    if (i == 0) t0 = global_ns();
    if ((i & 31u) == 31u) {
      const uint64_t since = max(t0, *reinterpret_cast<volatile uint64_t *>(&ctrl->alive_ns)), now = global_ns();
      const bool out = now > since && now - since > ctrl->wait_limit_ns;
      if (__any_sync(0xFFFFFFFFu, out || *reinterpret_cast<volatile int *>(&ctrl->abort_flag))) {
        if (out) {
          *reinterpret_cast<volatile int *>(&ctrl->abort_flag) = 1;
          ctrl->status[0] = kDevTimeout;
          ctrl->status[1] = code;
        }
        return false;
      }
    }
  }
}
template <int kD, int kRole>
__device__ __noinline__ bool wait_call(uint32_t bar, uint32_t parity, int code) { return wait_long<kD>(bar, parity, code); }
// kRole: 0 softmax, 1 the others (whose registers are fewer: a call is compiled for either), 2 within a function that is one already
template <int kD, int kRole>
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, int code) {
  const uint32_t at = smem_u32(bar);
  if (__all_sync(0xFFFFFFFFu, test_bar(at, parity))) return true;
  if constexpr (kRole == 2) return wait_long<kD>(at, parity, code);
  else return wait_call<kD, kRole>(at, parity, code);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float4 ld_shared_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ int4 ld_shared_i4(uint32_t addr) {
  int4 v;
  asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float2 fmul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ uint32_t pack_e5m2(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e5m2x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }
__device__ __forceinline__ void copy_codes(uint32_t dst, const uint8_t *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 ld_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// (asm so that these stay where they are written, tiles ahead of their use)
__device__ __forceinline__ uint32_t ld_word(const uint8_t *p) {  // four scales, as ld_scale
  uint32_t v;
  asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ int2 ld_pair(const void *p) {
  int2 v;
  asm volatile("ld.global.nc.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ void st_shared(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void st_shared2(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}

// P = exp2(t) for 64 exponents, as halves over the first half of the score buffer; returns their fp32 sum and, worked out in the shadow of the
// exponentials, the largest t.
__device__ __forceinline__ float exp_half(const uint32_t (&t)[64], uint32_t addr, float &t_max) {
  float2 acc0 = make_float2(0.f, 0.f), acc1 = make_float2(0.f, 0.f);
  float m0 = -INFINITY, m1 = -INFINITY;
  uint32_t pk[32];
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    float2 y0, y1;
    m0 = max3(m0, bits_f(t[i]), bits_f(t[i + 1]));
    y0.x = ex2(bits_f(t[i]));
    y0.y = ex2(bits_f(t[i + 1]));
    m1 = max3(m1, bits_f(t[i + 2]), bits_f(t[i + 3]));
    y1.x = ex2(bits_f(t[i + 2]));
    y1.y = ex2(bits_f(t[i + 3]));
    acc0 = fadd2(acc0, y0);
    acc1 = fadd2(acc1, y1);
    pk[i >> 1] = pack_f16(y0.x, y0.y);
    pk[(i >> 1) + 1] = pack_f16(y1.x, y1.y);
  }
  tmem_st32(addr, pk);
  t_max = fmaxf(m0, m1);
  acc0 = fadd2(acc0, acc1);
  return acc0.x + acc0.y;
}

// O *= alpha.  The PV product of the previous half-unit must have retired first; the one before it has (its commit precedes the s_full this thread has just
// seen), so o_done has completed done_needed or done_needed - 1 phases and the parity says which, whether or not this thread has looked at the
// earlier ones.
template <int kD>
__device__ __noinline__ bool rescale_rows(uint32_t o_addr, float alpha, uint64_t *o_done, uint32_t done_needed, int code) {
  if (!wait<kD, 2>(o_done, (done_needed - 1) & 1u, code)) return false;
  tc_fence_after();
#pragma unroll 1
  for (int ch = 0; ch < kD / 32; ++ch) {
    uint32_t o[32];
    tmem_ld32(o_addr + ch * 32, o);
    tc_wait_ld();
#pragma unroll
    for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(bits_f(o[c]) * alpha);
    tmem_st32(o_addr + ch * 32, o);
  }
  tc_wait_st();
  return true;
}

// Which of the 16 keys of a half-tile's page have a row of V that stands for NaN.
__device__ __forceinline__ uint32_t nan_keys(const uint8_t *nan4, int page) {
  const uint32_t w = *reinterpret_cast<const volatile uint32_t *>(nan4 + 4 * page);  // a byte of it: four keys
  return (w & 15u) | ((w >> 4) & 0xF0u) | ((w >> 8) & 0xF00u) | ((w >> 12) & 0xF000u);
}
// Whether the row sees a key of the half-tile whose row of V stands for NaN.  pages: null where it sees all keys.
__device__ __noinline__ bool sees_nan(const uint8_t *nan4, const TcPage *pages, RowInfo ri) {
  bool seen = false;
  for (int p = 0; p < kPagesPerTile / 2; ++p) {
    const uint32_t keys = nan_keys(nan4, p);
    const int n = pages != nullptr ? page_n_ok(pages[p].meta, ri) : kPage;
    seen = seen || (keys & ((1u << n) - 1u)) != 0u;
  }
  return seen;
}

// Rows r0 .. r0 + n - 1 of a tile (q_index of row r0 + i: in lane i0 + i), each scaled by a power of two to lie within 448, as their two terms, e4m3 and e5m2; 2 to the
// exponent taken out goes to unit[row], NaN for a row that is not finite (its scores are no numbers either), and beside it what the terms may leave of all its
// channels together.  The rows come by asynchronous copies into
// the place of their terms (bf16 is as long as the two) and are converted where they lie, a row's channels across lanes.  Registers for 32 rows in flight
// there are none, and with a row to a thread this took 17,000 cycles at the start of every piece, a third of a short call.
template <int kD>
__device__ __noinline__ void convert_q(const uint16_t *__restrict__ q, int64_t q_index, uint32_t tile, float2 *unit, int r0, int n, int i0) {
  constexpr int kLanes = kD / 8, kRows = 32 / kLanes;  // lanes to a row, 8 channels each; rows at a time
  const int lane = threadIdx.x & 31, sub = lane / kLanes, c = lane % kLanes;
  const uint32_t raw = tile + (r0 + sub) * kD + (c % (kLanes / 2)) * 16 + (c / (kLanes / 2)) * Shape<kD>::kTermBytes;
#pragma unroll 1
  for (int p = 0; p < n; p += kRows) {
    const int64_t index = __shfl_sync(0xFFFFFFFFu, q_index, (i0 + p + sub) & 31);
    if (p + sub < n) copy_codes(raw + p * kD, reinterpret_cast<const uint8_t *>(q + index * kD + c * 8));
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
#pragma unroll 1
  for (int p0 = 0; p0 < n; p0 += 2 * kRows) {  // two of the warp's rows (or four, or eight) at a time, for their latencies' sake
    uint32_t w[2][4], top[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int p = p0 + b * kRows;
      const uint4 x = p + sub < n ? ld_shared(raw + p * kD) : make_uint4(0, 0, 0, 0);
      w[b][0] = x.x, w[b][1] = x.y, w[b][2] = x.z, w[b][3] = x.w;
      const uint32_t t = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
      top[b] = max(t & 0xFFFFu, t >> 16);
    }
#pragma unroll
    for (int m = kLanes / 2; m > 0; m >>= 1)
#pragma unroll
      for (int b = 0; b < 2; ++b) top[b] = max(top[b], __shfl_xor_sync(0xFFFFFFFFu, top[b], m));
    __syncwarp();  // the rows have been read
    uint32_t small = 0;  // how many channels of this lane's two rows are below 2^-6 or just above: 16 bits each
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int p = p0 + b * kRows, e = min(max((int)(top[b] >> 7) - 135 + ((top[b] & 0x7Fu) > 0x60u ? 1 : 0), -126), 120);  // as lr_fp8_write
      const float by = pow2(-e);
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t w0 = w[b][2 * j], w1 = w[b][2 * j + 1];
        const float x0 = bits_f(w0 << 16) * by, x1 = bits_f(w0 & 0xFFFF0000u) * by, x2 = bits_f(w1 << 16) * by, x3 = bits_f(w1 & 0xFFFF0000u) * by;
        hi[j] = pack_e4m3(x0, x1, x2, x3);
        const float2 h0 = fp8_float2(hi[j] & 0xFFFFu), h1 = fp8_float2(hi[j] >> 16);
        lo[j] = pack_e5m2(x0 - h0.x, x1 - h0.y, x2 - h1.x, x3 - h1.y);
      }
      if (p + sub < n) {
        const uint32_t at = tile + row_unit<kD>(r0 + p + sub, c >> 1) + (c & 1) * 8;
        st_shared2(at, hi[0], hi[1]);
        st_shared2(at + Shape<kD>::kTermBytes, lo[0], lo[1]);
        if (c == 0) unit[r0 + p + sub] = make_float2(top[b] < 0x7F80u ? pow2(e) : __uint_as_float(0x7FC00000u), 0.f);
        // codes below 9, where 8 is 2^-6
        const uint32_t few0 = ~((hi[0] & 0x7F7F7F7Fu) + 0x77777777u) & 0x80808080u, few1 = ~((hi[1] & 0x7F7F7F7Fu) + 0x77777777u) & 0x80808080u;
        small += __popc(few0 | few1 >> 1) << (16 * b);
      }
    }
    if (__any_sync(0xFFFFFFFFu, small != 0u)) {
#pragma unroll
      for (int m = kLanes / 2; m > 0; m >>= 1) small += __shfl_xor_sync(0xFFFFFFFFu, small, m);
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if (c == 0 && p0 + b * kRows + sub < n) unit[r0 + p0 + b * kRows + sub].y = kTermsLeave * (float)((small >> (16 * b)) & 0xFFFFu);
    }
  }
}

// The store epilogue of a softmax thread: row r of the accumulator at o_addr times `self` (and, when the CTA's two streams worked on the same
// rows, of the other stream's at o_other times `other`) goes out as bf16 (slot < 0) or as an fp32 partial.  Not inlined: its two row
// buffers must not weigh on the register allocation of the sweep.
template <int kD>
__device__ __noinline__ void store_rows(uint32_t o_addr, uint32_t o_other, int slot, float self, float other, bool other_live, float m_out, float l_out, int r,
                                        int64_t q_index, uint16_t *__restrict__ out, float *__restrict__ lse, float *__restrict__ partial_o,
                                        float *__restrict__ partial_ml) {
  const bool any_other = __any_sync(0xFFFFFFFFu, other_live);
  if (slot < 0) {
    const float inv = 1.0f / l_out;
    self *= inv;
    other *= inv;
  }
#pragma unroll 1
  for (int ch = 0; ch < kD / 32; ++ch) {
    uint32_t o[32];
    tmem_ld32(o_addr + ch * 32, o);
    tc_wait_ld();
#pragma unroll
    for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(bits_f(o[c]) * self);
    if (any_other) {  // the loads are warp-wide; a row whose other stream saw nothing keeps its own values
      uint32_t p[32];
      tmem_ld32(o_other + ch * 32, p);
      tc_wait_ld();
      if (other_live) {
#pragma unroll
        for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(fmaf(bits_f(p[c]), other, bits_f(o[c])));
      }
    }
    if (q_index >= 0) {
      if (slot < 0) {
        uint4 *dst = reinterpret_cast<uint4 *>(out + q_index * kD + ch * 32);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          dst[j] = make_uint4(pack_bf16(bits_f(o[8 * j]), bits_f(o[8 * j + 1])), pack_bf16(bits_f(o[8 * j + 2]), bits_f(o[8 * j + 3])),
                              pack_bf16(bits_f(o[8 * j + 4]), bits_f(o[8 * j + 5])), pack_bf16(bits_f(o[8 * j + 6]), bits_f(o[8 * j + 7])));
      } else {
        // chunk-major: 16-byte chunk k of row r at [slot][k][r], so a warp's store is 512 contiguous bytes
        uint4 *dst = reinterpret_cast<uint4 *>(partial_o) + ((int64_t)slot * (kD / 4) + ch * 8) * 128 + r;
#pragma unroll
        for (int j = 0; j < 8; ++j) dst[j * 128] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
      }
    }
  }
  if (q_index < 0) return;
  if (slot >= 0) {
    // a sum that is not a number must not look like that of a row that saw nothing: the merge asks whether the sum is above 0
    const bool nan = l_out != l_out;
    *reinterpret_cast<float2 *>(partial_ml + ((int64_t)slot * 128 + r) * 2) = nan ? make_float2(l_out, 1.0f) : make_float2(m_out, l_out);
  } else if (lse != nullptr) {
    lse[q_index] = (m_out + log2f(l_out)) * 0.6931471805599453f;
  }
}

// The end of a piece whose keys the four warps of a stream have shared: row `lane` of each holds the sums over its keys (and those of stream 1).  Called by stream 0's
// warps.  m, l: the row's reference exponent and sum in this warp, joined with stream 1's.
template <int kD>
__device__ __noinline__ bool join_rows(uint32_t o_addr, uint32_t o_other, int slot, float self, float other, bool other_live, float m, float l, int quarter, int64_t q_index,
                                       uint32_t &joins, uint16_t *__restrict__ out, float *__restrict__ lse, float *__restrict__ partial_o, float *__restrict__ partial_ml) {
  Ctrl *ctrl = ctrl_at<kD>();
  const int lane = threadIdx.x & 31;
  float *part = reinterpret_cast<float *>(reinterpret_cast<unsigned char *>(ctrl) - kJoinBytes);
  const bool any_other = __any_sync(0xFFFFFFFFu, other_live);
  // (a thread's own entries of these have been read by then: stream 1's)
  ctrl->xch_m[quarter * 32 + lane] = m;
  ctrl->xch_l[quarter * 32 + lane] = l;
  mbar_arrive(&ctrl->join);
  if (!wait<kD, 2>(&ctrl->join, joins++ & 1u, 249)) return false;
  float m_all = -INFINITY, l_all = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) m_all = fmaxf(m_all, ctrl->xch_m[k * 32 + lane]);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (ctrl->xch_l[k * 32 + lane] != 0.f) l_all += ex2(ctrl->xch_m[k * 32 + lane] - m_all) * ctrl->xch_l[k * 32 + lane];  // (a warp that saw no key of the row has a sum of 0)
  const float by = l != 0.f ? ex2(m - m_all) * (slot < 0 ? 1.0f / l_all : 1.0f) : 0.f;
  self = l != 0.f ? self * by : 0.f;
  other = l != 0.f ? other * by : 0.f;
  const int row = quarter * 8 + lane / 4, c = (lane % 4) * 8;  // what this thread adds up
  const int64_t row_index = __shfl_sync(0xFFFFFFFFu, q_index, row);
#pragma unroll 1
  for (int ch = 0; ch < kD / 32; ++ch) {
    uint32_t o[32];
    tmem_ld32(o_addr + ch * 32, o);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(self != 0.f ? bits_f(o[i]) * self : 0.f);
    if (any_other) {
      uint32_t p[32];
      tmem_ld32(o_other + ch * 32, p);
      tc_wait_ld();
      if (other_live) {
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(fmaf(bits_f(p[i]), other, bits_f(o[i])));
      }
    }
    float4 *mine = reinterpret_cast<float4 *>(part + (quarter * 32 + lane) * kJoinRow);
#pragma unroll
    for (int i = 0; i < 8; ++i) mine[i] = make_float4(bits_f(o[4 * i]), bits_f(o[4 * i + 1]), bits_f(o[4 * i + 2]), bits_f(o[4 * i + 3]));
    mbar_arrive(&ctrl->join);
    if (!wait<kD, 2>(&ctrl->join, joins++ & 1u, 249)) return false;
    float t[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 *from = reinterpret_cast<const float4 *>(part + (k * 32 + row) * kJoinRow + c);
      const float4 a = from[0], b = from[1];
      const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = k == 0 ? x[i] : t[i] + x[i];
    }
    if (row_index >= 0) {
      if (slot < 0) {
        *reinterpret_cast<uint4 *>(out + row_index * kD + ch * 32 + c) =
            make_uint4(pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3]), pack_bf16(t[4], t[5]), pack_bf16(t[6], t[7]));
      } else {
        float4 *dst = reinterpret_cast<float4 *>(partial_o) + ((int64_t)slot * (kD / 4) + ch * 8 + c / 4) * 128 + row;
        dst[0] = make_float4(t[0], t[1], t[2], t[3]);
        dst[128] = make_float4(t[4], t[5], t[6], t[7]);
      }
    }
    mbar_arrive(&ctrl->join);  // before the next channels take the place of these
    if (!wait<kD, 2>(&ctrl->join, joins++ & 1u, 249)) return false;
  }
  if (quarter == 0 && q_index >= 0) {
    if (slot >= 0) {
      const bool nan = l_all != l_all;  // as in store_rows
      *reinterpret_cast<float2 *>(partial_ml + ((int64_t)slot * 128 + lane) * 2) = nan ? make_float2(l_all, 1.0f) : make_float2(m_all, l_all);
    } else if (lse != nullptr) {
      lse[q_index] = (m_all + log2f(l_all)) * 0.6931471805599453f;
    }
  }
  return true;
}

struct Fp8Pools {  // (K's codes are behind a tensor map too)
  const uint8_t *k, *v, *k_scale, *v_scale;
};

// Rows whose scores the terms of Q might put off by more than kScoreTol, one after another by a whole warp on the CUDA cores, with Q as it is: what store_rows or
// join_rows would have left for them.  rows: the lanes whose rows they are; s: the stream; split: whether four warps have the same rows.  As
// attn_fp8_generic.cu, from which it differs in the order of keys alone; that kernel has all of an SM's warps for it.
template <int kD>
__device__ __noinline__ void exact_rows(uint32_t rows, int pc, int s, bool split) {
  constexpr int kEach = kD / 32;  // output channels of a lane
  Ctrl *ctrl = ctrl_at<kD>();
  const Plain &in = ctrl->plain;
  const int lane = threadIdx.x & 31, row0 = split ? 0 : ((threadIdx.x >> 5) & 3) * 32;
  const TcPiece pi = in.pieces[pc];
  const TcReq rq = in.reqs[pi.req];
  const int n_tiles = pi.tile_end - pi.tile_begin, n_dense = rq.n_dense_tiles - pi.tile_begin, kv_head = pi.kv_head, slot = pi.slot[pi.n_mt == 2 ? s : 0];
  const TcPage *pages = in.pages + rq.page_off + pi.tile_begin * kPagesPerTile;
#pragma unroll 1
  for (; rows != 0u; rows &= rows - 1u) {
    const int i = __ffs(rows) - 1;
    DevBatch d;
    d.group = in.group;
    d.n_q_heads = in.n_q_heads;
    DevTcPlan tc;
    tc.rows = in.rows;
    const RowInfo one = row_info(d, tc, rq, in.tokens_per_mtile, pi.n_mt == 2 ? pi.mtile0 + s : pi.mtile0, row0 + i, kv_head);
    const uint4 *qp = reinterpret_cast<const uint4 *>(in.q + one.q_index * kD);
    float m = -INFINITY, l = 0.f, acc[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll 1
    for (int t = 0; t < 4 * n_tiles; ++t) {  // two pages, a key a lane
      if (lane == 0 && (t & 63) == 0) *reinterpret_cast<volatile uint64_t *>(&ctrl->alive_ns) = global_ns();
      const int2 e = ld_pair(pages + 2 * t + (lane >> 4));
      const int n_ok = (t >> 2) < n_dense ? kPage : page_n_ok((uint32_t)e.y, one);
      const bool valid = (lane & 15) < n_ok;
      const unsigned live = __ballot_sync(0xFFFFFFFFu, valid);
      if (live == 0u) continue;
      // (the page named, or page 0 in its place, as for the products)
      const int64_t page = e.x >= 0 && e.x < in.n_pool_pages ? e.x : 0, at = (page * in.n_kv_heads + kv_head) * kPage + (lane & 15);
      if (valid && page != e.x) {
        ctrl->status[0] = kDevBounds;
        ctrl->status[1] = 200;
      }
      float s = -INFINITY, vs = 0.f;
      if (valid) {
        const uint4 *kp = reinterpret_cast<const uint4 *>(in.k + at * kD);
        float a0 = 0.f, a1 = 0.f;
        uint4 code[kD / 16];
#pragma unroll
        for (int c = 0; c < kD / 16; ++c) code[c] = __ldcg(kp + c);
#pragma unroll
        for (int c = 0; c < kD / 16; ++c) {
          const uint4 kk = code[c], qa = qp[2 * c], qb = qp[2 * c + 1];
          const uint32_t w[4] = {kk.x, kk.y, kk.z, kk.w}, x[8] = {qa.x, qa.y, qa.z, qa.w, qb.x, qb.y, qb.z, qb.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 y0 = fp8_float2(w[j] & 0xFFFFu), y1 = fp8_float2(w[j] >> 16);
            a0 = fmaf(bits_f(x[2 * j] << 16), y0.x, a0);
            a1 = fmaf(bits_f(x[2 * j] & 0xFFFF0000u), y0.y, a1);
            a0 = fmaf(bits_f(x[2 * j + 1] << 16), y1.x, a0);
            a1 = fmaf(bits_f(x[2 * j + 1] & 0xFFFF0000u), y1.y, a1);
          }
        }
        s = (a0 + a1) * (fp8_scale(ld_scale(in.k_scale + at)) * in.scale_log2);
        vs = fp8_scale(ld_scale(in.v_scale + at));
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
      const float weight = valid ? p * vs : 0.f;
#pragma unroll 1
      for (int j0 = 0; j0 < 32; j0 += 8) {
        if (((live >> j0) & 0xFFu) == 0u) continue;
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // a key the row does not see: zeros, whatever is there
          const uint8_t *vp = in.v + (int64_t)__shfl_sync(0xFFFFFFFFu, (long long)at, j0 + j) * kD + lane * kEach;
          c[j] = 0u;
          if ((live >> (j0 + j)) & 1u) c[j] = kEach == 4 ? __ldcg(reinterpret_cast<const uint32_t *>(vp)) : (uint32_t)__ldcg(reinterpret_cast<const uint16_t *>(vp));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float w = __shfl_sync(0xFFFFFFFFu, weight, j0 + j);
          const float2 y = fp8_float2(c[j] & 0xFFFFu);
          acc[0] = fmaf(w, y.x, acc[0]);
          acc[1] = fmaf(w, y.y, acc[1]);
          if constexpr (kEach == 4) {
            const float2 z = fp8_float2(c[j] >> 16);
            acc[2] = fmaf(w, z.x, acc[2]);
            acc[3] = fmaf(w, z.y, acc[3]);
          }
        }
      }
    }
    if (slot < 0) {
      const float inv = 1.0f / l;
#pragma unroll
      for (int e = 0; e < kEach; e += 2)
        *reinterpret_cast<uint32_t *>(in.out + one.q_index * kD + lane * kEach + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
      if (lane == 0 && in.lse != nullptr) in.lse[one.q_index] = (m + log2f(l)) * 0.6931471805599453f;
    } else {
      const int r = row0 + i;
      float *dst = in.partial_o + (((int64_t)slot * (kD / 4) + lane * kEach / 4) * 128 + r) * 4 + (lane * kEach) % 4;
#pragma unroll
      for (int e = 0; e < kEach; e += 2) *reinterpret_cast<float2 *>(dst + e) = make_float2(acc[e], acc[e + 1]);
      if (lane == 0) *reinterpret_cast<float2 *>(in.partial_ml + ((int64_t)slot * 128 + r) * 2) = l != l ? make_float2(l, 1.0f) : make_float2(m, l);  // as in store_rows
    }
  }
}

__device__ __forceinline__ uint32_t valid_bytes(int valid, int lane) {  // of the four keys of this lane's word
  const int n = valid - (lane & 3) * 4;
  return n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}
// the largest of four scale bytes, but for those of rows that stand for NaN
__device__ __forceinline__ uint32_t top_byte(uint32_t bytes) {
  const uint32_t w = bytes & ~__vcmpeq4(bytes, 0xFFFFFFFFu), t = __vmaxu4(w, w >> 16);
  return max(t & 0xFFu, (t >> 8) & 0xFFu);
}
// 2^(byte - ref) of two keys, as halves; 0 for a row that stands for NaN
__device__ __forceinline__ uint32_t factors(uint32_t b0, uint32_t b1, int ref) {
  const float f0 = __uint_as_float((uint32_t)max((int)b0 - ref + 127, 0) << 23), f1 = __uint_as_float((uint32_t)max((int)b1 - ref + 127, 0) << 23);
  return pack_f16(b0 == kFp8NanScale ? 0.f : f0, b1 == kFp8NanScale ? 0.f : f1);
}
// four codes times a key's factor, as four halves
__device__ __forceinline__ void halves4(uint32_t c, uint32_t by, uint32_t &lo, uint32_t &hi) {
  asm("{\n\t.reg .b16 a, b;\n\t.reg .b32 x, y;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 x, a;\n\tcvt.rn.f16x2.e4m3x2 y, b;\n\tmul.rn.f16x2 %0, x, %3;\n\tmul.rn.f16x2 %1, y, %3;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(c), "r"(by));
}

// kFew: some piece has few enough rows to share its keys among the warps; the code for that costs the other pieces 2 % (instruction fetch)
template <int kD, bool kFew>
__global__ void __launch_bounds__(kThreads, 1)
attn_fp8_kernel(const __grid_constant__ CUtensorMap k_map, DevBatch d, DevTcPlan tc, const uint16_t *__restrict__ q, Fp8Pools in, uint16_t *__restrict__ out, float *__restrict__ lse,
                float scale_log2) {
  using Sh = Shape<kD>;
  constexpr int kQBytes = Sh::kQBytes, kTermBytes = Sh::kTermBytes, kCodeBytes = Sh::kCodeBytes, kVBytes = Sh::kVBytes, kGroupBytes = Sh::kGroupBytes;
  constexpr int kKStages = Sh::kKStages, kVStages = Sh::kVStages;
  if ((smem_u32(smem) & 1023u) != 0u) {  // the swizzled tiles need a 1024-byte aligned base
    if (threadIdx.x == 0) {
      d.status[0] = kDevBounds;
      d.status[1] = 260;
    }
    return;
  }
  unsigned char *q_smem = smem;                // two M-tiles
  unsigned char *k_smem = q_smem + 2 * kQBytes;  // kKStages half-tiles of codes
  unsigned char *v_smem = k_smem + kKStages * kCodeBytes;  // kVStages half-tiles of halves
  unsigned char *code_smem = v_smem + kVStages * kVBytes;  // a half-tile of V's codes for each converter
  Ctrl *ctrl = ctrl_at<kD>();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // the plan is uploaded by copies, so it may be read in front of the wait for the kernel before
  const TcCtaHead *head = tc.heads + blockIdx.x;
  const int piece0 = head->piece0, piece1 = head->piece1;
  if (warp == 8) {
    if (lane < (int)(sizeof(TcCtaHead) / 16)) reinterpret_cast<uint4 *>(&ctrl->head)[lane] = __ldg(reinterpret_cast<const uint4 *>(head) + lane);
    if (elect_one()) asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kKStages; ++s) {
      mbar_init(&ctrl->k_full[s], 1);
      mbar_init(&ctrl->k_empty[s], 2);  // one arrival per MMA issuer
    }
    for (int s = 0; s < kVStages; ++s) {
      mbar_init(&ctrl->v_full[s], 1);
      mbar_init(&ctrl->v_empty[s], 2);
    }
    mbar_init(&ctrl->q_full, 256);
    mbar_init(&ctrl->q_empty, 2);
    for (int s = 0; s < 2; ++s) {
      for (int h = 0; h < 2; ++h) {
        mbar_init(&ctrl->s_full[s][h], 1);
        mbar_init(&ctrl->p_full[s][h], 128);
      }
      mbar_init(&ctrl->o_done[s], 1);
      mbar_init(&ctrl->drain[s], 1);
    }
    mbar_init(&ctrl->epi_done, 256);
    mbar_init(&ctrl->xch, 128);
    mbar_init(&ctrl->join, 128);
    for (int i = 0; i < kInfos; ++i) mbar_init(&ctrl->info_full[i], 1);
    ctrl->abort_flag = 0;
    ctrl->alive_ns = 0;
    ctrl->wait_limit_ns = (uint64_t)tc.wait_limit_us * 1000ull;
    ctrl->status = d.status;
    fence_barrier_init();
  }
  if (threadIdx.x == 32)
    ctrl->plain = Plain{q, in.k, in.v, in.k_scale, in.v_scale, out, lse, tc.partial_o, tc.partial_ml, tc.pages, tc.rows, tc.pieces, tc.reqs, d.n_pool_pages,
                        d.n_q_heads, d.n_kv_heads, d.group, tc.tokens_per_mtile, scale_log2};
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctrl->tmem_base)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&ctrl->tmem_base);
  asm volatile("griddepcontrol.wait;" ::: "memory");  // queries and cache may come from the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const int T = tc.tokens_per_mtile;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    const TcCtaHead *head = &ctrl->head;
    // the page a table names, or page 0 in its place: never fetch outside the pool
    auto page_in_pool = [&](int32_t page) -> int32_t {
      if (page >= 0 && page < d.n_pool_pages) return page;
      d.status[0] = kDevBounds;
      d.status[1] = 200;
      return 0;
    };
    if (warp == 13 || warp == 14) {
      // ======================= MMA issuer of stream s ====================================
      // Both issuers walk every position of both rings in order: a half-tile this stream uses is consumed by its MMAs (released by a
      // tcgen05.commit), one it does not use is released with a plain arrive once it has landed.
      const int s = __shfl_sync(0xFFFFFFFFu, warp, 0) - 13;
      uint32_t base = 0, k_seen = 0, v_seen = 0, p_cnt = 0, pc_idx = 0;  // base: half-tiles of the pieces before
      bool ok = true;
      const uint32_t tmem_u = __shfl_sync(0xFFFFFFFFu, tmem, 0);
      const uint32_t s_tmem = tmem_u + s * 128, o_tmem = tmem_u + 256 + s * 128;
      // Descriptors differ from a base only in the start-address field (units of 16 bytes).
      const uint64_t qdesc0 = make_row_desc<kD>(smem_u32(q_smem)), kdesc0 = make_row_desc<kD>(smem_u32(k_smem)),
                     vdesc0 = make_desc(smem_u32(v_smem), kAtomBytes, kGroupBytes);
      auto issue_qk = [&](int m, uint32_t stage, int half) {  // S_s[half] = (hi + lo) of Q_m times K^T over 64 keys
        const uint64_t a = qdesc0 + (uint64_t)(m * (kQBytes >> 4)), b = kdesc0 + (uint64_t)(stage * (kCodeBytes >> 4));
#pragma unroll 1
        for (int term = 0; term < 2; ++term)
#pragma unroll
          for (int kk = 0; kk < kD / 32; ++kk)
            mma_f8(s_tmem + half * 64, a + (uint64_t)(term * (kTermBytes >> 4) + kk * 2), b + (uint64_t)(kk * 2), kIdescQK | (term != 0 ? kAIsE5M2 : 0u), (term | kk) != 0);
      };
      auto issue_pv = [&](uint32_t stage, int half, bool acc) {  // O_s (+)= P_s[half] V over 64 keys
        const uint64_t b = vdesc0 + (uint64_t)(stage * (kVBytes >> 4));
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
          mma_ts(o_tmem, s_tmem + half * 64 + k4 * 8, b + (uint64_t)(k4 * (2 * kGroupBytes >> 4)), kIdescPV<kD>, acc || k4 != 0);
      };
      // waits, in ring order, until position `pos` has landed; positions on the way belong to the other stream and are released here
      auto need_k = [&](uint32_t pos) -> bool {
        for (; k_seen <= pos; ++k_seen) {
          if (!wait<kD, 1>(&ctrl->k_full[k_seen % kKStages], (k_seen / kKStages) & 1u, 271)) return false;
          if (k_seen < pos && elect_one()) mbar_arrive(&ctrl->k_empty[k_seen % kKStages]);
        }
        return true;
      };
      auto need_v = [&](uint32_t pos) -> bool {
        for (; v_seen <= pos; ++v_seen) {
          if (!wait<kD, 1>(&ctrl->v_full[v_seen % kVStages], (v_seen / kVStages) & 1u, 272)) return false;
          if (v_seen < pos && elect_one()) mbar_arrive(&ctrl->v_empty[v_seen % kVStages]);
        }
        return true;
      };
      for (int pc = piece0; pc < piece1 && ok; ++pc, ++pc_idx) {
        const TcPiece *pi = pc == piece0 ? &head->first : tc.pieces + pc;
        const int n = pi->tile_end - pi->tile_begin, mode = pi->n_mt;
        const int my_units = mode == 2 ? n : (n - s + 1) / 2, step = mode == 2 ? 2 : 4;  // half-tiles from a tile of this stream to its next
        const int m_tile = mode == 2 ? s : 0;
        const uint32_t pos = base + (mode == 2 ? 0u : 2u * s);  // of the stream's first tile
        ok = wait<kD, 1>(&ctrl->q_full, pc_idx & 1u, 270);
        if (!ok) break;
        if (my_units == 0) {
          if (elect_one()) mbar_arrive(&ctrl->q_empty);
          // a stream with nothing to do here looks at the epilogue before too, so that the parity never is two phases behind
          if (pc_idx > 0) ok = wait<kD, 1>(&ctrl->epi_done, (pc_idx - 1) & 1u, 273);
        }
        // step j: O += P V of tile j, and the scores of tile j + 1 into the buffers that its weights leave; step -1 has scores alone
#pragma unroll 1
        for (int j = my_units > 0 ? -1 : 0; j < my_units && ok; ++j) {
          opaque(j);
          if (j == 0 && pc_idx > 0) {  // the epilogue of the previous piece has read O_0 and O_1
            ok = wait<kD, 1>(&ctrl->epi_done, (pc_idx - 1) & 1u, 273);
            if (!ok) break;
          }
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            opaque(j);
            const bool has_pv = j >= 0, has_qk = j + 1 < my_units;
            const uint32_t pos_v = pos + j * step + half, pos_k = pos_v + step;
            ok = (!has_pv || need_v(pos_v)) && (!has_qk || need_k(pos_k));
            if (ok && has_pv) ok = wait<kD, 1>(&ctrl->p_full[s][half], p_cnt & 1u, 274 + s);  // P of this half is in place
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              if (has_pv) {
                issue_pv(pos_v % kVStages, half, (j | half) != 0);
                tc_commit(&ctrl->o_done[s]);
                tc_commit(&ctrl->v_empty[pos_v % kVStages]);
              }
              if (has_qk) {
                issue_qk(m_tile, pos_k % kKStages, half);
                tc_commit(&ctrl->s_full[s][half]);
                tc_commit(&ctrl->k_empty[pos_k % kKStages]);
                if (half == 1 && j + 2 == my_units) tc_commit(&ctrl->q_empty);  // last QK of the piece: this stream is done with the Q buffers
              }
            }
            __syncwarp();
          }
          if (j >= 0) ++p_cnt;
        }
        if (!ok) break;
        // half-tiles of the piece behind the last of this stream
        base += 2u * (uint32_t)n;
        if (k_seen < base) {
          ok = need_k(base - 1);
          if (!ok) break;
          if (elect_one()) mbar_arrive(&ctrl->k_empty[(base - 1) % kKStages]);
        }
        if (v_seen < base) {
          ok = need_v(base - 1);
          if (!ok) break;
          if (elect_one()) mbar_arrive(&ctrl->v_empty[(base - 1) % kVStages]);
        }
      }
      if (!ok && elect_one()) {
        // let every MMA already issued retire before tensor memory is released (a commit covers what its own thread issued)
        tc_commit(&ctrl->drain[s]);
        const uint64_t t0 = global_ns();
        while (!mbar_try_wait(&ctrl->drain[s], 0))
          if (global_ns() - t0 > kDrainLimitNs) break;
      }
      __syncwarp();
    } else if (warp < 12) {
      // ======================= converters ====================================================
      constexpr int kCols = Sh::kCols, kGroups = Sh::kGroups, kRounds = Sh::kRounds;
      const int team = warp - 8;
      const int col = lane % kCols, grp = lane / kCols;  // 16 channels of keys (round * kGroups + grp) * 4 .. + 3
      // Eight neighbouring lanes store to two lines at a time whose 16-byte units lie in the same banks (both channel halves of a key, or with head size 64
      // keys four apart); half of them take their four keys in the order 1, 0, 3, 2, which brings the units of the two lines apart.
      const int odd = kD == 128 ? col >> 2 : grp & 1;
      uint32_t off[4];  // in a stage: of the first of the two units of each key
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = (grp & 1) * 4 + (j ^ odd);
        off[j] = smem_u32(v_smem) + (kD == 128 ? (col >> 2) * kAtomBytes : 0) + (grp >> 1) * kGroupBytes + r * 128 + ((((col & 3) * 2) ^ r) << 4);
      }
      const int32_t k_off = (grp & 3) * 4 * kD + col * 16;  // within the page of the keys
      // A lane alone copies and reads its part of the warp's codes, so that nothing but its own copies has to be waited for; a part
      // is asked for again as soon as it has been read, a whole half-tile's work ahead.
      const uint32_t mine = smem_u32(code_smem) + team * kCodeBytes + lane * 16;

      // the half-tiles of this warp: every kTeams-th of the CTA's
      int pc = piece0 - 1, x = team, n_half = 0, n_whole = 0, kv_head = 0;  // x: the one asked for next, its number within piece pc
      const TcPage *pages = nullptr;
      auto fetch = [&](int32_t row, int u) {  // part u of the codes of the pages with those rows
        // (a lane whose row is that of the page of this lane's keys; an absent page of the last tile reads page 0 and is cleared below)
        const uint8_t *at = in.v + k_off + (int64_t)__shfl_sync(0xFFFFFFFFu, row, ((u * kGroups + grp) >> 2) * 4) * kD;
        const uint8_t *even = at + odd * kD, *other = at - odd * kD;
        copy_codes(mine + u * 2048, even);
        copy_codes(mine + u * 2048 + 512, other + kD);
        copy_codes(mine + u * 2048 + 1024, even + 2 * kD);
        copy_codes(mine + u * 2048 + 1536, other + 3 * kD);
      };
      // Loads into registers are looked at a half-tile later: the page entries of one, the scale bytes of the one before it, whose codes of K and V are asked
      // for, and the one before that, whose V is converted.
      int2 e = make_int2(0, 0);
      int e_head = -1;                // KV head of the half-tile whose page entries are on their way, -1: there is none
      uint32_t k_word = 0, word = 0, meta = 0;  // scale bytes of keys 4 lane .. 4 lane + 3 (lanes 16-31: again) and valid tokens of their page, of the one before
      bool e_clear = false, word_clear = false;  // whether it has slots without a valid token
      bool words = false, ok = true;
      uint32_t asked = (uint32_t)team;  // ring position of K asked for next
#pragma unroll 1
      for (uint32_t ring = (uint32_t)team;;) {
        const bool there = words, clear = word_clear;
        const uint32_t live = valid_bytes((int)(meta & 31u), lane), bytes = word & live;
        words = e_head >= 0;
        int32_t row = 0;
        if (words) {
          row = (page_in_pool(e.x) * d.n_kv_heads + e_head) * kPage;  // rows of the pools are numbered within 32 bits (tc_plan_structure)
          meta = (uint32_t)e.y;
          word = ld_word(in.v_scale + row + (lane & 3) * 4);
          k_word = ld_word(in.k_scale + row + (lane & 3) * 4);
          word_clear = e_clear;
        }
        while (pc < piece1 && x >= n_half) {
          x -= n_half;
          if (++pc >= piece1) break;
          const TcPiece *pi = pc == piece0 ? &head->first : tc.pieces + pc;
          const TcReq *rq = pc == piece0 ? &head->first_req : tc.reqs + pi->req;
          n_half = 2 * (pi->tile_end - pi->tile_begin);
          n_whole = 2 * (rq->n_dense_tiles - pi->tile_begin);  // half-tiles without slots of no valid token
          kv_head = pi->kv_head;
          pages = tc.pages + rq->page_off + pi->tile_begin * kPagesPerTile + ((lane >> 2) & 3);
        }
        e_head = -1;
        if (pc < piece1) {
          e = ld_pair(pages + x * (kPagesPerTile / 2));
          e_head = kv_head;
          e_clear = x >= n_whole;
          x += kTeams;
        }
        const uint32_t stage = ring % kVStages, to = stage * kVBytes;
        uint32_t f01 = 0, f23 = 0;
        if (there) {
          const int ref = (int)max(__reduce_max_sync(0xFFFFFFFFu, top_byte(bytes)), 1u);
          // the factors of this lane's four keys, which other lanes ask for
          f01 = factors(bytes & 0xFFu, (bytes >> 8) & 0xFFu, ref);
          f23 = factors((bytes >> 16) & 0xFFu, bytes >> 24, ref);
          ok = wait<kD, 1>(&ctrl->v_empty[stage], ((ring / kVStages) & 1u) ^ 1u, 212);
          if (!ok) break;
        }
        int conv = there ? 1 : 0, ask = words ? 1 : 0, wipe = clear ? 1 : 0;
#pragma unroll 1
        for (int u = 0; u < kRounds; ++u) {
          opaque(conv);
          opaque(ask);
          opaque(wipe);
          if (conv) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRounds - 1) : "memory");
            uint4 c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = ld_shared(mine + u * 2048 + j * 512);
            const uint32_t by[2] = {__shfl_sync(0xFFFFFFFFu, f01, u * kGroups + grp), __shfl_sync(0xFFFFFFFFu, f23, u * kGroups + grp)};
            if (wipe) {
              const uint32_t l4 = __shfl_sync(0xFFFFFFFFu, live, u * kGroups + grp);
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (((l4 >> (8 * (j ^ odd))) & 1u) == 0u) c[j] = make_uint4(0, 0, 0, 0);
            }
            const uint32_t at = to + u * (kGroups / 2) * kGroupBytes;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t f = __byte_perm(by[j >> 1], 0u, ((j & 1) != 0) != (odd != 0) ? 0x3232 : 0x1010);
              uint32_t h[8];
              halves4(c[j].x, f, h[0], h[1]);
              halves4(c[j].y, f, h[2], h[3]);
              halves4(c[j].z, f, h[4], h[5]);
              halves4(c[j].w, f, h[6], h[7]);
              st_shared(off[j] + at, h[0], h[1], h[2], h[3]);
              st_shared((off[j] + at) ^ 16u, h[4], h[5], h[6], h[7]);
            }
          }
          if (ask) fetch(row, u);
          asm volatile("cp.async.commit_group;" ::: "memory");
        }
        if (there) {
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctrl->v_full[stage]);
          ring += kTeams;
        }
        if (words) {
          // K of the next half-tile, and what the softmax has to know of its keys, V's scales among it
          const uint32_t k_stage = asked % kKStages;
          ok = wait<kD, 1>(&ctrl->k_empty[k_stage], ((asked / kKStages) & 1u) ^ 1u, 210);
          if (!ok) break;
          if (lane == 0)
            mbar_arrive_expect_tx(&ctrl->k_full[k_stage], (uint32_t)kCodeBytes + ((blockIdx.x == 0 && asked == 0) ? tc.phantom_tx_bytes : 0u));
          __syncwarp();
          // one box per page, absent pages of the last tile included (page 0 in their place: nobody looks at these scores)
          if (lane < 16 && (lane & 3) == 0)
            tma_load_2d(smem_u32(k_smem) + k_stage * kCodeBytes + (lane >> 2) * (kPage * kD), &k_map, 0, row, &ctrl->k_full[k_stage]);
          Info &info = ctrl->info[asked % kInfos];
          const uint32_t now = valid_bytes((int)(meta & 31u), lane), kb = k_word & now, vb = word & now, nan = __vcmpeq4(vb, 0xFFFFFFFFu);
          const uint32_t v_ref = max(__reduce_max_sync(0xFFFFFFFFu, top_byte(vb)), 1u), k_ref = __reduce_max_sync(0xFFFFFFFFu, top_byte(kb));
          const bool any = __any_sync(0xFFFFFFFFu, nan != 0u);
          if (lane < 16) {  // (a byte of a slot without a valid token is 0 here: its scores are not looked at)
            float4 f;
            f.x = __uint_as_float((kb & 0xFFu) << 23);
            f.y = __uint_as_float((kb << 15) & 0x7F800000u);
            f.z = __uint_as_float((kb << 7) & 0x7F800000u);
            f.w = __uint_as_float((kb >> 1) & 0x7F800000u);
            reinterpret_cast<float4 *>(info.k_scale)[lane] = f;
            if (any) info.nan4[lane] = (uint8_t)((nan & 1u) | ((nan >> 7) & 2u) | ((nan >> 14) & 4u) | ((nan >> 21) & 8u));
          }
          if (lane == 0) *reinterpret_cast<int4 *>(&info.v_ref) = make_int4((int)v_ref, any ? 1 : 0, (int)k_ref, 0);
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctrl->info_full[asked % kInfos]);
          asked += kTeams;
        }
        if (!words && e_head < 0) break;
      }
      if (!ok) {
        // give the copies of K already in flight a bounded time to land before the CTA exits
        for (int back = 0; back < kKStages; ++back) {
          if (asked < (uint32_t)kTeams + (uint32_t)team) break;
          asked -= kTeams;
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(&ctrl->k_full[asked % kKStages], (asked / kKStages) & 1u))
            if (global_ns() - t0 > kDrainLimitNs) break;
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");  // (after an abort some are still on their way)
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    // ======================= softmax warpgroups ======================================
    const int s = warp >> 2;        // stream
    const int quarter = warp & 3;   // tensor-memory lane quarter this warp may access
    const int r = quarter * 32 + lane;  // row within the M-tile
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_base + s * 128, o_addr = lane_base + 256 + s * 128;
    uint32_t s_cnt = 0, o_cnt = 0;  // tiles / half-units of this stream so far
    uint32_t x_cnt = 0;             // pieces so far in which the two streams were combined
    uint32_t joins = 0;             // phases of ctrl->join so far
    uint32_t tiles = 0;             // tiles of both streams so far
    bool ok = true;
    for (int pc = piece0; pc < piece1; ++pc) {
      const TcPiece pi = pc == piece0 ? head->first : tc.pieces[pc];
      const TcReq rq = pc == piece0 ? head->first_req : tc.reqs[pi.req];
      const int n = pi.tile_end - pi.tile_begin, mode = pi.n_mt;
      const int my_units = mode == 2 ? n : (n - s + 1) / 2;
      const bool split = kFew && shares_keys(pi, rq, T, d.group);
      const RowInfo ri = row_info(d, tc, rq, T, mode == 2 ? pi.mtile0 + s : pi.mtile0, split ? lane : r, pi.kv_head);
      float sc_row = 0.f;
      if (ok) {
        // the queries, once the products of the piece before no longer read the buffers; of one M-tile each stream takes half of every warp's rows.
        // Padding is left as it is: what comes of it reaches rows that nobody reads.
        ok = wait<kD, 0>(&ctrl->q_empty, ((uint32_t)(pc - piece0) & 1u) ^ 1u, 245);
        if (ok) {
          const int live = __popc(__ballot_sync(0xFFFFFFFFu, ri.q_index >= 0)), i0 = mode == 2 ? 0 : s * 16;  // (live rows come first)
          float2 *unit = ctrl->q_unit[(pc - piece0) & 1][mode == 2 ? s : 0];
          convert_q<kD>(q, ri.q_index, smem_u32(q_smem) + (mode == 2 ? s : 0) * kQBytes, unit, quarter * 32 + i0, min(live - i0, mode == 2 ? 32 : 16), i0);
          fence_proxy_async();
          mbar_arrive(&ctrl->q_full);
          ok = wait<kD, 0>(&ctrl->q_full, (uint32_t)(pc - piece0) & 1u, 246);
          if (ok && ri.q_index >= 0) sc_row = scale_log2 * unit[r].x;
        }
      }
      if (ok && my_units > 0) {
        float m_used = -INFINITY, l = 0.f;  // the row's reference exponent and sum
        int base = 0, k_top = 0;  // k_top: the largest scale byte of K so far
        bool s_ready = false, nan_v = false;
        // A warp whose 32 rows are all padding only keeps the barriers' counts: what it leaves as weights multiplies into rows
        // of O that nobody reads.
        const bool idle = __all_sync(0xFFFFFFFFu, ri.q_index < 0);
        if (kFew && split) {  // as below, for the warp's 16 keys of a half-tile
#pragma unroll 1
          for (int u = 0; u < 2 * my_units; ++u) {
            const int j = u >> 1, half = u & 1, local = 2 * j + s, t = pi.tile_begin + local;
            const uint32_t sh_addr = s_addr + half * 64, at = (tiles + (uint32_t)local) * 2u + half, info = smem_u32(&ctrl->info[at % kInfos]), g = o_cnt + (uint32_t)u;
            if (!s_ready) {
              ok = wait<kD, 0>(&ctrl->s_full[s][half], (s_cnt + (uint32_t)j) & 1u, 230 + s) && wait<kD, 0>(&ctrl->info_full[at % kInfos], (at / kInfos) & 1u, 248);
              if (!ok) break;
            }
            tc_fence_after();
            uint32_t v[16];
            tmem_ld16(sh_addr + quarter * 16, v);
            const int4 of_v = ld_shared_i4(info + 256);
            k_top = max(k_top, of_v.z);
            const int n_ok = t >= rq.n_dense_tiles ? page_n_ok(__ldg(&tc.pages[rq.page_off + t * kPagesPerTile + half * 4 + quarter].meta), ri) : kPage;
            float alpha = 1.0f;
            bool moved = false;
            if (u == 0) base = of_v.x + 1;
            if (of_v.x > base + kRise) {
              alpha = pow2(base - (of_v.x + 1));
              base = of_v.x + 1;
              moved = true;
            }
            const int off = of_v.x - base;
            bool apart = off < -kApart;
            float bias = apart ? 0.f : (float)off + kHead, neg = m_used == -INFINITY ? 0.f : bias - m_used;
            tc_wait_ld();
            const uint32_t next = at + (half == 0 ? 1u : 3u);
            const uint32_t next_ready =
                mbar_test_wait2(&ctrl->s_full[s][half ^ 1], (s_cnt + (uint32_t)(j + half)) & 1u, &ctrl->info_full[next % kInfos], (next / kInfos) & 1u) == 3u;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 ks = ld_shared_f4(info + quarter * 64 + i * 4);
              const float2 row = make_float2(sc_row, sc_row), n2 = make_float2(neg, neg);
              const float2 t0 = ffma2(make_float2(bits_f(v[i]), bits_f(v[i + 1])), fmul2(make_float2(ks.x, ks.y), row), n2);
              const float2 t1 = ffma2(make_float2(bits_f(v[i + 2]), bits_f(v[i + 3])), fmul2(make_float2(ks.z, ks.w), row), n2);
              v[i] = __float_as_uint(n_ok > i ? t0.x : -INFINITY);
              v[i + 1] = __float_as_uint(n_ok > i + 1 ? t0.y : -INFINITY);
              v[i + 2] = __float_as_uint(n_ok > i + 2 ? t1.x : -INFINITY);
              v[i + 3] = __float_as_uint(n_ok > i + 3 ? t1.y : -INFINITY);
            }
            const uint32_t none[8] = {0, 0, 0, 0, 0, 0, 0, 0};  // the other warps' keys
#pragma unroll
            for (int k = 1; k < 4; ++k) tmem_st8(sh_addr + ((quarter + k) & 3) * 8, none);
            for (;;) {
              float t_max = max3(bits_f(v[0]), bits_f(v[1]), bits_f(v[2])), sum = 0.f;
              uint32_t pk[8];
#pragma unroll
              for (int i = 3; i < 15; i += 2) t_max = max3(t_max, bits_f(v[i]), bits_f(v[i + 1]));
              t_max = fmaxf(t_max, bits_f(v[15]));
              float2 acc = make_float2(0.f, 0.f);
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                const float2 y = make_float2(ex2(bits_f(v[i])), ex2(bits_f(v[i + 1])));
                acc = fadd2(acc, y);
                pk[i >> 1] = pack_f16(y.x, y.y);
              }
              sum = acc.x + acc.y;
              tmem_st8(sh_addr + quarter * 8, pk);
              const bool grow = t_max > kGrow + bias || (m_used == -INFINITY && t_max > -INFINITY);
              const bool grows = __any_sync(0xFFFFFFFFu, grow);
              if (!grows && !apart) {
                if (off >= -kApart) l = fmaf(sum, pow2(-off - (int)kHead), l);
                break;
              }
              float down_by = 0.f, up_by = 0.f;
              if (grows) {
                if (grow) {
                  const float to = t_max - neg + kLift;
                  if (m_used > -INFINITY) {
                    const float down = ex2(m_used - to);
                    alpha *= down;
                    l *= down;
                  }
                  m_used = to;
                  down_by = t_max;
                  up_by = bias - kLift;
                }
                moved = u != 0;
              } else {
                l += sum;
                apart = false;
                up_by = (float)off + kHead;
                bias = up_by;
              }
#pragma unroll
              for (int i = 0; i < 16; ++i) v[i] = __float_as_uint((bits_f(v[i]) - down_by) + up_by);
              tc_wait_st();
            }
            if (moved) {
              ok = rescale_rows<kD>(o_addr, alpha, &ctrl->o_done[s], g, 235 + s);
              if (!ok) break;
            }
            tc_wait_st();
            tc_fence_before();
            s_ready = __all_sync(0xFFFFFFFFu, next_ready) != 0;
            if (u + 1 == 2 * my_units) {
              ok = wait<kD, 0>(&ctrl->o_done[s], (g - 1) & 1u, 237 + s);
              if (!ok) break;
            }
            if (of_v.y) nan_v = nan_v || (nan_keys(ctrl->info[at % kInfos].nan4, quarter) & ((1u << n_ok) - 1u)) != 0u;
            mbar_arrive(&ctrl->p_full[s][half]);
          }
          s_cnt += (uint32_t)my_units;
        } else if (idle) {
          for (int u = 0; u < 2 * my_units && ok; ++u) {
            ok = wait<kD, 0>(&ctrl->s_full[s][u & 1], (s_cnt + (uint32_t)(u >> 1)) & 1u, 230 + s);
            if (ok && u + 1 == 2 * my_units) ok = wait<kD, 0>(&ctrl->o_done[s], (o_cnt + (uint32_t)u - 1) & 1u, 237 + s);
            if (ok) mbar_arrive(&ctrl->p_full[s][u & 1]);
          }
          s_cnt += (uint32_t)my_units;
        }
#pragma unroll 1
        for (int j = 0; j < my_units && ok && !idle && !split; ++j) {
          const int local = mode == 2 ? j : 2 * j + s, t = pi.tile_begin + local;
          const TcPage *pages = t >= rq.n_dense_tiles ? tc.pages + rq.page_off + t * kPagesPerTile : nullptr;
#pragma unroll 1  // one copy of the sweep: the unrolled pair is slower (instruction fetch)
          for (int half = 0; half < 2; ++half) {
            opaque(half);
            const uint32_t sh_addr = s_addr + half * 64;
            const uint32_t at = (tiles + (uint32_t)local) * 2u + half;  // half-tiles of both streams before this one
            const uint32_t info = smem_u32(&ctrl->info[at % kInfos]);
            const uint32_t g = o_cnt + (uint32_t)(2 * j + half);  // half-units of this stream before this one
            const bool first = (j | half) == 0;
            if (!s_ready) {
              // (in this order: a warp need not have looked at what the slot of `info` held before, and its parity says something only once the
              // phase before is over, as it is when the scores are there)
              ok = wait<kD, 0>(&ctrl->s_full[s][half], s_cnt & 1u, 230 + s) && wait<kD, 0>(&ctrl->info_full[at % kInfos], (at / kInfos) & 1u, 248);
              if (!ok) break;
            }
            tc_fence_after();
            uint32_t v[64];
            tmem_ld64(sh_addr, v);
            const int4 of_v = ld_shared_i4(info + 256);  // largest scale byte, whether some row stands for NaN; K's largest scale byte
            k_top = max(k_top, of_v.z);
            float alpha = 1.0f;  // what O has to be multiplied by before this half's product
            bool moved = false;  // ... in some row of the warp
            if (first) base = of_v.x + 1;
            if (of_v.x > base + kRise) {
              alpha = pow2(base - (of_v.x + 1));
              base = of_v.x + 1;
              moved = true;
            }
            const int off = of_v.x - base;
            bool apart = off < -kApart;  // values far below the accumulator's unit: the sum first, of weights as they are
            float bias = apart ? 0.f : (float)off + kHead, neg = m_used == -INFINITY ? 0.f : bias - m_used;
            tc_wait_ld();
            // the scores after these (and what is known of their keys) are looked for under the exponentials: a test costs over 100 cycles even
            // when it succeeds
            const uint32_t next = at + (half == 0 || mode == 2 ? 1u : 3u);
            const uint32_t next_ready = mbar_test_wait2(&ctrl->s_full[s][half ^ 1], (s_cnt + (uint32_t)half) & 1u, &ctrl->info_full[next % kInfos], (next / kInfos) & 1u) == 3u;
#pragma unroll
            for (int i = 0; i < 64; i += 4) {  // the exponents, in log2: score * (key's scale * row's factor) + neg
              const float4 ks = ld_shared_f4(info + i * 4);
              const float2 row = make_float2(sc_row, sc_row), n2 = make_float2(neg, neg);
              const float2 t0 = ffma2(make_float2(bits_f(v[i]), bits_f(v[i + 1])), fmul2(make_float2(ks.x, ks.y), row), n2);
              const float2 t1 = ffma2(make_float2(bits_f(v[i + 2]), bits_f(v[i + 3])), fmul2(make_float2(ks.z, ks.w), row), n2);
              v[i] = __float_as_uint(t0.x);
              v[i + 1] = __float_as_uint(t0.y);
              v[i + 2] = __float_as_uint(t1.x);
              v[i + 3] = __float_as_uint(t1.y);
            }
            if (pages != nullptr) {
              int n_ok[kPagesPerTile / 2];
#pragma unroll
              for (int p = 0; p < kPagesPerTile / 2; ++p) n_ok[p] = page_n_ok(__ldg(&pages[half * 4 + p].meta), ri);
              mask_half(v, n_ok);
            }
            for (;;) {  // three times at most: a row's reference moves once, the sum apart is taken once
              float t_max;
              const float sum = exp_half(v, sh_addr, t_max);
              // beyond what a half holds, or a row's first keys: again, with the reference moved
              const bool grow = t_max > kGrow + bias || (m_used == -INFINITY && t_max > -INFINITY);
              const bool grows = __any_sync(0xFFFFFFFFu, grow);
              if (!grows && !apart) {
                if (off >= -kApart) l = fmaf(sum, pow2(-off - (int)kHead), l);
                break;
              }
              float down_by = 0.f, up_by = 0.f;  // in two steps: the first leaves exactly 0 at the largest, however large that was, so that this ends
              if (grows) {
                if (grow) {
                  const float to = t_max - neg + kLift;
                  if (m_used > -INFINITY) {
                    const float down = ex2(m_used - to);
                    alpha *= down;
                    l *= down;
                  }
                  m_used = to;
                  down_by = t_max;
                  up_by = bias - kLift;
                }
                moved = !first;
              } else {
                l += sum;
                apart = false;
                up_by = (float)off + kHead;
                bias = up_by;
              }
#pragma unroll
              for (int i = 0; i < 64; i += 2) {
                const float2 t = fadd2(fadd2(make_float2(bits_f(v[i]), bits_f(v[i + 1])), make_float2(-down_by, -down_by)), make_float2(up_by, up_by));
                v[i] = __float_as_uint(t.x);
                v[i + 1] = __float_as_uint(t.y);
              }
              tc_wait_st();
            }
            if (moved) {
              ok = rescale_rows<kD>(o_addr, alpha, &ctrl->o_done[s], g, 235 + s);
              if (!ok) break;
            }
            tc_wait_st();
            tc_fence_before();
            s_ready = __all_sync(0xFFFFFFFFu, next_ready) != 0;
            // The wait at the end must not find o_done two phases back (one parity for both): the last arrive comes
            // after the product before has been seen to retire.
            if (half == 1 && j + 1 == my_units) {
              ok = wait<kD, 0>(&ctrl->o_done[s], (g - 1) & 1u, 237 + s);
              if (!ok) break;
            }
            // (before the arrival: what it looks at may be replaced behind it)
            if (of_v.y) nan_v = sees_nan(ctrl->info[at % kInfos].nan4, pages == nullptr ? nullptr : pages + half * 4, ri) || nan_v;
            mbar_arrive(&ctrl->p_full[s][half]);
          }
          ++s_cnt;
        }
        if (ok) {
          // epilogue: wait for the last PV of this stream, then normalise and store
          o_cnt += 2u * (uint32_t)my_units;
          ok = wait<kD, 0>(&ctrl->o_done[s], (o_cnt - 1) & 1u, 240 + s);
        }
        // what the accumulator's numbers are worth; NaN for a row that sees a row of V that is
        const float unit = nan_v ? __uint_as_float(0x7FC00000u) : exp2f((float)(base - 127) - kHead);
        // The two streams of a one-M-tile piece hold partial results of the same rows (even and odd tiles).
        // Stream 1 publishes its sums; stream 0 reads them and stream 1's accumulator -- the same tensor-memory
        // lanes, so the thread of row r can load both -- and writes one combined result.
        const bool pair = mode == 1 && n >= 2;
        float m_out = m_used, l_out = l, self = unit, other = 0.0f;
        bool writer = true, other_live = false;
        if (ok && pair) {
          if (s == 1) {
            ctrl->xch_m[r] = m_used;
            ctrl->xch_l[r] = l;
            ctrl->xch_unit[r] = unit;
            if (r == 0) ctrl->xch_k = k_top;
            tc_fence_before();
            mbar_arrive(&ctrl->xch);
            writer = false;
          } else {
            ok = wait<kD, 0>(&ctrl->xch, x_cnt & 1u, 242);
            if (ok) {
              tc_fence_after();
              const float om = ctrl->xch_m[r], ol = ctrl->xch_l[r];
              other_live = ol != 0.f;  // a stream that saw no key of the row has a sum of 0
              m_out = fmaxf(m_used, om);
              const float w_self = l != 0.f ? ex2(m_used - m_out) : 0.f, w_other = other_live ? ex2(om - m_out) : 0.f;
              self = l != 0.f ? unit * w_self : 0.f;
              other = other_live ? ctrl->xch_unit[r] * w_other : 0.f;
              l_out = w_self * l + w_other * ol;
              k_top = max(k_top, ctrl->xch_k);
            }
          }
        }
        if (pair) ++x_cnt;
        // A key's codes are 448 at most: no score of the row is off by more than this.  (What the terms leave is looked up here: one more register through the sweep, or
        // more for exact_rows to be given, costs short pieces 5 %.)
        uint32_t again = __ballot_sync(0xFFFFFFFFu, writer && ri.q_index >= 0 &&
                                                        sc_row * ctrl->q_unit[(pc - piece0) & 1][mode == 2 ? s : 0][r].y * 448.0f * pow2(k_top - 127) > kScoreTol);
        const int64_t q_index = (again >> lane) & 1u ? -1 : ri.q_index;
        if (kFew && ok && writer && split) {
          tc_fence_after();
          ok = join_rows<kD>(o_addr, lane_base + 256 + 128, pi.slot[0], self, other, other_live, m_out, l_out, quarter, q_index, joins, out, lse, tc.partial_o, tc.partial_ml);
          tc_fence_before();
        } else if (ok && writer && !idle) {
          tc_fence_after();
          store_rows<kD>(o_addr, lane_base + 256 + (1 - s) * 128, pi.slot[pair ? 0 : s], self, other, other_live, m_out, l_out, r, q_index, out, lse,
                         tc.partial_o, tc.partial_ml);
          tc_fence_before();
        }
        if (split) again &= 0x11111111u << quarter;  // the four warps have the same rows
        if (ok && writer && again != 0u) exact_rows<kD>(again, pc, s, split);
      }
      // One arrival per thread and piece.  A stream with units in this piece cannot get here before the previous
      // piece's phase is complete (its PV products were issued behind a wait for it); a stream with none must look
      // itself, or its arrival would be counted into the previous phase while the other stream is still storing.
      if (my_units == 0 && pc > piece0 && ok) ok = wait<kD, 0>(&ctrl->epi_done, (uint32_t)(pc - piece0 - 1) & 1u, 243);
      mbar_arrive(&ctrl->epi_done);
      tiles += (uint32_t)n;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

template <int kD, int kBatch>
__global__ void __launch_bounds__(256, kMergeCtas<kBatch>)
attn_fp8_merge_kernel(DevBatch d, DevTcPlan tc, uint16_t *__restrict__ out, float *__restrict__ lse) {
  merge_cta<kD, kBatch>(d, tc, blockIdx.x, blockIdx.y, out, lse);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// K's codes as rows of head_dim bytes; a box is one page of one KV head, 16 rows.  Made for every call: it takes a fraction of a microsecond.
int encode_k(lr_ctx *ctx, const void *codes, int64_t n_pages, CUtensorMap *map) {
  if (!ctx->tmap_encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn) {
      set_error("cuTensorMapEncodeTiled is not available from the driver");
      return LR_ECUDA;
    }
    ctx->tmap_encode = fn;
  }
  const lr_model &m = ctx->model;
  const cuuint64_t dims[2] = {(cuuint64_t)m.head_dim, (cuuint64_t)n_pages * m.n_kv_heads * kPage}, strides[1] = {(cuuint64_t)m.head_dim};
  const cuuint32_t box[2] = {(cuuint32_t)m.head_dim, kPage}, estr[2] = {1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->tmap_encode)(
      map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(codes), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
      m.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_error("cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
    return LR_ECUDA;
  }
  return LR_OK;
}

template <int kD>
int launch(lr_plan *p, const CUtensorMap &k_map, const uint16_t *q, const Fp8Pools &in, uint16_t *out, float *lse, float scale_log2, cudaStream_t s) {
  const DevTcPlan &tc = p->tc;
  p->ctx->launches++;
  if (int rc = cuda_fail(launch_dependent(p->tc_few_rows ? attn_fp8_kernel<kD, true> : attn_fp8_kernel<kD, false>, dim3((unsigned)tc.n_cta), dim3(kThreads), kSmemBytes<kD>, s, k_map, p->dev, tc, q, in, out,
                                          lse, scale_log2),
                         "attn_fp8_kernel launch"))
    return rc;
  if (tc.n_targets == 0) return LR_OK;
  p->ctx->launches++;  // the merge grid is set up while the attention grid drains
  return cuda_fail(launch_dependent(tc.most_slots <= 4 ? attn_fp8_merge_kernel<kD, 4> : attn_fp8_merge_kernel<kD, 8>, dim3((unsigned)tc.n_targets, kD / 8),
                                    dim3(256), 0, s, p->dev, tc, out, lse),
                   "attn_fp8_merge_kernel launch");
}

}  // namespace

int init_attn_fp8_kernel() {
  cudaError_t e = cudaFuncSetAttribute(attn_fp8_kernel<128, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes<128>);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_fp8_kernel<128, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes<128>);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_fp8_kernel<64, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes<64>);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_fp8_kernel<64, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes<64>);
  return cuda_fail(e, "attn_fp8_kernel shared-memory attribute");
}

int launch_attn_fp8(lr_plan *p, const void *q, const lr_fp8_cache &c, void *out, float *lse, float scale, cudaStream_t s) {
  alignas(64) CUtensorMap k_map;
  if (int rc = encode_k(p->ctx, c.k_d, p->dev.n_pool_pages, &k_map)) return rc;
  const Fp8Pools in = {reinterpret_cast<const uint8_t *>(c.k_d), reinterpret_cast<const uint8_t *>(c.v_d), c.k_scale_d, c.v_scale_d};
  return (p->dev.head_dim == 128 ? launch<128> : launch<64>)(p, k_map, reinterpret_cast<const uint16_t *>(q), in, reinterpret_cast<uint16_t *>(out), lse,
                                                             scale * 1.4426950408889634f, s);
}

}  // namespace lr
