// Tensor-core nested-prefix attention over the 4-bit cache (head_dim 64 or 128).
//
// The plan, the two streams of a CTA, the ring of tiles and what the issuers and the softmax threads do are those of attn_tc.cu.  What is different is how K and V get
// into the ring: one warp brings codes and scales from the cache, four turn them into halves and store those as the operands.
//
// Numbers.  Q, K, V and the weights are halves (attn_fp4.cuh): a code and its scale are one exactly, two instructions for a pair of codes, where bf16 takes twice as many and the
// converters, one warp to a scheduler, are what a tile waits for.  A row of Q is scaled by a power of two, which the softmax takes out again; eight channels of K
// and Q lie in the order in which the bytes of a word give them, those of O are put right as they are stored.  Weights lie 2^kLift above what they are when the row's
// reference is set, and may rise to 2^15: off by 2^-12 of themselves, or by 2^-25 where they are below 2^-14, 2^-27 of the weight that set it.  Rows that this
// does not serve are worked out once more when their piece is done (exact_row).  Slots that hold no valid token become zeros, whatever they held.
//
// One CTA = 16 warps in four warpgroups, registers moved with setmaxnreg (184 x 256 + 72 x 256 = 128 x 512):
//   warps 8-11  converters, a quarter of every tile each (two pages, 32 keys).  A lane has the 16 bytes of one group of a key at a time, 32 channels with one scale, and stores
//               four 16-byte units of the swizzled operand; lanes are dealt to keys and groups so that eight neighbours' loads and stores lie in different banks.
//   warp 15     brings codes and scales into shared memory, kRaw tiles ahead, by asynchronous copies of 16 bytes.
//   warp 12     brings the queries, by TMA; the softmax threads turn them into halves where they lie, a row each.
//   warps 13, 14  MMA issuers of stream 0 and 1.
//   warps 0-3, 4-7  softmax of stream 0 and 1, one thread per query row.
//
// What bounds it, in cycles of a half-unit (64 keys of either stream).  96 query tokens over 32 K keys (68 us): 1460 of a softmax warp, in which the exponentials of the two warps that share
// a unit take 1024, and 390 of waiting: products at N = 64 read Q's tile again for every half, which with the converters' stores is, by count, three quarters of what shared memory gives (no counter at hand has
// the products' reads: those of loads and stores show 25 to 29 %).  16 requests over 8 to
// 32 K keys (172 us), whose pieces have one M-tile: converters, 1010 a tile, two of them a half-unit (twice the warps do not help: their stores
// and the products' reads share a memory); without them it would take 161.  64-wide heads: the softmax, 1540 of 1710.
#include <cuda.h>

#include <algorithm>

#include "attn_fp4.cuh"

namespace lr {

namespace {

constexpr int kHalfBytes = 16384;  // 128 rows or keys x 64 channels
constexpr int kAtomBytes = 1024;   // K/V tiles: 8 keys x 64 channels, one 128-byte-swizzle atom
constexpr int kMaxStages = 8;
constexpr int kThreads = 512;
constexpr int kTeams = 4;          // converter warps
constexpr int kKeys = 128 / kTeams;  // of a tile, that a warp converts

template <int kD>
struct Shape {
  static_assert(kD == 64 || kD == 128, "head sizes of the tensor-core path");
  static constexpr int kHalves = kD / 64;                 // 64-channel halves of a row (one 128-byte swizzle line each)
  static constexpr int kTileBytes = kHalves * kHalfBytes; // [halves][128 rows][128 B] for Q, [16 groups][halves][8 keys][128 B] for K/V
  static constexpr int kGroupBytes = kHalves * kAtomBytes;  // the atoms of one 8-key group
  static constexpr int kStages = kD == 128 ? 4 : 8;
  static constexpr int kRaw = kD == 128 ? 3 : 6;          // tiles of codes on their way or being converted
  static constexpr int kScales = kD / kFp4Group;          // scale bytes of a row
  static constexpr int kPasses = kD / 32;                 // 16-byte groups of a lane in a tile
  // ... whose codes are asked for at once: 178 us where one at a time takes 188 (16 requests over 8 to 32 K keys, with the launch); with two passes, of head size 64, one is 1% faster
  static constexpr int kBatch = kD == 128 ? 2 : 1;
  static constexpr int kPassKeys = kKeys / kPasses;
  static constexpr int kCodeBytes = 128 * kD / 2, kScaleBytes = 128 * kScales;
  static constexpr int kSlotBytes = kCodeBytes + kScaleBytes + 32;  // of a tile: codes, scales, valid tokens of its pages
  static constexpr int kRawBytes = kRaw * kSlotBytes;
  static constexpr int kSmemBytes = 2 * kTileBytes + kStages * kTileBytes + kRawBytes + 4096;  // tiles, codes, Ctrl; the base must be 1024-aligned
};
constexpr int kMaxRaw = 6;
// Marks of pieces with a scale beyond halves, of as many pieces in turn as may be under way.  Softmax threads read that of a piece at its end, and until all of them have, no issuer
// starts on the next (q_full).  So the ring ends kStages positions behind the piece, two of which are the least that one takes: converters are kStages / 2 pieces ahead at most.
constexpr int kMarks = 8;
static_assert((kMarks & (kMarks - 1)) == 0 && kMarks > Shape<64>::kStages / 2 && kMarks > Shape<128>::kStages / 2, "a mark is read before its place is another piece's");
constexpr float kLift = 2.0f;   // log2 units: a row's reference is set this much below its maximum so far; the more, the smaller the weights that are more than 0,
constexpr float kGrow = 15.0f;  // ... and keys beyond this are done again with another one: halves end at 2^16

struct __align__(16) Ctrl {
  TcCtaHead head;         // this CTA's record
  uint64_t kv_full[kMaxStages], kv_empty[kMaxStages];
  uint64_t q_full, q_empty;
  uint64_t s_full[2][2], p_full[2][2], o_done[2];  // [stream][half]
  uint64_t epi_done, drain[2];
  uint64_t xch;           // stream 1 -> stream 0: its (m, l) are published and its accumulator is final
  uint32_t tmem_base;
  int abort_flag;
  uint64_t wait_limit_ns;  // bound of every wait, measured on the global timer
  uint64_t raw_full[kMaxRaw], raw_empty[kMaxRaw], q_raw;
  uint64_t alive_ns;      // when a warp was last seen at work that may take longer than a wait (exact_row)
  int32_t odd_piece[kMarks];  // 1 + the last piece of kMarks in turn that has a scale beyond halves
  Fp4Call call;
  float2 ml_xch[128];     // (reference exponent, row sum) of stream 1's rows, for the in-CTA combination
  float q_unit[2][128];   // of the rows of either M-tile: what a score is worth (score_unit)
};
static_assert(sizeof(Ctrl) <= 4096, "Ctrl must fit behind the tiles");
static_assert(Shape<64>::kSmemBytes <= 227 * 1024 && Shape<128>::kSmemBytes <= 227 * 1024, "shared memory per CTA");
static_assert(Shape<64>::kSlotBytes % 16 == 0 && Shape<128>::kSlotBytes % 16 == 0, "16-byte copies");

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ uint4 ld_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_shared_byte(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared(uint32_t addr, const uint32_t *r) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

extern __shared__ __align__(1024) unsigned char smem[];
template <int kD>
__device__ __forceinline__ Ctrl *ctrl_at() {
  return reinterpret_cast<Ctrl *>(smem + Shape<kD>::kSmemBytes - 4096);
}

// The bounded wait of a whole warp (as wait_bar), in functions of their own: waits that last are rare, and all roles share an SM's instruction cache.  The limit counts from when
// somebody was last seen at exact_row.  kRole: 0 softmax, 1 the others, whose registers are fewer.
template <int kD, int kRole>
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, int code) {
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
          ctrl->call.status[0] = kDevTimeout;
          ctrl->call.status[1] = code;
        }
        return false;
      }
    }
  }
}
template <int kD, int kRole>
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, int code) {
  if (__all_sync(0xFFFFFFFFu, mbar_test_wait(bar, parity) != 0u)) return true;
  return wait_long<kD, kRole>(smem_u32(bar), parity, code);
}

// Instruction descriptors: D fp32, A and B f16, M = 128 (bits 24-28 = M/16), N in bits 17-22 (= N/8).
// QK: N = 64 keys of a half-tile, both operands K-major.  PV: N = head size, bit 16 selects the N-major B operand.
constexpr uint32_t kIdescBase = (1u << 4) | (8u << 24);
constexpr uint32_t kIdescQK = kIdescBase | ((64u >> 3) << 17);
template <int kD>
constexpr uint32_t kIdescPV = kIdescBase | (((uint32_t)kD >> 3) << 17) | (1u << 16);

// P = exp2(scale * s - m) for 64 scores, as halves over the first half of the score buffer; returns the fp32 sum.  With kMax also (in the shadow of the
// exponentials) the maximum of the raw scores.
template <bool kMax>
__device__ __forceinline__ float exp_half(const uint32_t (&v)[64], uint32_t addr, float scale_log2, float neg_m, float &raw_max) {
  const float2 sc = make_float2(scale_log2, scale_log2), nm = make_float2(neg_m, neg_m);
  float2 acc0 = make_float2(0.f, 0.f), acc1 = make_float2(0.f, 0.f);
  float m0 = -INFINITY, m1 = -INFINITY;
  uint32_t pk[32];
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    float2 y0 = ffma2(make_float2(bits_f(v[i]), bits_f(v[i + 1])), sc, nm);
    float2 y1 = ffma2(make_float2(bits_f(v[i + 2]), bits_f(v[i + 3])), sc, nm);
    if (kMax) m0 = max3(m0, bits_f(v[i]), bits_f(v[i + 1]));
    y0.x = ex2(y0.x);
    y0.y = ex2(y0.y);
    if (kMax) m1 = max3(m1, bits_f(v[i + 2]), bits_f(v[i + 3]));
    y1.x = ex2(y1.x);
    y1.y = ex2(y1.y);
    acc0 = fadd2(acc0, y0);
    acc1 = fadd2(acc1, y1);
    pk[i >> 1] = pack_f16(y0.x, y0.y);
    pk[(i >> 1) + 1] = pack_f16(y1.x, y1.y);
  }
  tmem_st32(addr, pk);
  if (kMax) raw_max = fmaxf(m0, m1);
  acc0 = fadd2(acc0, acc1);
  return acc0.x + acc0.y;
}

// O *= alpha.  The PV product of the previous half-unit must have retired first; the one before it has (its commit precedes the s_full this thread has just
// seen), so o_done has completed done_needed or done_needed - 1 phases and the parity says which, whether or not this thread has looked at the
// earlier ones.
template <int kD>
__device__ __noinline__ bool rescale_rows(uint32_t o_addr, float alpha, uint64_t *o_done, uint32_t done_needed, int code) {
  if (!wait<kD, 0>(o_done, (done_needed - 1) & 1u, code)) return false;
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

// The store epilogue of a softmax thread: row r of the accumulator at o_addr times `self` (and, when the CTA's two streams worked on the same
// rows, of the other stream's at o_other times `other`) goes out as bf16 (slot < 0) or as an fp32 partial.  Not inlined: its two row
// buffers must not weigh on the register allocation of the sweep.  Of eight channels those that come are 0, 2, 4, 6, 1, 3, 5, 7.
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
          dst[j] = make_uint4(pack_bf16(bits_f(o[8 * j]), bits_f(o[8 * j + 4])), pack_bf16(bits_f(o[8 * j + 1]), bits_f(o[8 * j + 5])),
                              pack_bf16(bits_f(o[8 * j + 2]), bits_f(o[8 * j + 6])), pack_bf16(bits_f(o[8 * j + 3]), bits_f(o[8 * j + 7])));
      } else {
        // chunk-major: 16-byte chunk k of row r at [slot][k][r], so a warp's store is 512 contiguous bytes
        uint4 *dst = reinterpret_cast<uint4 *>(partial_o) + ((int64_t)slot * (kD / 4) + ch * 8) * 128 + r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dst[2 * j * 128] = make_uint4(o[8 * j], o[8 * j + 4], o[8 * j + 1], o[8 * j + 5]);
          dst[(2 * j + 1) * 128] = make_uint4(o[8 * j + 2], o[8 * j + 6], o[8 * j + 3], o[8 * j + 7]);
        }
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

// Row r of an M-tile of Q, which lies as the copy left it, as halves times a power of two; zeros where no query is.  Returns what a score is worth (score_unit),
// negative if the row has a channel too small beside its largest to be a half.
template <int kD>
__device__ __noinline__ float convert_row(uint32_t tile, int r, bool live, float scale_log2) {
  uint32_t top2 = 0, least2 = 0xFFFFFFFFu;  // of low and high halves: largest magnitudes, least ones that are not 0, less one
#pragma unroll 1
  for (int h = 0; h < kD / 64; ++h)
#pragma unroll 4
    for (int u = 0; u < 8; ++u) {
      const uint4 x = ld_shared(tile + h * kHalfBytes + r * 128 + ((u ^ (r & 7)) << 4));
      const uint32_t m = 0x7FFF7FFFu, a = x.x & m, b = x.y & m, c = x.z & m, d = x.w & m;
      top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(a, b), __vmaxu2(c, d)));
      least2 = __vminu2(least2, __vminu2(__vminu2(__vsub2(a, 0x00010001u), __vsub2(b, 0x00010001u)), __vminu2(__vsub2(c, 0x00010001u), __vsub2(d, 0x00010001u))));
    }
  const uint32_t top = max(top2 & 0xFFFFu, top2 >> 16), least = min(least2 & 0xFFFFu, least2 >> 16);
  const int e = min(half_exponent(top), (int)kQMostExponent);
  const float by = live ? __uint_as_float((uint32_t)(127 + e) << 23) : 0.f;
  const bool odd = least != 0xFFFFu && ((least + 1u) >> 7) + e < 127 - 17;
#pragma unroll 1
  for (int h = 0; h < kD / 64; ++h)
#pragma unroll 2
    for (int u = 0; u < 8; ++u) {
      const uint32_t at = tile + h * kHalfBytes + r * 128 + ((u ^ (r & 7)) << 4);
      uint4 x = ld_shared(at);
      if (live) x = as_halves8(x);
      else x = make_uint4(0, 0, 0, 0);  // (whatever the copy brought along, or left)
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      uint32_t t[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = pack_f16(bits_f(w[i] << 16) * by, bits_f(w[i] & 0xFFFF0000u) * by);
      st_shared(at, t);
    }
  return live ? score_unit(scale_log2, e, top, odd) : 1.0f;
}

template <int kD>
__global__ void __launch_bounds__(kThreads, 1)
attn_fp4_kernel(const __grid_constant__ CUtensorMap q_map, DevBatch d, DevTcPlan tc, const __grid_constant__ Fp4Call in) {
  using Sh = Shape<kD>;
  constexpr int kTileBytes = Sh::kTileBytes, kGroupBytes = Sh::kGroupBytes, kStages = Sh::kStages, kHalves = Sh::kHalves, kRaw = Sh::kRaw;
  if ((smem_u32(smem) & 1023u) != 0u) {  // the swizzled tiles need a 1024-byte aligned base
    if (threadIdx.x == 0) {
      d.status[0] = kDevBounds;
      d.status[1] = 280;
    }
    return;
  }
  unsigned char *q_smem = smem;                           // two M-tiles
  unsigned char *kv_smem = smem + 2 * kTileBytes;         // kStages tiles
  unsigned char *raw_smem = kv_smem + kStages * kTileBytes;  // kRaw tiles of codes and scales
  Ctrl *ctrl = ctrl_at<kD>();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // the plan is uploaded by copies, so it may be read in front of the wait for the kernel before
  const TcCtaHead *head = tc.heads + blockIdx.x;
  const int piece0 = head->piece0, piece1 = head->piece1;
  if (warp == 8) {
    if (lane < (int)(sizeof(TcCtaHead) / 16)) reinterpret_cast<uint4 *>(&ctrl->head)[lane] = __ldg(reinterpret_cast<const uint4 *>(head) + lane);
    if (elect_one()) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
    __syncwarp();
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctrl->kv_full[s], kTeams);
      mbar_init(&ctrl->kv_empty[s], 2);  // one arrival per MMA issuer
    }
    for (int s = 0; s < kRaw; ++s) {
      mbar_init(&ctrl->raw_full[s], 32 + kPagesPerTile);  // the copies of every lane, and what some say of the pages
      mbar_init(&ctrl->raw_empty[s], kTeams);
    }
    mbar_init(&ctrl->q_raw, 1);
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
    ctrl->abort_flag = 0;
    ctrl->alive_ns = 0;
    for (int i = 0; i < kMarks; ++i) ctrl->odd_piece[i] = 0;
    ctrl->wait_limit_ns = (uint64_t)tc.wait_limit_us * 1000ull;
    fence_barrier_init();
  }
  if (threadIdx.x == 32) ctrl->call = in;
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
  const int G = d.group;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    const TcCtaHead *head = &ctrl->head;
    if (warp < 12) {
      // ======================= converters ====================================================
      const int team = warp - 8;
      constexpr int kPasses = Sh::kPasses, kBatch = Sh::kBatch, kPassKeys = Sh::kPassKeys, kScales = Sh::kScales;
      // this lane's key within a pass and its group of 32 channels
      const int key0 = (lane >> 1) & (kPassKeys - 1), grp = kD == 128 ? ((lane >> 4) << 1) | (lane & 1) : lane & 1;
      const int key = team * kKeys + key0;
      // where they lie in a slot (the units of keys 2 and 3 of four are swapped by two, see the copies)
      const uint32_t raw = smem_u32(raw_smem), codes = key * (kD / 2) + (kD == 128 ? grp ^ (key0 & 2) : grp) * 16, scales = Sh::kCodeBytes + key * kScales + grp;
      // of pass 0 in a stage; the four units of 16 bytes are this ^ 16, ^ 32, ^ 48 (key0's bits below 8 do not change from pass to pass)
      const uint32_t to0 = smem_u32(kv_smem) + (key >> 3) * kGroupBytes + (grp >> 1) * kAtomBytes + (key0 & 7) * 128 + ((((grp & 1) * 4) ^ (key0 & 7)) << 4);
      uint32_t ring = 0, slot = 0, slot_parity = 0;
      bool ok = true;
      for (int pc = piece0; pc < piece1 && ok; ++pc) {
        const TcPiece *pi = pc == piece0 ? &head->first : tc.pieces + pc;
        const int steps = 2 * (pi->tile_end - pi->tile_begin);
#pragma unroll 1
        for (int i = 0; i < steps; ++i, ++ring) {
          const uint32_t stage = ring % kStages, parity = ((ring / kStages) & 1u) ^ 1u, from = raw + slot * Sh::kSlotBytes;
          if (!__all_sync(0xFFFFFFFFu, mbar_test_wait2(&ctrl->raw_full[slot], slot_parity, &ctrl->kv_empty[stage], parity) == 3u)) {
            ok = wait<kD, 1>(&ctrl->raw_full[slot], slot_parity, 211) && wait<kD, 1>(&ctrl->kv_empty[stage], parity, 210);
            if (!ok) break;
          }
          // valid tokens of this warp's two pages, and whether a scale is beyond halves
          uint32_t valid[2], word;
          asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(valid[0]), "=r"(valid[1]) : "r"(from + Sh::kCodeBytes + Sh::kScaleBytes + team * 8) : "memory");
          if constexpr (kD == 128) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(word) : "r"(from + Sh::kCodeBytes + (team * kKeys + lane) * 4) : "memory");
          else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(word) : "r"(from + Sh::kCodeBytes + team * kKeys * 2 + (lane & 15) * 4) : "memory");
          const bool whole = valid[0] + valid[1] == 2 * kPage;
          if (__any_sync(0xFFFFFFFFu, any_odd_scale(word))) {  // (among it what a slot of no valid token holds)
            bool odd = false;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int k = kD == 128 ? lane : (lane & 15) * 2 + (x >> 1);
              odd = odd || (odd_scale((word >> (8 * x)) & 0xFFu) && (k & (kPage - 1)) < (int)valid[k >> 4]);
            }
            if (odd) *reinterpret_cast<volatile int32_t *>(&ctrl->odd_piece[pc & (kMarks - 1)]) = pc + 1;
          }
          uint32_t to = to0 + stage * kTileBytes;
#pragma unroll 1
          for (int p0 = 0; p0 < kPasses; p0 += kBatch) {
            uint4 c[kBatch];
            uint32_t f[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              c[u] = ld_shared(from + codes + (p0 + u) * kPassKeys * (kD / 2));
              f[u] = ld_shared_byte(from + scales + (p0 + u) * kPassKeys * kScales);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              f[u] = half_factor(f[u]);
              const int k = (p0 + u) * kPassKeys + key0;
              if (!whole && (k & (kPage - 1)) >= (int)valid[k >> 4]) f[u] = 0u;
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u, to += (kPassKeys / 8) * kGroupBytes) {
              uint32_t h[4];
              halves8(h, c[u].x, f[u]);
              st_shared(to, h);
              halves8(h, c[u].y, f[u]);
              st_shared(to ^ 16u, h);
              halves8(h, c[u].z, f[u]);
              st_shared(to ^ 32u, h);
              halves8(h, c[u].w, f[u]);
              st_shared(to ^ 48u, h);
            }
          }
          fence_proxy_async();
          __syncwarp();  // the slot has been read, the tile's part is written
          if (lane == 0) {
            mbar_arrive(&ctrl->raw_empty[slot]);
            if (blockIdx.x == 0 && ring == 0 && team == 0 && tc.phantom_tx_bytes != 0u) mbar_arrive_expect_tx(&ctrl->kv_full[stage], tc.phantom_tx_bytes);
            else mbar_arrive(&ctrl->kv_full[stage]);
          }
          if (++slot == (uint32_t)kRaw) slot = 0, slot_parity ^= 1u;
        }
      }
    } else if (warp == 15) {
      // ======================= codes and scales =================================================
      uint32_t slot = 0, parity = 1;
      bool ok = true;
      // the entry of page lane & 7 of the tile asked for next, on its way a tile ahead
      int pc = piece0 - 1, i = 0, n = 0, mode = 1, kv_head = 0;
      const TcPage *pages = nullptr;
      bool is_v = false, more = true;
      int2 e = make_int2(0, 0);
      auto next_step = [&]() {
        while (i >= 2 * n) {
          if (++pc >= piece1) {
            more = false;
            return;
          }
          const TcPiece *pi = pc == piece0 ? &head->first : tc.pieces + pc;
          const TcReq *rq = pc == piece0 ? &head->first_req : tc.reqs + pi->req;
          n = pi->tile_end - pi->tile_begin;
          mode = pi->n_mt;
          kv_head = pi->kv_head;
          pages = tc.pages + rq->page_off + pi->tile_begin * kPagesPerTile + (lane & 7);
          i = 0;
        }
        const RingOrder ord(n, mode);
        const int t = ord.step(i, is_v);
        ++i;
        e = ld_pair(pages + t * kPagesPerTile);
      };
      next_step();
#pragma unroll 1
      while (more) {
        int32_t page = e.x;
        if (page < 0 || page >= d.n_pool_pages) {  // never fetch outside the pool
          d.status[0] = kDevBounds;
          d.status[1] = 200;
          page = 0;
        }
        const int32_t row = (page * d.n_kv_heads + kv_head) * kPage;  // rows of the pools are numbered within 32 bits (tc_plan_structure)
        const uint32_t valid = (uint32_t)e.y & 31u, to = smem_u32(raw_smem) + slot * Sh::kSlotBytes;
        const uint8_t *codes = (is_v ? in.v : in.k) + lane * 16, *scales = is_v ? in.v_scale : in.k_scale;
        next_step();
        ok = wait<kD, 1>(&ctrl->raw_empty[slot], parity, 212);
        if (!ok) break;
        constexpr int kCopies = kD / 64;  // of 512 bytes, a page; a key has kD / 32 units, of which those of keys 2 and 3 of four are swapped by two
        const uint32_t unit = kD == 128 ? (uint32_t)lane ^ ((lane >> 3) & 1) << 1 : (uint32_t)lane;
#pragma unroll
        for (int p = 0; p < kPagesPerTile; ++p) {
          const uint8_t *src = codes + (int64_t)__shfl_sync(0xFFFFFFFFu, row, p) * (kD / 2);
#pragma unroll
          for (int c = 0; c < kCopies; ++c) copy16(to + (p * kCopies + c) * 512 + unit * 16, src + c * 512);
        }
        constexpr int kScaleUnits = Sh::kScaleBytes / 16, kEach = kScaleUnits / kPagesPerTile;  // units of scales, of a page
        const int32_t scale_row = __shfl_sync(0xFFFFFFFFu, row, (lane / kEach) & 7);
        if (lane < kScaleUnits) copy16(to + Sh::kCodeBytes + lane * 16, scales + (int64_t)scale_row * Sh::kScales + lane % kEach * 16);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&ctrl->raw_full[slot])) : "memory");
        if (lane < kPagesPerTile) {
          asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + Sh::kCodeBytes + Sh::kScaleBytes + lane * 4), "r"(valid) : "memory");
          mbar_arrive(&ctrl->raw_full[slot]);
        }
        if (++slot == (uint32_t)kRaw) slot = 0, parity ^= 1u;
      }
      asm volatile("cp.async.wait_all;" ::: "memory");  // (after an abort some are still on their way)
    } else if (warp == 12) {
      // ======================= queries =========================================================
      uint32_t q_count = 0;
      bool ok = true;
      const uint32_t q_box_bytes = (uint32_t)(64 * G * T * 2);
      for (int pc = piece0; pc < piece1 && ok; ++pc) {
        const TcPiece pi = pc == piece0 ? head->first : tc.pieces[pc];
        const TcReq rq = pc == piece0 ? head->first_req : tc.reqs[pi.req];
        // once the MMAs of the previous piece no longer read the buffers
        ok = wait<kD, 1>(&ctrl->q_empty, (q_count & 1u) ^ 1u, 205);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&ctrl->q_raw, (uint32_t)(pi.n_mt * kHalves) * q_box_bytes);
        __syncwarp();
        if (lane < kHalves * pi.n_mt)
          tma_load_3d(smem_u32(q_smem) + lane * kHalfBytes, &q_map, (lane % kHalves) * 64, pi.kv_head * G, rq.q_row0 + (pi.mtile0 + lane / kHalves) * T,
                      &ctrl->q_raw);
        ++q_count;
      }
      // copies that nobody waited for, after an abort, must land before the CTA exits
      if (q_count > 0) {
        const uint64_t t0 = global_ns();
        while (!mbar_try_wait(&ctrl->q_raw, (q_count - 1u) & 1u))
          if (global_ns() - t0 > kDrainLimitNs) break;
      }
      __syncwarp();
    } else if (warp < 15) {
      // ======================= MMA issuer of stream s ====================================
      // Both issuers walk every ring position of a piece in order: a position this stream uses is
      // consumed by its MMAs (released by a tcgen05.commit), one it does not use (the other
      // stream's tiles in the even/odd split) is released with a plain arrive once it has landed.
      const int s = __shfl_sync(0xFFFFFFFFu, warp, 0) - 13;
      uint32_t ring_base = 0, waited = 0, p_cnt = 0, pc_idx = 0;
      bool ok = true;
      const uint32_t q_addr = smem_u32(q_smem), kv_addr = smem_u32(kv_smem);
      const uint32_t tmem_u = __shfl_sync(0xFFFFFFFFu, tmem, 0);
      const uint32_t s_tmem = tmem_u + s * 128, o_tmem = tmem_u + 256 + s * 128;
      // Descriptors differ from a base only in the start-address field (units of 16 bytes).
      const uint64_t qdesc0 = make_desc(q_addr, 16, 1024), kdesc0 = make_desc(kv_addr, 16, kGroupBytes),
                     vdesc0 = make_desc(kv_addr, kAtomBytes, kGroupBytes);
      auto issue_qk = [&](int m, uint32_t stage, int half) {  // S_s[half] = Q_m K^T over 64 of the 128 keys
        const uint64_t a = qdesc0 + (uint64_t)(m * (kTileBytes >> 4)),
                       b = kdesc0 + (uint64_t)(stage * (kTileBytes >> 4) + half * (8 * kGroupBytes >> 4));
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_ss(s_tmem + half * 64, a + (uint64_t)(h * (kHalfBytes >> 4) + kk * 2), b + (uint64_t)(h * (kAtomBytes >> 4) + kk * 2),
                   kIdescQK, (h | kk) != 0);
      };
      auto issue_pv = [&](uint32_t stage, int half, bool acc) {  // O_s (+)= P_s[half] V over 64 of the 128 keys
        const uint64_t b = vdesc0 + (uint64_t)(stage * (kTileBytes >> 4) + half * (8 * kGroupBytes >> 4));
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
          mma_ts(o_tmem, s_tmem + half * 64 + k4 * 8, b + (uint64_t)(k4 * (2 * kGroupBytes >> 4)), kIdescPV<kD>, acc || k4 != 0);
      };
      for (int pc = piece0; pc < piece1 && ok; ++pc, ++pc_idx) {
        const TcPiece *pi = pc == piece0 ? &head->first : tc.pieces + pc;
        const int n = pi->tile_end - pi->tile_begin, mode = pi->n_mt;
        const RingOrder ord(n, mode);
        const int my_units = mode == 2 ? n : (n - s + 1) / 2;
        const int m_tile = mode == 2 ? s : 0;
        // waits, in ring order, until absolute ring position `pos` has landed; positions on the way
        // belong to the other stream and are released here
        auto need = [&](uint32_t pos, int code) -> bool {
          while (waited <= pos) {
            if (!wait<kD, 1>(&ctrl->kv_full[waited % kStages], (waited / kStages) & 1u, code)) return false;
            if (waited < pos && elect_one()) mbar_arrive(&ctrl->kv_empty[waited % kStages]);
            ++waited;
          }
          return true;
        };
        // after the MMAs that read the stage: arrives when they retire (the other issuer arrives for itself)
        auto release = [&](uint32_t pos) { tc_commit(&ctrl->kv_empty[pos % kStages]); };
        ok = wait<kD, 1>(&ctrl->q_full, pc_idx & 1u, 220);
        if (!ok) break;
        if (my_units > 0) {
          const uint32_t pos = ring_base + ord.pos_k(mode == 2 ? 0 : s);
          ok = need(pos, 221);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            issue_qk(m_tile, pos % kStages, 0);
            tc_commit(&ctrl->s_full[s][0]);
            issue_qk(m_tile, pos % kStages, 1);
            tc_commit(&ctrl->s_full[s][1]);
            release(pos);
            if (my_units == 1) tc_commit(&ctrl->q_empty);  // last QK of the piece: this stream is done with the Q buffers
          }
          __syncwarp();
        } else {
          if (elect_one()) mbar_arrive(&ctrl->q_empty);
          // nothing to issue in this piece: still observe the previous piece's epilogue phase, so that the parity
          // wait of a later piece never finds this issuer two phases behind
          if (pc_idx > 0) {
            ok = wait<kD, 1>(&ctrl->epi_done, (pc_idx - 1) & 1u, 228);
            if (!ok) break;
          }
        }
        for (int j = 0; j < my_units && ok; ++j) {
          const uint32_t pos_v = ring_base + ord.pos_v(mode == 2 ? j : 2 * j + s), sV = pos_v % kStages;
          ok = need(pos_v, 222);
          if (!ok) break;
          const bool has_next = j + 1 < my_units;
          const uint32_t pos_k = has_next ? ring_base + ord.pos_k(mode == 2 ? j + 1 : 2 * (j + 1) + s) : 0u;
          // the K tile behind: with stages to spare it has landed by now, with four it is waited for under the first product
          if (kStages > 4 && has_next) {
            ok = need(pos_k, 226);
            if (!ok) break;
          }
          if (j == 0 && pc_idx > 0) {  // the epilogue of the previous piece has read O_0 and O_1
            ok = wait<kD, 1>(&ctrl->epi_done, (pc_idx - 1) & 1u, 223);
            if (!ok) break;
          }
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            // P of this half is in place: O += P V, then the buffer takes the scores of the next tile's half
            ok = wait<kD, 1>(&ctrl->p_full[s][half], p_cnt & 1u, 224 + s);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              issue_pv(sV, half, (j | half) != 0);
              tc_commit(&ctrl->o_done[s]);
              if (half == 1) release(pos_v);
            }
            __syncwarp();
            if (!has_next) continue;
            if (kStages <= 4 && half == 0) {
              ok = need(pos_k, 226);
              if (!ok) break;
              tc_fence_after();
            }
            if (elect_one()) {
              issue_qk(m_tile, pos_k % kStages, half);
              tc_commit(&ctrl->s_full[s][half]);
              if (half == 1) {
                release(pos_k);
                if (j + 2 == my_units) tc_commit(&ctrl->q_empty);  // last QK of the piece
              }
            }
            __syncwarp();
          }
          ++p_cnt;
        }
        if (!ok) break;
        // positions of the piece this stream never touched (the tail of the other stream's tiles)
        ring_base += 2u * (uint32_t)n;
        if (waited < ring_base) {
          ok = need(ring_base - 1, 227);
          if (!ok) break;
          if (elect_one()) mbar_arrive(&ctrl->kv_empty[(ring_base - 1) % kStages]);
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
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    // ======================= softmax warpgroups ======================================
    const int s = warp >> 2;                       // stream
    const int quarter = warp & 3;                  // tensor-memory lane quarter this warp may access
    const int r = quarter * 32 + lane;             // row within the M-tile
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_base + s * 128, o_addr = lane_base + 256 + s * 128;
    uint32_t s_cnt = 0, o_cnt = 0;  // tiles / half-units of this stream so far
    uint32_t x_cnt = 0;             // pieces so far in which the two streams were combined
    bool ok = true;
    for (int pc = piece0; pc < piece1; ++pc) {
      const TcPiece pi = pc == piece0 ? head->first : tc.pieces[pc];
      const TcReq rq = pc == piece0 ? head->first_req : tc.reqs[pi.req];
      const int n = pi.tile_end - pi.tile_begin, mode = pi.n_mt;
      const int my_units = mode == 2 ? n : (n - s + 1) / 2;
      const RowInfo ri = row_info(d, tc, rq, T, mode == 2 ? pi.mtile0 + s : pi.mtile0, r, pi.kv_head);
      float sc_row = 0.f;
      if (ok) {
        // the queries as halves; those of one M-tile, which both streams use, by stream 0
        if (mode == 2 || s == 0) {
          ok = wait<kD, 0>(&ctrl->q_raw, (uint32_t)(pc - piece0) & 1u, 245);
          if (ok) {
            ctrl->q_unit[mode == 2 ? s : 0][r] = convert_row<kD>(smem_u32(q_smem) + (mode == 2 ? s : 0) * kTileBytes, r, ri.q_index >= 0, in.scale_log2);
            fence_proxy_async();
          }
        }
        if (ok) {
          mbar_arrive(&ctrl->q_full);
          ok = wait<kD, 0>(&ctrl->q_full, (uint32_t)(pc - piece0) & 1u, 246);
          sc_row = fabsf(ctrl->q_unit[mode == 2 ? s : 0][r]);
        }
      }
      if (ok && my_units > 0) {
        float m_used = -INFINITY, l = 0.f;
        bool s_ready = false;
        // A warp whose 32 rows are all padding only keeps the barriers' counts: what it leaves as weights multiplies into rows
        // of O that nobody reads.
        const bool idle = __all_sync(0xFFFFFFFFu, ri.q_index < 0);
        if (idle) {
          for (int u = 0; u < 2 * my_units && ok; ++u) {
            ok = wait<kD, 0>(&ctrl->s_full[s][u & 1], (s_cnt + (uint32_t)(u >> 1)) & 1u, 230 + s);
            if (ok && u + 1 == 2 * my_units) ok = wait<kD, 0>(&ctrl->o_done[s], (o_cnt + (uint32_t)u - 1) & 1u, 237 + s);
            if (ok) mbar_arrive(&ctrl->p_full[s][u & 1]);
          }
          s_cnt += (uint32_t)my_units;
        }
        for (int j = 0; j < my_units && ok && !idle; ++j) {
          const int t = pi.tile_begin + (mode == 2 ? j : 2 * j + s);
          const bool masked = t >= rq.n_dense_tiles;
          const TcPage *pages = tc.pages + rq.page_off + t * kPagesPerTile;
#pragma unroll 1  // one copy of the sweep: the unrolled pair was slower (instruction fetch)
          for (int half = 0; half < 2; ++half) {
            const uint32_t sh_addr = s_addr + half * 64;
            const uint32_t g = o_cnt + (uint32_t)(2 * j + half);  // half-units of this stream before this one
            const bool first = (j | half) == 0;
            if (!s_ready) {
              ok = wait<kD, 0>(&ctrl->s_full[s][half], s_cnt & 1u, 230 + s);
              if (!ok) break;
            }
            tc_fence_after();
            uint32_t v[64];
            tmem_ld64(sh_addr, v);
            tc_wait_ld();
            // the scores after these are looked for under the exponentials: a test costs over 100 cycles even when it succeeds
            const uint32_t next_ready = mbar_test_wait(&ctrl->s_full[s][half ^ 1], (s_cnt + (uint32_t)half) & 1u);
            if (masked) {
              int n_ok[kPagesPerTile / 2];
#pragma unroll
              for (int p = 0; p < kPagesPerTile / 2; ++p) n_ok[p] = page_n_ok(__ldg(&pages[half * 4 + p].meta), ri);
              mask_half(v, n_ok);
            }
            float sum = 0.f, mx, raw;
            // Fast path: exponentials against the running reference exponent; the maximum of the 64 scores is
            // computed beside them and only checked afterwards.
            bool fast = __all_sync(0xFFFFFFFFu, m_used > -INFINITY);
            if (fast) {
              sum = exp_half<true>(v, sh_addr, sc_row, -m_used, raw);
              mx = raw * sc_row;
              if (__any_sync(0xFFFFFFFFu, mx > m_used + kGrow)) fast = false;
            } else {
              mx = max_half(v) * sc_row;
            }
            if (!fast) {
              // the first half-unit of a stream, rows that have seen no key yet, scores that rise beyond halves: the maximum first
              const bool grow = mx > m_used + kGrow;
              const float alpha = grow ? ex2(m_used - (mx - kLift)) : 1.0f;
              if (grow) {
                l *= alpha;
                m_used = mx - kLift;
              }
              tc_wait_st();
              sum = exp_half<false>(v, sh_addr, sc_row, (m_used == -INFINITY) ? 0.f : -m_used, raw);
              if (!first && __any_sync(0xFFFFFFFFu, grow)) {  // (the scores are no longer held then)
                ok = rescale_rows<kD>(o_addr, alpha, &ctrl->o_done[s], g, 235 + s);
                if (!ok) break;
              }
            }
            l += sum;
            tc_wait_st();
            tc_fence_before();
            s_ready = __all_sync(0xFFFFFFFFu, next_ready) != 0;
            // The wait at the end must not find o_done two phases back (one parity for both): the last arrive comes
            // after the product before has been seen to retire.
            if (half == 1 && j + 1 == my_units) {
              ok = wait<kD, 0>(&ctrl->o_done[s], (g - 1) & 1u, 237 + s);
              if (!ok) break;
            }
            mbar_arrive(&ctrl->p_full[s][half]);
          }
          ++s_cnt;
        }
        if (ok) {
          // epilogue: wait for the last PV of this stream, then normalise and store
          o_cnt += 2u * (uint32_t)my_units;
          ok = wait<kD, 0>(&ctrl->o_done[s], (o_cnt - 1) & 1u, 240 + s);
        }
        // The two streams of a one-M-tile piece hold partial results of the same rows (even and odd tiles).
        // Stream 1 publishes its (m, l); stream 0 reads them and stream 1's accumulator -- the same tensor-memory
        // lanes, so the thread of row r can load both -- and writes one combined result.
        const bool pair = mode == 1 && n >= 2;
        float m_out = m_used, l_out = l, self = 1.0f, other = 0.0f;
        bool writer = true, other_live = false;
        if (ok && pair) {
          if (s == 1) {
            ctrl->ml_xch[r] = make_float2(m_used, l);
            tc_fence_before();
            mbar_arrive(&ctrl->xch);
            writer = false;
          } else {
            ok = wait<kD, 0>(&ctrl->xch, x_cnt & 1u, 242);
            if (ok) {
              tc_fence_after();
              const float2 o = ctrl->ml_xch[r];
              other_live = o.y != 0.f;  // a stream that saw no key of the row has a sum of 0
              m_out = fmaxf(m_used, o.x);
              const float w_self = l != 0.f ? ex2(m_used - m_out) : 0.f, w_other = other_live ? ex2(o.x - m_out) : 0.f;
              self = w_self;
              other = w_other;
              l_out = w_self * l + w_other * o.y;
            }
          }
        }
        if (pair) ++x_cnt;
        if (ok && writer && !idle) {
          // rows to be gone through again: those of a piece with scales beyond halves, and of queries that are
          const int slot = pi.slot[pair ? 0 : s];
          const bool odd_piece = *reinterpret_cast<volatile int32_t *>(&ctrl->odd_piece[pc & (kMarks - 1)]) == pc + 1;
          uint32_t again = __ballot_sync(0xFFFFFFFFu, ri.q_index >= 0 && (odd_piece || ctrl->q_unit[mode == 2 ? s : 0][r] < 0.f));
          tc_fence_after();
          store_rows<kD>(o_addr, lane_base + 256 + (1 - s) * 128, slot, self, other, other_live, m_out, l_out, r, (again >> lane) & 1u ? -1 : ri.q_index, in.out, in.lse,
                         in.partial_o, in.partial_ml);
          tc_fence_before();
          for (; again != 0u; again &= again - 1u) exact_row<kD>(ctrl->call, pc, s, quarter * 32 + __ffs(again) - 1, &ctrl->alive_ns);
        }
      }
      // One arrival per thread and piece.  A stream with units in this piece cannot get here before the previous
      // piece's phase is complete (its PV products were issued behind a wait for it); a stream with none must look
      // itself, or its arrival would be counted into the previous phase while the other stream is still storing.
      if (my_units == 0 && pc > piece0 && ok) ok = wait<kD, 0>(&ctrl->epi_done, (uint32_t)(pc - piece0 - 1) & 1u, 243);
      mbar_arrive(&ctrl->epi_done);
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
attn_fp4_merge_kernel(DevBatch d, DevTcPlan tc, uint16_t *__restrict__ out, float *__restrict__ lse) {
  merge_cta<kD, kBatch>(d, tc, blockIdx.x, blockIdx.y, out, lse);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Q of n rows as [rows][q heads][head size], box = 64 channels x G heads x T tokens.  Made for every call: it takes a fraction of a microsecond.
int encode_q(lr_ctx *ctx, const void *q, int64_t n, CUtensorMap *map) {
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
  const int G = m.n_q_heads / m.n_kv_heads, T = 128 / G;
  const cuuint64_t dims[3] = {(cuuint64_t)m.head_dim, (cuuint64_t)m.n_q_heads, (cuuint64_t)n};
  const cuuint64_t strides[2] = {(cuuint64_t)m.head_dim * 2, (cuuint64_t)m.n_q_heads * m.head_dim * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)T}, estr[3] = {1, 1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->tmap_encode)(
      map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    set_error("cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
    return LR_ECUDA;
  }
  return LR_OK;
}

template <int kD>
int launch(lr_plan *p, const CUtensorMap &q_map, const Fp4Call &in, cudaStream_t s) {
  p->ctx->launches++;
  return cuda_fail(launch_dependent(attn_fp4_kernel<kD>, dim3((unsigned)p->tc.n_cta), dim3(kThreads), Shape<kD>::kSmemBytes, s, q_map, p->dev, p->tc, in),
                   "attn_fp4_kernel launch");
}

template <int kD>
int launch_merge(lr_plan *p, uint16_t *out, float *lse, cudaStream_t s) {
  const DevTcPlan &tc = p->tc;
  if (tc.n_targets == 0) return LR_OK;
  p->ctx->launches++;  // the merge grid is set up while the attention grid drains
  return cuda_fail(launch_dependent(tc.most_slots <= 4 ? attn_fp4_merge_kernel<kD, 4> : attn_fp4_merge_kernel<kD, 8>, dim3((unsigned)tc.n_targets, kD / 8),
                                    dim3(256), 0, s, p->dev, tc, out, lse),
                   "attn_fp4_merge_kernel launch");
}

}  // namespace

int init_attn_fp4_kernel() {
  cudaError_t e = cudaFuncSetAttribute(attn_fp4_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<128>::kSmemBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_fp4_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<64>::kSmemBytes);
  return cuda_fail(e, "attn_fp4_kernel shared-memory attribute");
}

int launch_attn_fp4(lr_plan *p, const void *q, const lr_fp4_cache &c, void *out, float *lse, float scale, cudaStream_t s) {
  const DevTcPlan &tc = p->tc;
  const Fp4Call in = {reinterpret_cast<const uint16_t *>(q), reinterpret_cast<const uint8_t *>(c.k_d), reinterpret_cast<const uint8_t *>(c.v_d), c.k_scale_d, c.v_scale_d,
                      reinterpret_cast<uint16_t *>(out), lse, tc.partial_o, tc.partial_ml, tc.pages, tc.rows, tc.pieces, tc.reqs, p->dev.n_pool_pages, p->dev.status,
                      p->dev.n_q_heads, p->dev.n_kv_heads, p->dev.group, tc.tokens_per_mtile, scale * 1.4426950408889634f};
  if (p->tc_most_rows <= kFp4FewRows) {
    if (int rc = launch_attn_fp4_few(p, in, s)) return rc;
  } else {
    alignas(64) CUtensorMap q_map;
    if (int rc = encode_q(p->ctx, q, p->dev.n_q_rows, &q_map)) return rc;
    if (int rc = (p->dev.head_dim == 128 ? launch<128> : launch<64>)(p, q_map, in, s)) return rc;
  }
  return (p->dev.head_dim == 128 ? launch_merge<128> : launch_merge<64>)(p, in.out, lse, s);
}

}  // namespace lr
