// Tensor-core nested-prefix attention over the 4-bit cache (head_dim 64 or 128).
//
// The plan, the two streams of a CTA, the ring of tiles and what the issuers and the softmax threads do are those of attn_tc.cu.  What is different is how K and V get
// into the ring: four warps bring their codes and scales from the cache and leave them there as bf16.
//
// Numbers.  A code times its scale has two bits of fraction at most: as bf16 it is exact, and so is its product with a bf16 query in fp32.  Codes become
// bf16 by moving their bits (fp4_place: the code times 2^-126) and one multiplication with 2^(byte - 1 - kShift), which brings the number to 2^-kShift of what it is; the scale of
// the softmax and the epilogue take that out again.  With kShift = 16 that factor is a bf16 number for scales up to 2^17 (channels up to 786,432) and what the cache can
// hold below 2^-117 is lost; groups with a larger scale take a second multiplication, which a warp skips where it has none.
//
// A row of K or V that stands for NaN becomes a row of K that is (and zeros in V): the score of its key is no number, nor is the sum of a query that sees it, and one that does
// not see it has a weight of 0 times finite numbers.  Slots that hold no valid token become zeros in V, whatever they held; their scores are masked.
//
// One CTA = 16 warps in four warpgroups, registers moved with setmaxnreg (184 x 256 + 72 x 256 = 128 x 512):
//   warps 8-11  converters, a quarter of every tile each (two pages, 32 keys).  A lane brings the 16 bytes of one group of a key, 32 channels with one scale, by an
//               asynchronous copy into a place of its own, kRaw tiles ahead, reads them back and stores four 16-byte units of the swizzled operand; lanes are dealt to
//               keys and groups so that eight neighbours' stores lie in different banks.
//   warp 12     brings the queries, by TMA.
//   warps 13, 14  MMA issuers of stream 0 and 1.
//   warps 0-3, 4-7  softmax of stream 0 and 1, one thread per query row.
#include <cuda.h>

#include <algorithm>

#include "attn_mma.cuh"
#include "fp4_cache.cuh"

namespace lr {

namespace {

constexpr int kHalfBytes = 16384;  // 128 rows or keys x 64 channels
constexpr int kAtomBytes = 1024;   // K/V tiles: 8 keys x 64 channels, one 128-byte-swizzle atom
constexpr int kMaxStages = 8;
constexpr int kThreads = 512;
constexpr int kTeams = 4;          // converter warps
constexpr int kKeys = 128 / kTeams;  // of a tile, that a warp converts
constexpr int kShift = 16;         // numbers in the ring are 2^-kShift of what they are
constexpr int kMostScale = 128 + kShift;  // the largest scale byte whose factor, 2^(byte - 1 - kShift), is a bf16 number

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
  static constexpr int kPassKeys = kKeys / kPasses;
  static constexpr int kCodeBytes = kKeys * kD / 2, kScaleBytes = kKeys * kScales;
  static constexpr int kSlotBytes = kCodeBytes + 2 * kScaleBytes + 16;  // of a warp: codes, scales, V's scales beside K's, what the keys are
  static constexpr int kRawBytes = kTeams * kRaw * kSlotBytes;
  static constexpr int kSmemBytes = 2 * kTileBytes + kStages * kTileBytes + kRawBytes + 4096;  // tiles, codes, Ctrl; the base must be 1024-aligned
};
constexpr float kRescaleThreshold = 8.0f;  // log2 units: the reference exponent follows the row maximum within 2^8
constexpr float kRedoThreshold = 64.0f;    // log2 units: beyond this a tile is redone with its own maximum as reference

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
  float2 ml_xch[128];     // (reference exponent, row sum) of stream 1's rows, for the in-CTA combination
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
// past L1, as everything that reads the cache (fp8_cache.cuh)
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
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
__device__ __forceinline__ int2 ld_pair(const void *p) {
  int2 v;
  asm volatile("ld.global.nc.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// Instruction descriptors: D fp32, A and B bf16, M = 128 (bits 24-28 = M/16), N in bits 17-22 (= N/8).
// QK: N = 64 keys of a half-tile, both operands K-major.  PV: N = head size, bit 16 selects the N-major B operand.
constexpr uint32_t kIdescBase = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);
constexpr uint32_t kIdescQK = kIdescBase | ((64u >> 3) << 17);
template <int kD>
constexpr uint32_t kIdescPV = kIdescBase | (((uint32_t)kD >> 3) << 17) | (1u << 16);

// P = exp2(scale * s - m) for 64 scores, as bf16 over the first half of the score buffer; returns the fp32 sum.  With kMax also (in the shadow of the
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
    pk[i >> 1] = pack_bf16(y0.x, y0.y);
    pk[(i >> 1) + 1] = pack_bf16(y1.x, y1.y);
  }
  tmem_st32(addr, pk);
  if (kMax) raw_max = fmaxf(m0, m1);
  acc0 = fadd2(acc0, acc1);
  return acc0.x + acc0.y;
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

struct Fp4Pools {
  const uint8_t *k, *v, *k_scale, *v_scale;
};

// The steps of a CTA's ring, tile after tile: which piece, K or V, which tile.
struct Walk {
  int pc, i, n, mode, tile_begin, kv_head;
  const TcPage *pages;  // of the piece's list
};

template <int kD>
__global__ void __launch_bounds__(kThreads, 1)
attn_fp4_kernel(const __grid_constant__ CUtensorMap q_map, DevBatch d, DevTcPlan tc, Fp4Pools in, uint16_t *__restrict__ out, float *__restrict__ lse, float scale_log2) {
  using Sh = Shape<kD>;
  constexpr int kTileBytes = Sh::kTileBytes, kGroupBytes = Sh::kGroupBytes, kStages = Sh::kStages, kHalves = Sh::kHalves, kRaw = Sh::kRaw;
  extern __shared__ __align__(1024) unsigned char smem[];
  if ((smem_u32(smem) & 1023u) != 0u) {  // the swizzled tiles need a 1024-byte aligned base
    if (threadIdx.x == 0) {
      d.status[0] = kDevBounds;
      d.status[1] = 280;
    }
    return;
  }
  unsigned char *q_smem = smem;                           // two M-tiles
  unsigned char *kv_smem = smem + 2 * kTileBytes;         // kStages tiles
  unsigned char *raw_smem = kv_smem + kStages * kTileBytes;  // [team][kRaw] codes and scales
  Ctrl *ctrl = reinterpret_cast<Ctrl *>(raw_smem + Sh::kRawBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // the plan is uploaded by copies, so it may be read in front of the wait for the kernel before
  const TcCtaHead *head = tc.heads + blockIdx.x;
  const int piece0 = head->piece0, piece1 = head->piece1;
  if (warp == 8) {
    if (lane < (int)(sizeof(TcCtaHead) / 16)) reinterpret_cast<uint4 *>(&ctrl->head)[lane] = __ldg(reinterpret_cast<const uint4 *>(head) + lane);
    if (elect_one()) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
    __syncwarp();
  } else {
    // rows of a Q tile that no copy writes must hold finite values: those behind the box of T tokens
    const int live = tc.tokens_per_mtile * d.group, spare = (128 - live) * 8, at = threadIdx.x < 256 ? threadIdx.x : threadIdx.x - 32;  // 16-byte pieces a half-tile
    for (int i = at; i < spare * 2 * kHalves; i += kThreads - 32)
      *reinterpret_cast<uint4 *>(q_smem + (i / spare) * kHalfBytes + live * 128 + (i % spare) * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctrl->kv_full[s], kTeams);
      mbar_init(&ctrl->kv_empty[s], 2);  // one arrival per MMA issuer
    }
    mbar_init(&ctrl->q_full, 1);
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
    ctrl->wait_limit_ns = (uint64_t)tc.wait_limit_us * 1000ull;
    fence_barrier_init();
  }
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
      constexpr int kPasses = Sh::kPasses, kPassKeys = Sh::kPassKeys, kScales = Sh::kScales;
      // this lane's key within a pass and its group of 32 channels
      const int key0 = (lane >> 1) & (kPassKeys - 1), grp = kD == 128 ? ((lane >> 4) << 1) | (lane & 1) : lane & 1;
      const uint32_t raw = smem_u32(raw_smem) + team * (kRaw * Sh::kSlotBytes);
      // of pass 0 in a stage; the four units of 16 bytes are this ^ 16, ^ 32, ^ 48 (key0's bits below 8 do not change from pass to pass)
      const uint32_t to0 = smem_u32(kv_smem) + (team * (kKeys / 8) + (key0 >> 3)) * kGroupBytes + (grp >> 1) * kAtomBytes + (key0 & 7) * 128 + ((((grp & 1) * 4) ^ (key0 & 7)) << 4);
      Walk at;  // what is asked for next
      at.pc = piece0 - 1;
      at.i = at.n = 0;
      int2 e = make_int2(0, 0);  // page entry of lane & 1 of this warp's two pages, of that step
      bool is_v = false, more = true;
      auto load_entry = [&]() {  // of the step at `at`, or no more
        while (at.i >= 2 * at.n) {
          if (++at.pc >= piece1) {
            more = false;
            return;
          }
          const TcPiece *pi = at.pc == piece0 ? &head->first : tc.pieces + at.pc;
          const TcReq *rq = at.pc == piece0 ? &head->first_req : tc.reqs + pi->req;
          at.n = pi->tile_end - pi->tile_begin;
          at.mode = pi->n_mt;
          at.kv_head = pi->kv_head;
          at.pages = tc.pages + rq->page_off + pi->tile_begin * kPagesPerTile + team * (kKeys / kPage) + (lane & 1);
          at.i = 0;
        }
        const RingOrder ord(at.n, at.mode);
        const int t = ord.step(at.i, is_v);
        ++at.i;
        e = ld_pair(at.pages + t * kPagesPerTile);
      };
      uint32_t asked = 0;
      auto ask = [&]() {
        if (more) {
          int32_t page = e.x;
          if (page < 0 || page >= d.n_pool_pages) {  // never fetch outside the pool
            d.status[0] = kDevBounds;
            d.status[1] = 200;
            page = 0;
          }
          const int32_t row = (page * d.n_kv_heads + at.kv_head) * kPage;  // rows of the pools are numbered within 32 bits (tc_plan_structure)
          const int32_t row0 = __shfl_sync(0xFFFFFFFFu, row, 0), row1 = __shfl_sync(0xFFFFFFFFu, row, 1);
          const int32_t valid0 = __shfl_sync(0xFFFFFFFFu, e.y & 31, 0), valid1 = __shfl_sync(0xFFFFFFFFu, e.y & 31, 1);
          const uint32_t slot = raw + (asked % kRaw) * Sh::kSlotBytes;
          const uint8_t *codes = (is_v ? in.v : in.k) + key0 * (kD / 2) + grp * 16;
#pragma unroll
          for (int p = 0; p < kPasses; ++p)
            copy16(slot + p * 512 + lane * 16, codes + (int64_t)((p * kPassKeys >= kPage ? row1 : row0) + p * kPassKeys % kPage) * (kD / 2));
          // a page's scales are kScales units of 16 bytes; V's also beside K's, for rows that stand for NaN
          const int u = lane & 7;
          if (u < 2 * kScales && (lane < 8 || (lane < 16 && !is_v)))
            copy16(slot + Sh::kCodeBytes + (lane >> 3) * Sh::kScaleBytes + u * 16,
                   (is_v || lane >= 8 ? in.v_scale : in.k_scale) + (int64_t)(u >= kScales ? row1 : row0) * kScales + (u % kScales) * 16);
          if (lane == 0)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %3};" ::"r"(slot + Sh::kCodeBytes + 2 * Sh::kScaleBytes), "r"(valid0), "r"(valid1), "r"(is_v ? 1 : 0) : "memory");
          ++asked;
          load_entry();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      load_entry();
#pragma unroll 1
      for (int i = 0; i + 1 < kRaw; ++i) ask();
      bool ok = true;
#pragma unroll 1
      for (uint32_t ring = 0;; ++ring) {
        ask();
        if (ring == asked) break;
        const uint32_t stage = ring % kStages, slot = raw + (ring % kRaw) * Sh::kSlotBytes;
        asm volatile("cp.async.wait_group %0;" ::"n"(kRaw - 1) : "memory");
        __syncwarp();  // the scales and the word about the keys are other lanes'
        ok = wait_bar(&ctrl->kv_empty[stage], ((ring / kStages) & 1u) ^ 1u, ctrl, d.status, 210);
        if (!ok) break;
        const uint4 what = ld_shared(slot + Sh::kCodeBytes + 2 * Sh::kScaleBytes);
        const bool v_tile = what.z != 0u;
        uint32_t to = to0 + stage * kTileBytes;
#pragma unroll 1
        for (int p = 0; p < kPasses; ++p, to += (kPassKeys / 8) * kGroupBytes) {
          const uint4 c = ld_shared(slot + p * 512 + lane * 16);
          const int key = p * kPassKeys + key0;
          const uint32_t from = slot + Sh::kCodeBytes + key * kScales + grp;
          const uint32_t byte = ld_shared_byte(from);
          uint32_t f = twice((min(byte, (uint32_t)kMostScale) + (126 - kShift)) << 7);
          if (v_tile) {
            if (byte == kFp4NanScale || (key & (kPage - 1)) >= (int)(key >= kPage ? what.y : what.x)) f = 0u;
          } else if (byte == kFp4NanScale || ld_shared_byte(from + Sh::kScaleBytes) == kFp4NanScale) {
            f = 0x7FFF7FFFu;
          }
          uint32_t h[16];
          const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            h[4 * j] = mul_bf16x2(fp4_place<0>(w[j]), f);
            h[4 * j + 1] = mul_bf16x2(fp4_place<1>(w[j]), f);
            h[4 * j + 2] = mul_bf16x2(fp4_place<2>(w[j]), f);
            h[4 * j + 3] = mul_bf16x2(fp4_place<3>(w[j]), f);
          }
          if (__any_sync(0xFFFFFFFFu, byte > (uint32_t)kMostScale && byte != kFp4NanScale)) {
            const uint32_t more_f = twice((byte > (uint32_t)kMostScale && byte != kFp4NanScale ? byte - kMostScale + 127u : 127u) << 7);
#pragma unroll
            for (int j = 0; j < 16; ++j) h[j] = mul_bf16x2(h[j], more_f);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) st_shared(to ^ (j << 4), h + 4 * j);
        }
        fence_proxy_async();
        __syncwarp();  // the slot has been read, the tile's part is written
        if (lane == 0) {
          if (blockIdx.x == 0 && ring == 0 && team == 0 && tc.phantom_tx_bytes != 0u) mbar_arrive_expect_tx(&ctrl->kv_full[stage], tc.phantom_tx_bytes);
          else mbar_arrive(&ctrl->kv_full[stage]);
        }
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
        ok = wait_bar(&ctrl->q_empty, (q_count & 1u) ^ 1u, ctrl, d.status, 205);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&ctrl->q_full, (uint32_t)(pi.n_mt * kHalves) * q_box_bytes);
        __syncwarp();
        if (lane < kHalves * pi.n_mt)
          tma_load_3d(smem_u32(q_smem) + lane * kHalfBytes, &q_map, (lane % kHalves) * 64, pi.kv_head * G, rq.q_row0 + (pi.mtile0 + lane / kHalves) * T,
                      &ctrl->q_full);
        ++q_count;
      }
      // copies that nobody waited for, after an abort, must land before the CTA exits
      if (q_count > 0) {
        const uint64_t t0 = global_ns();
        while (!mbar_try_wait(&ctrl->q_full, (q_count - 1u) & 1u))
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
        const TcPiece pi = pc == piece0 ? head->first : tc.pieces[pc];
        const TcReq rq = pc == piece0 ? head->first_req : tc.reqs[pi.req];
        const int n = pi.tile_end - pi.tile_begin, mode = pi.n_mt;
        const RingOrder ord(n, mode);
        const int my_units = mode == 2 ? n : (n - s + 1) / 2;
        const int m_tile = mode == 2 ? s : 0;
        // waits, in ring order, until absolute ring position `pos` has landed; positions on the way
        // belong to the other stream and are released here
        auto need = [&](uint32_t pos, int code) -> bool {
          while (waited <= pos) {
            if (!wait_bar(&ctrl->kv_full[waited % kStages], (waited / kStages) & 1u, ctrl, d.status, code)) return false;
            if (waited < pos && elect_one()) mbar_arrive(&ctrl->kv_empty[waited % kStages]);
            ++waited;
          }
          return true;
        };
        // after the MMAs that read the stage: arrives when they retire (the other issuer arrives for itself)
        auto release = [&](uint32_t pos) { tc_commit(&ctrl->kv_empty[pos % kStages]); };
        ok = wait_bar(&ctrl->q_full, pc_idx & 1u, ctrl, d.status, 220);
        if (!ok) break;
        // the box of a last M-tile brought queries of the next request along: zeros cost the tensor core less power (attn_tc.cu)
        const int live = min(T, rq.n_q - (pi.mtile0 + m_tile) * T) * d.group;
        if (my_units > 0 && live < T * d.group) {
          unsigned char *qs = q_smem + m_tile * kTileBytes;
          for (int idx = lane; idx < (128 - live) * 8; idx += 32)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) *reinterpret_cast<uint4 *>(qs + h * kHalfBytes + live * 128 + idx * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async();
          __syncwarp();
        }
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
            ok = wait_bar(&ctrl->epi_done, (pc_idx - 1) & 1u, ctrl, d.status, 228);
            if (!ok) break;
          }
        }
        for (int j = 0; j < my_units && ok; ++j) {
          const uint32_t pos_v = ring_base + ord.pos_v(mode == 2 ? j : 2 * j + s), sV = pos_v % kStages;
          ok = need(pos_v, 222);
          if (!ok) break;
          const bool has_next = j + 1 < my_units;
          uint32_t pos_k = 0;
          if (has_next) {
            pos_k = ring_base + ord.pos_k(mode == 2 ? j + 1 : 2 * (j + 1) + s);
            ok = need(pos_k, 226);
            if (!ok) break;
          }
          if (j == 0 && pc_idx > 0) {  // the epilogue of the previous piece has read O_0 and O_1
            ok = wait_bar(&ctrl->epi_done, (pc_idx - 1) & 1u, ctrl, d.status, 223);
            if (!ok) break;
          }
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            // P of this half is in place: O += P V, then the buffer takes the scores of the next tile's half
            ok = wait_bar(&ctrl->p_full[s][half], p_cnt & 1u, ctrl, d.status, 224 + s);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              issue_pv(sV, half, (j | half) != 0);
              tc_commit(&ctrl->o_done[s]);
              if (half == 1) release(pos_v);
              if (has_next) {
                issue_qk(m_tile, pos_k % kStages, half);
                tc_commit(&ctrl->s_full[s][half]);
                if (half == 1) {
                  release(pos_k);
                  if (j + 2 == my_units) tc_commit(&ctrl->q_empty);  // last QK of the piece
                }
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
      if (ok && my_units > 0) {
        const RowInfo ri = row_info(d, tc, rq, T, mode == 2 ? pi.mtile0 + s : pi.mtile0, r, pi.kv_head);
        float m_used = -INFINITY, l = 0.f, m_new = 0.f;
        bool pend = false, s_ready = false;
        // O *= alpha.  The PV product of the previous half-unit must have retired first; the one before
        // it has (its commit precedes the s_full this thread has just seen), so o_done has completed done_needed or
        // done_needed - 1 phases and the parity says which, whether or not this thread has looked at the earlier ones.
        auto rescale_o = [&](float alpha, uint32_t done_needed) -> bool {
          if (!wait_bar(&ctrl->o_done[s], (done_needed - 1) & 1u, ctrl, d.status, 235 + s)) return false;
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
        };
        // A warp whose 32 rows are all padding only keeps the barriers' counts: what it leaves as weights multiplies into rows
        // of O that nobody reads.
        const bool idle = __all_sync(0xFFFFFFFFu, ri.q_index < 0);
        if (idle) {
          for (int u = 0; u < 2 * my_units && ok; ++u) {
            ok = wait_bar(&ctrl->s_full[s][u & 1], (s_cnt + (uint32_t)(u >> 1)) & 1u, ctrl, d.status, 230 + s);
            if (ok && u + 1 == 2 * my_units) ok = wait_bar(&ctrl->o_done[s], (o_cnt + (uint32_t)u - 1) & 1u, ctrl, d.status, 237 + s);
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
              ok = wait_bar(&ctrl->s_full[s][half], s_cnt & 1u, ctrl, d.status, 230 + s);
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
            // A growth of the maximum noticed in an earlier half-unit is applied now.
            if (__any_sync(0xFFFFFFFFu, pend)) {
              const float alpha = pend ? ex2(m_used - m_new) : 1.0f;
              if (pend) {
                l *= alpha;
                m_used = m_new;
                pend = false;
              }
              ok = rescale_o(alpha, g);
              if (!ok) break;
            }
            float sum = 0.f, mx, raw;
            // Fast path: exponentials against the running reference exponent; the maximum of the 64 scores is
            // computed beside them and only checked afterwards.
            bool fast = __all_sync(0xFFFFFFFFu, m_used > -INFINITY);
            if (fast) {
              sum = exp_half<true>(v, sh_addr, scale_log2, -m_used, raw);
              mx = raw * scale_log2;
              if (__any_sync(0xFFFFFFFFu, mx > m_used + kRedoThreshold)) fast = false;  // could overflow: redo exactly
            } else {
              mx = max_half(v) * scale_log2;
            }
            if (!fast) {
              // Exact path (first half-unit of a stream, rows that have seen no key yet, a jump of the
              // scores): adopt the maximum before the exponentials.
              const bool grow = mx > m_used + kRescaleThreshold;
              if (__any_sync(0xFFFFFFFFu, grow)) {
                const float alpha = grow ? ex2(m_used - mx) : 1.0f;
                if (grow) {
                  l *= alpha;
                  m_used = mx;
                }
                if (!first) {
                  ok = rescale_o(alpha, g);
                  if (!ok) break;
                }
              }
              tc_wait_st();
              sum = exp_half<false>(v, sh_addr, scale_log2, (m_used == -INFINITY) ? 0.f : -m_used, raw);
            } else if (mx > m_used + kRescaleThreshold) {
              pend = true;
              m_new = mx;
            }
            l += sum;
            tc_wait_st();
            tc_fence_before();
            s_ready = __all_sync(0xFFFFFFFFu, next_ready) != 0;
            // The wait at the end must not find o_done two phases back (one parity for both): the last arrive comes
            // after the product before has been seen to retire.
            if (half == 1 && j + 1 == my_units) {
              ok = wait_bar(&ctrl->o_done[s], (g - 1) & 1u, ctrl, d.status, 237 + s);
              if (!ok) break;
            }
            mbar_arrive(&ctrl->p_full[s][half]);
          }
          ++s_cnt;
        }
        if (ok) {
          // epilogue: wait for the last PV of this stream, then normalise and store
          o_cnt += 2u * (uint32_t)my_units;
          ok = wait_bar(&ctrl->o_done[s], (o_cnt - 1) & 1u, ctrl, d.status, 240 + s);
        }
        // The two streams of a one-M-tile piece hold partial results of the same rows (even and odd tiles).
        // Stream 1 publishes its (m, l); stream 0 reads them and stream 1's accumulator -- the same tensor-memory
        // lanes, so the thread of row r can load both -- and writes one combined result.
        constexpr float kUnit = (float)(1 << kShift);  // what the accumulator's numbers are worth
        const bool pair = mode == 1 && n >= 2;
        float m_out = m_used, l_out = l, self = kUnit, other = 0.0f;
        bool writer = true, other_live = false;
        if (ok && pair) {
          if (s == 1) {
            ctrl->ml_xch[r] = make_float2(m_used, l);
            tc_fence_before();
            mbar_arrive(&ctrl->xch);
            writer = false;
          } else {
            ok = wait_bar(&ctrl->xch, x_cnt & 1u, ctrl, d.status, 242);
            if (ok) {
              tc_fence_after();
              const float2 o = ctrl->ml_xch[r];
              other_live = o.y != 0.f;  // a stream that saw no key of the row has a sum of 0
              m_out = fmaxf(m_used, o.x);
              const float w_self = l != 0.f ? ex2(m_used - m_out) : 0.f, w_other = other_live ? ex2(o.x - m_out) : 0.f;
              self = kUnit * w_self;
              other = kUnit * w_other;
              l_out = w_self * l + w_other * o.y;
            }
          }
        }
        if (pair) ++x_cnt;
        if (ok && writer && !idle) {
          tc_fence_after();
          store_rows<kD>(o_addr, lane_base + 256 + (1 - s) * 128, pi.slot[pair ? 0 : s], self, other, other_live, m_out, l_out, r, ri.q_index, out, lse,
                         tc.partial_o, tc.partial_ml);
          tc_fence_before();
        }
      }
      // One arrival per thread and piece.  A stream with units in this piece cannot get here before the previous
      // piece's phase is complete (its PV products were issued behind a wait for it); a stream with none must look
      // itself, or its arrival would be counted into the previous phase while the other stream is still storing.
      if (my_units == 0 && pc > piece0 && ok) ok = wait_bar(&ctrl->epi_done, (uint32_t)(pc - piece0 - 1) & 1u, ctrl, d.status, 243);
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
int launch(lr_plan *p, const CUtensorMap &q_map, const Fp4Pools &in, uint16_t *out, float *lse, float scale_log2, cudaStream_t s) {
  p->ctx->launches++;
  return cuda_fail(launch_dependent(attn_fp4_kernel<kD>, dim3((unsigned)p->tc.n_cta), dim3(kThreads), Shape<kD>::kSmemBytes, s, q_map, p->dev, p->tc, in, out, lse,
                                    scale_log2 * (float)(1 << kShift)),
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
  const float scale_log2 = scale * 1.4426950408889634f;
  auto *o = reinterpret_cast<uint16_t *>(out);
  if (p->tc_most_rows <= kFp4FewRows) {
    if (int rc = launch_attn_fp4_few(p, q, c, out, lse, scale_log2, s)) return rc;
  } else {
    alignas(64) CUtensorMap q_map;
    if (int rc = encode_q(p->ctx, q, p->dev.n_q_rows, &q_map)) return rc;
    const Fp4Pools in = {reinterpret_cast<const uint8_t *>(c.k_d), reinterpret_cast<const uint8_t *>(c.v_d), c.k_scale_d, c.v_scale_d};
    if (int rc = (p->dev.head_dim == 128 ? launch<128> : launch<64>)(p, q_map, in, o, lse, scale_log2, s)) return rc;
  }
  return (p->dev.head_dim == 128 ? launch_merge<128> : launch_merge<64>)(p, o, lse, s);
}

}  // namespace lr
