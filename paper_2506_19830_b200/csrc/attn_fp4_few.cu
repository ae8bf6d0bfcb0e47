// Attention over the 4-bit cache for few query rows (head_dim 64 or 128): single tokens, short drafts.
//
// With at most 16 rows to a (request, KV head) the cache's bytes are the work, and a tile of 128 rows for the tensor cores is padding.  Here a warp takes pages of 16 keys
// by itself: codes wait in shared memory, become the operands of mma.sync in registers, and there are no barriers or roles.  The plan is that of attn_tc.cu
// (pieces, partial results, merge); the warps of a CTA take a piece's pages in turn and join their sums through shared memory at its end.
//
//   S^T = K Q^T    16 keys x 8 queries.  A lane of quarter t = lane % 4 has of keys lane / 4 and lane / 4 + 8 the t-th quarter of the channels, one load each (which channels a
//                  step of the product takes is free, as long as Q's are the same), of one group of 32 or half of one: a key's factor is one number a lane.
//   O^T += V^T P^T 16 channels x 8 queries over 16 keys.  A lane has of keys 2t, 2t + 1 and the two 8 behind them an eighth of the channels; with the codes of two keys in the
//                  halves of a byte, neighbouring keys of a channel come out side by side, as the product wants them.  P^T comes out of S^T by movmatrix.
//
// Numbers are those of attn_fp4.cu.  A row's reference exponent is set again when a score is more than 2^kRescale above it; the lanes that see it so ask the others for the
// maximum then.
//
// What bounds it is turning codes into operands: nine instructions for a word of eight, some 350 for a page of K and V, 16 of which are products; a scheduler takes 530 cycles for a page,
// its issue slots are taken for two thirds of the time and what only every other cycle takes (conversions, shifts, masks) for half of it.  48 single tokens over 2 to 32 K keys,
// 40 heads of 128 on 8: 128 us, 434 MB at 3.4 TB/s.  As bf16 a word took 17 instructions and the call 158 us; with every warp turning the queries of its pieces by itself
// (5500 cycles a piece) 142, with one page entry asked for at a time 138.
#include <algorithm>

#include "attn_fp4.cuh"

namespace lr {

namespace {

constexpr float kLift = 2.0f;               // log2 units: a row's reference is set this much below its maximum so far,
constexpr float kRescale = 15.0f;           // ... and set again once a score is this much above it: halves end at 2^16
constexpr float kNoKey = -3.0e38f;          // a row's reference before its first key: everything is above it, and a score of -infinity less it is no NaN
constexpr int kHeld = 32;                   // pieces whose records a CTA keeps in shared memory

template <int kD, int kNB>
struct Shape {
  static constexpr int kRows = 8 * kNB;     // queries
  // A lane's sums, queries and a page take 128 registers for 8 queries of 128 channels, 230 for 16, 160 for 16 of 64: with more warps than there is room for it spills (48 requests
  // of 16 rows over 2 to 32 K keys: 128-wide 189 us with 8 warps, 208 with 10; 64-wide 120 with 12, 126 with 16, 140 with 8).
  static constexpr int kWarps = kNB == 1 ? 16 : kD == 64 ? 12 : 8, kThreads = kWarps * 32;
  static constexpr int kStride = kD + 8;    // floats of a query's sums in shared memory: the four quarters of a warp then write to different banks
  static constexpr int kSumBytes = kWarps * kRows * kStride * 4;
  // pages of a warp on their way or being used: K's codes, V's, their scales, what the keys are
  static constexpr int kStages = 4, kCodeBytes = kPage * kD / 2, kScaleBytes = kPage * kD / kFp4Group, kPageBytes = 2 * kCodeBytes + 2 * kScaleBytes + 16;
  static constexpr int kSmemBytes = kSumBytes + kWarps * kStages * kPageBytes;
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {  // of 8 x 8 halves, two a lane
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <int kWords>
__device__ __forceinline__ void ld_codes(uint32_t (&w)[kWords], uint32_t p) {
  if constexpr (kWords == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(p) : "memory");
  else if constexpr (kWords == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(p) : "memory");
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(p) : "memory");
}
__device__ __forceinline__ uint32_t ld_byte(uint32_t p) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(p) : "memory");
  return v;
}
// Where 16-byte unit c of a key's row of V lies in a stage: even keys first and, with two rows to the banks' width, units swapped from four on, so that what the lanes ask for
// at once (two units of keys 2t, t = 0 .. 3) is in different banks.
template <int kD>
__device__ __forceinline__ uint32_t v_unit(int key, int c) {
  const int row = (key & 8) | ((key >> 1) & 3) | ((key & 1) << 2);
  return (uint32_t)(row * (kD / 2) + (kD == 128 ? c ^ (((key >> 2) & 1) << 1) : c) * 16);
}
template <int kD, int kNB>
__global__ void __launch_bounds__(Shape<kD, kNB>::kThreads, 1)
attn_fp4_few_kernel(DevBatch d, DevTcPlan tc, const __grid_constant__ Fp4Call in) {
  using Sh = Shape<kD, kNB>;
  constexpr int kWarps = Sh::kWarps, kThreads = Sh::kThreads, kRows = Sh::kRows, kStride = Sh::kStride, kKWords = kD / 32, kVWords = kD / 64, kMTiles = kD / 16;
  extern __shared__ __align__(16) float s_sum[];  // [warp][query][kStride], then the warps' stages
  __shared__ float2 s_ml[kWarps][kRows];
  __shared__ uint4 s_raw[kRows][kD / 8];  // the next piece's queries,
  __shared__ int2 s_sees[kRows];          // and what they see, as the plan has it
  __shared__ __align__(16) uint16_t s_q[kRows][kD + 8];  // a piece's queries as halves
  __shared__ int4 s_info[kRows];  // what they see (RowInfo), and what a score is worth (score_unit)
  __shared__ TcPiece s_piece[kHeld];
  __shared__ TcReq s_req[kHeld];
  __shared__ int s_odd;  // 1 + the last piece that has a scale beyond halves
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3, g = lane >> 2;
  // the plan is uploaded by copies, so it may be read in front of the wait for the kernel before
  const int piece0 = tc.heads[blockIdx.x].piece0, piece1 = tc.heads[blockIdx.x].piece1;
  if (threadIdx.x < kHeld && piece0 + (int)threadIdx.x < piece1) {
    const TcPiece pi = tc.pieces[piece0 + threadIdx.x];
    s_piece[threadIdx.x] = pi;
    s_req[threadIdx.x] = tc.reqs[pi.req];
  }
  if (threadIdx.x == 0) s_odd = 0;
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");  // queries and cache may come from the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto piece_of = [&](int pc) { return pc - piece0 < kHeld ? s_piece[pc - piece0] : tc.pieces[pc]; };
  auto req_of = [&](int pc, const TcPiece &pi) { return pc - piece0 < kHeld ? s_req[pc - piece0] : tc.reqs[pi.req]; };

  // What is asked for: entries of the page list first, those of the warp's next 32 pages of a piece at once, one a lane and such a set ahead; then the pages that they name.
  int ask_pc = piece0 - 1, ask_i = 0, ask_n = 0, ask_head = 0, ask_dense = 0;
  const TcPage *ask_list = nullptr;
  struct Entries {
    int2 mine;        // this lane's
    int n, head;      // how many there are; their KV head
    uint32_t masked;  // which of them have keys that not every row sees
  } now, next;
  auto ask_entries = [&]() {
    while (ask_i >= ask_n) {
      if (ask_pc + 1 >= piece1) {
        next.n = 0;
        return;
      }
      ++ask_pc;
      const TcPiece pi = piece_of(ask_pc);
      const TcReq rq = req_of(ask_pc, pi);
      ask_i = warp;
      ask_n = min(pi.tile_end * kPagesPerTile, rq.n_pages) - pi.tile_begin * kPagesPerTile;
      ask_dense = (rq.n_dense_tiles - pi.tile_begin) * kPagesPerTile;
      ask_head = pi.kv_head;
      ask_list = tc.pages + rq.page_off + pi.tile_begin * kPagesPerTile;
    }
    const int i = ask_i + lane * kWarps;
    if (i < ask_n) next.mine = ld_pair(ask_list + i);
    next.n = min((ask_n - ask_i + kWarps - 1) / kWarps, 32);
    next.head = ask_head;
    next.masked = __ballot_sync(0xFFFFFFFFu, i >= ask_dense);
    ask_i += 32 * kWarps;
  };
  // A page's codes and scales come by asynchronous copies, kStages - 1 pages ahead: 16 bytes a lane, twice from K and from V (once with head size 64), and 16 of scales from
  // the first lanes.
  constexpr int kUnits = kD / 64;  // of K, and of V, a lane copies
  const uint32_t ring = smem_u32(s_sum) + Sh::kSumBytes + warp * (Sh::kStages * Sh::kPageBytes);
  const int copy_key = lane / (kD / 32), copy_unit = lane % (kD / 32);
  const uint8_t *const codes_at[2] = {in.k + lane * 16, in.v + lane * 16};
  const uint8_t *const scales_at = (lane * 16 < Sh::kScaleBytes ? in.k_scale : in.v_scale) + lane * 16 % Sh::kScaleBytes;
  uint32_t to_v[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) to_v[u] = Sh::kCodeBytes + v_unit<kD>(copy_key + u * 8, copy_unit);
  const uint32_t v_lane = Sh::kCodeBytes + v_unit<kD>(2 * t, g * (kD / 16) / 16) + g * (kD / 16) % 16;  // where this lane's channels of key 2t lie
  uint32_t asked = 0;  // stage
  int at_entry = 0;
  auto ask_page = [&]() {
    if (at_entry >= now.n) {
      now = next;
      at_entry = 0;
      if (now.n > 0) ask_entries();
    }
    if (at_entry < now.n) {
      int32_t page = __shfl_sync(0xFFFFFFFFu, now.mine.x, at_entry);
      const int32_t meta = __shfl_sync(0xFFFFFFFFu, now.mine.y, at_entry);
      if (page < 0 || page >= d.n_pool_pages) {  // never fetch outside the pool
        d.status[0] = kDevBounds;
        d.status[1] = 200;
        page = 0;
      }
      const int64_t row = (page * d.n_kv_heads + now.head) * kPage;  // rows of the pools are numbered within 32 bits (tc_plan_structure)
      const uint32_t to = ring + asked * Sh::kPageBytes;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        copy16(to + u * 512 + lane * 16, codes_at[0] + row * (kD / 2) + u * 512);
        copy16(to + to_v[u], codes_at[1] + row * (kD / 2) + u * 512);
      }
      if (lane * 16 < 2 * Sh::kScaleBytes) copy16(to + 2 * Sh::kCodeBytes + lane * 16, scales_at + row * (kD / kFp4Group));
      if (lane == 0)
        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to + 2 * Sh::kCodeBytes + 2 * Sh::kScaleBytes), "r"(meta), "r"(now.masked >> at_entry & 1u) : "memory");
      ++at_entry;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    asked = asked + 1 == Sh::kStages ? 0u : asked + 1;
  };

  const int G = d.group;
  // The queries of a piece: eight channels a lane, some rows a warp, on their way under the pages of the piece before; as halves they wait in shared memory for all warps.
  constexpr int kRowLanes = kD / 8;
  const int q_row = warp * (32 / kRowLanes) + lane / kRowLanes, q_part = lane % kRowLanes;
  auto ask_queries = [&](int pc) {
    if (q_row >= kRows || pc >= piece1) return;  // (whole warps)
    const TcPiece pi = piece_of(pc);
    const TcReq rq = req_of(pc, pi);
    if (q_row >= rq.n_q * G) return;
    const int row = rq.q_row0 + q_row / G;
    copy16(smem_u32(&s_raw[q_row][q_part]), reinterpret_cast<const uint8_t *>(in.q + ((int64_t)row * d.n_q_heads + pi.kv_head * G + q_row % G) * kD + q_part * 8));
    if (q_part == 0) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(&s_sees[q_row])), "l"(tc.rows + row) : "memory");
  };
  auto leave_queries = [&](int pc) {
    if (q_row >= kRows || pc >= piece1) return;
    const bool live = q_row < req_of(pc, piece_of(pc)).n_q * G;
    const uint4 q_raw = live ? s_raw[q_row][q_part] : make_uint4(0, 0, 0, 0);
    const uint32_t m = 0x7FFF7FFFu, two = __vmaxu2(__vmaxu2(q_raw.x & m, q_raw.y & m), __vmaxu2(q_raw.z & m, q_raw.w & m));
    uint32_t top = max(two & 0xFFFFu, two >> 16);
#pragma unroll
    for (int y = 1; y < kRowLanes; y <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, y));
    const int e = min(half_exponent(top), (int)kQMostExponent);
    const float by = __uint_as_float((uint32_t)(127 + e) << 23);
    const uint4 p = as_halves8(q_raw);
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
    uint32_t h[4];
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float lo = bits_f(w[j] << 16) * by, hi = bits_f(w[j] & 0xFFFF0000u) * by;
      odd = odd || (lo != 0.f && fabsf(lo) < 0x1p-17f) || (hi != 0.f && fabsf(hi) < 0x1p-17f);
      h[j] = pack_f16(lo, hi);
    }
    const unsigned any = __ballot_sync(0xFFFFFFFFu, odd) >> (lane - q_part) & ((1u << kRowLanes) - 1u);
    *reinterpret_cast<uint4 *>(&s_q[q_row][q_part * 8]) = make_uint4(h[0], h[1], h[2], h[3]);
    if (q_part == 0) {
      const int2 sees = live ? s_sees[q_row] : make_int2(-1, -1);
      s_info[q_row] = make_int4(live ? sees.x & 0xFFFF : -1, sees.x >> 16, sees.y, __float_as_int(score_unit(in.scale_log2, e, top, any != 0u)));
    }
  };
  now.n = 0;
  now.mine = next.mine = make_int2(0, 0);
  ask_entries();
  ask_queries(piece0);
  asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll 1
  for (int i = 0; i + 1 < Sh::kStages; ++i) ask_page();
  asm volatile("cp.async.wait_group %0;" ::"n"(Sh::kStages - 1) : "memory");
  leave_queries(piece0);
  __syncthreads();
  uint32_t from = 0;  // stage
  for (int pc = piece0; pc < piece1; ++pc) {
    const TcPiece pi = piece_of(pc);
    const TcReq rq = req_of(pc, pi);
    const int rows = min(rq.n_q * G, kRows), n_pages = min(pi.tile_end * kPagesPerTile, rq.n_pages) - pi.tile_begin * kPagesPerTile;
    uint32_t qf[kNB][kD / 8];
    float sc[kNB][2];
    int depth[kNB][2], branch[kNB][2], limit[kNB][2];  // of this lane's columns, queries 2t and 2t + 1
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
#pragma unroll
      for (int i = 0; i < kD / 32; ++i) {
        const uint4 x = *reinterpret_cast<const uint4 *>(&s_q[b * 8 + g][t * (kD / 4) + i * 8]);
        qf[b][4 * i] = x.x, qf[b][4 * i + 1] = x.y, qf[b][4 * i + 2] = x.z, qf[b][4 * i + 3] = x.w;
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int4 x = s_info[b * 8 + 2 * t + y];
        depth[b][y] = x.x, branch[b][y] = x.y, limit[b][y] = x.z, sc[b][y] = fabsf(__int_as_float(x.w));
      }
    }
    // rows with a channel too small beside their largest to be a half, or scores beyond fp32
    unsigned again = __ballot_sync(0xFFFFFFFFu, lane < kRows && s_info[lane % kRows].w < 0);
    ask_queries(pc + 1);
    float o[kNB][kMTiles][4], ref[kNB][2], l[kNB][2];
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      ref[b][0] = ref[b][1] = kNoKey;
      l[b][0] = l[b][1] = 0.f;
#pragma unroll
      for (int m = 0; m < kMTiles; ++m) o[b][m][0] = o[b][m][1] = o[b][m][2] = o[b][m][3] = 0.f;
    }
#pragma unroll 1
    for (int i = warp; i < n_pages; i += kWarps) {
      __syncwarp();  // the stage asked for next has been read
      ask_page();
      asm volatile("cp.async.wait_group %0;" ::"n"(Sh::kStages - 1) : "memory");
      __syncwarp();  // what the other lanes have copied is there
      const uint32_t at = ring + from * Sh::kPageBytes, scales = at + 2 * Sh::kCodeBytes;
      from = from + 1 == Sh::kStages ? 0u : from + 1;
      uint32_t k[2][kKWords], kb[2], v[4][kVWords], vb[4], what[2], word[1];
      const uint32_t k_from = at + g * (kD / 2) + t * (kD / 8), kb_from = scales + g * (kD / kFp4Group) + t * (kD / 4) / kFp4Group;
      const uint32_t v_from = at + v_lane, vb_from = scales + Sh::kScaleBytes + 2 * t * (kD / kFp4Group) + g * (kD / 8) / kFp4Group;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        ld_codes(k[j], k_from + j * 8 * (kD / 2));
        kb[j] = ld_byte(kb_from + j * 8 * (kD / kFp4Group));
      }
      ld_codes(what, scales + 2 * Sh::kScaleBytes);
      ld_codes(word, scales + lane % (Sh::kScaleBytes / 2) * 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) vb[j] = ld_byte(vb_from + ((j >> 1) * 8 + (j & 1)) * (kD / kFp4Group));
      const uint32_t meta = what[0];
      const bool masked = what[1] != 0u;
      const int valid = (int)(meta & 31u);
      if (__any_sync(0xFFFFFFFFu, any_odd_scale(word[0]))) {  // (among it what a slot of no valid token holds)
        bool odd = false;
#pragma unroll
        for (int x = 0; x < 4; ++x) odd = odd || (odd_scale((word[0] >> (8 * x)) & 0xFFu) && (lane * 4 + x) % Sh::kScaleBytes / (kD / kFp4Group) < valid);
        if (odd) *reinterpret_cast<volatile int *>(&s_odd) = pc + 1;
      }
      float s[kNB][4];
#pragma unroll
      for (int b = 0; b < kNB; ++b) s[b][0] = s[b][1] = s[b][2] = s[b][3] = 0.f;
      uint32_t f[2] = {half_factor(kb[0]), half_factor(kb[1])};
#pragma unroll
      for (int w = 0; w < kKWords; ++w) {
        uint32_t a[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) halves8(a[j], k[j][w], f[j]);
#pragma unroll
        for (int b = 0; b < kNB; ++b) {
          mma16816(s[b], a[0][0], a[1][0], a[0][1], a[1][1], qf[b][4 * w], qf[b][4 * w + 1]);
          mma16816(s[b], a[0][2], a[1][2], a[0][3], a[1][3], qf[b][4 * w + 2], qf[b][4 * w + 3]);
        }
      }
      uint32_t pt[kNB][2];
#pragma unroll
      for (int b = 0; b < kNB; ++b) {
        if (masked) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            RowInfo ri;
            ri.depth = depth[b][e], ri.branch = branch[b][e], ri.limit = limit[b][e];
            const int n_ok = page_n_ok(meta, ri);
            if (g >= n_ok) s[b][e] = -INFINITY;
            if (g + 8 >= n_ok) s[b][2 + e] = -INFINITY;
          }
        }
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = fmaf(s[b][i], sc[b][i & 1], -ref[b][i & 1]);
        if (__any_sync(0xFFFFFFFFu, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) > kRescale)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(s[b][e], s[b][2 + e]) * sc[b][e];
#pragma unroll
            for (int y = 4; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, y));
            if (top > ref[b][e] + kRescale) {
              const float down = ex2(ref[b][e] - (top - kLift));
              ref[b][e] = top - kLift;
              l[b][e] *= down;
#pragma unroll
              for (int m = 0; m < kMTiles; ++m) o[b][m][e] *= down, o[b][m][2 + e] *= down;
            }
            x[e] = fmaf(s[b][e], sc[b][e], -ref[b][e]);
            x[2 + e] = fmaf(s[b][2 + e], sc[b][e], -ref[b][e]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = ex2(x[i]);
        l[b][0] += x[0] + x[2];
        l[b][1] += x[1] + x[3];
        const uint32_t p0 = pack_f16(x[0], x[1]), p1 = pack_f16(x[2], x[3]);
        pt[b][0] = transpose8(p0);
        pt[b][1] = transpose8(p1);
      }
      // O^T += V^T P^T
#pragma unroll
      for (int j = 0; j < 4; ++j) ld_codes(v[j], v_from + ((j >> 1) * 8 + (j & 1) * 4) * (kD / 2));  // (odd keys four rows behind the even ones)
#pragma unroll
      for (int j = 0; j < 2; ++j) f[j] = half_factors(vb[2 * j], vb[2 * j + 1]);
      if (masked) {  // slots of no valid token
#pragma unroll
        for (int j = 0; j < 2; ++j) f[j] &= (2 * t + 8 * j < valid ? 0xFFFFu : 0u) | (2 * t + 8 * j + 1 < valid ? 0xFFFF0000u : 0u);
      }
#pragma unroll
      for (int w = 0; w < kVWords; ++w) {
        uint32_t a[2][2][4];  // [which two keys][channels 0, 4, 1, 5 or 2, 6, 3, 7]
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t x = v[2 * j][w], y = v[2 * j + 1][w], m = 0x0F0F0F0Fu;
          halves8(a[j][0], (x & m) | ((y << 4) & ~m), f[j]);
          halves8(a[j][1], ((x >> 4) & m) | (y & ~m), f[j]);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)  // channels 2y and 2y + 1
#pragma unroll
          for (int b = 0; b < kNB; ++b)
            mma16816(o[b][4 * w + y], a[0][y & 1][y >> 1], a[0][y & 1][2 + (y >> 1)], a[1][y & 1][y >> 1], a[1][y & 1][2 + (y >> 1)], pt[b][0], pt[b][1]);
      }
    }
    // the warps' sums, joined
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[b][e] += __shfl_xor_sync(0xFFFFFFFFu, l[b][e], x);
        const int r = b * 8 + 2 * t + e;
        if (g == 0) s_ml[warp][r] = make_float2(ref[b][e], l[b][e]);
        float *to = s_sum + (warp * kRows + r) * kStride + g * 2;
#pragma unroll
        for (int m = 0; m < kMTiles; ++m) *reinterpret_cast<float2 *>(to + m * 16) = make_float2(o[b][m][e], o[b][m][2 + e]);
      }
    }
    __syncthreads();
    const int slot = pi.slot[0];
    if (s_odd == pc + 1) again = (1u << kRows) - 1u;
    for (int i = threadIdx.x; i < rows * (kD / 2); i += kThreads) {  // a pair of channels: 2m and 2m + 1 of eighth x
      const int r = i / (kD / 2), c = i % (kD / 2), ch = (c % 8) * (kD / 8) + 2 * (c / 8);
      if ((again >> r) & 1u) continue;
      float top = -INFINITY, sum = 0.f;
      float2 acc = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = s_ml[w][r].y != 0.f ? fmaxf(top, s_ml[w][r].x) : top;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = s_ml[w][r];
        if (ml.y != 0.f) {  // (a warp that saw no key of the row has a sum of 0)
          const float by = ex2(ml.x - top);
          const float2 x = *reinterpret_cast<const float2 *>(s_sum + (w * kRows + r) * kStride + 2 * c);
          sum = fmaf(by, ml.y, sum);
          acc.x = fmaf(by, x.x, acc.x);
          acc.y = fmaf(by, x.y, acc.y);
        }
      }
      const int64_t q_index = (int64_t)(rq.q_row0 + r / G) * d.n_q_heads + pi.kv_head * G + r % G;
      if (slot < 0) {
        const float inv = 1.0f / sum;
        *reinterpret_cast<uint32_t *>(in.out + q_index * kD + ch) = pack_bf16(acc.x * inv, acc.y * inv);
        if (c == 0 && in.lse != nullptr) in.lse[q_index] = (top + log2f(sum)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float2 *>(in.partial_o + (((int64_t)slot * (kD / 4) + ch / 4) * 128 + r) * 4 + ch % 4) = acc;
        // a sum that is not a number must not look like that of a row that saw nothing: the merge asks whether the sum is above 0
        if (c == 0) *reinterpret_cast<float2 *>(in.partial_ml + ((int64_t)slot * 128 + r) * 2) = sum != sum ? make_float2(sum, 1.0f) : make_float2(top, sum);
      }
    }
    for (int r = warp; r < rows; r += kWarps)
      if ((again >> r) & 1u) exact_row<kD>(in, pc, 0, r, nullptr);
    if (q_row < kRows && pc + 1 < piece1 && n_pages - warp <= (Sh::kStages - 1) * kWarps)
      asm volatile("cp.async.wait_all;" ::: "memory");  // (the queries; with kStages pages or more they have been waited for)
    leave_queries(pc + 1);
    __syncthreads();  // the sums have been read, the queries are there
  }
}

template <int kD, int kNB>
int launch(lr_plan *p, const Fp4Call &in, cudaStream_t s) {
  p->ctx->launches++;
  return cuda_fail(launch_dependent(attn_fp4_few_kernel<kD, kNB>, dim3((unsigned)p->tc.n_cta), dim3(Shape<kD, kNB>::kThreads), Shape<kD, kNB>::kSmemBytes, s, p->dev, p->tc, in),
                   "attn_fp4_few_kernel launch");
}

template <int kD, int kNB>
cudaError_t allow() {
  return cudaFuncSetAttribute(attn_fp4_few_kernel<kD, kNB>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<kD, kNB>::kSmemBytes);
}

}  // namespace

int init_attn_fp4_few_kernel() {
  cudaError_t e = allow<128, 1>();
  if (e == cudaSuccess) e = allow<128, 2>();
  if (e == cudaSuccess) e = allow<64, 1>();
  if (e == cudaSuccess) e = allow<64, 2>();
  return cuda_fail(e, "attn_fp4_few_kernel shared-memory attribute");
}

int launch_attn_fp4_few(lr_plan *p, const Fp4Call &in, cudaStream_t s) {
  if (p->dev.head_dim == 128) return p->tc_most_rows <= 8 ? launch<128, 1>(p, in, s) : launch<128, 2>(p, in, s);
  return p->tc_most_rows <= 8 ? launch<64, 1>(p, in, s) : launch<64, 2>(p, in, s);
}

}  // namespace lr
