// Rotary positions between a joint projection and attention: queries turned, keys turned and written with their values into a cache.
//
// A CTA takes the heads of a few tokens.  It first works out their angles: a position times a frequency in turns, in 64 bits, of which the whole quarters are dropped; what is
// left, an eighth of a turn at most, is exact to 2^-53 of the angle however far the position.  Its sine and cosine are Taylor series in 64 bits, times the amplitude, rounded once: with sinpi
// and cospi in fp32 two and a half times as many codes of an 8-bit cache came out one off.  All heads of a token share them through shared memory.
// A thread then has 8 pairs of a head, both channels of each, so that rows may be turned where they are.  With the channels of a pair half a turned
// part apart these are 8 channels in each half, else 16 side by side: two 16-byte loads and stores.  Where the halves do not start on 16 bytes (rot_dim no multiple of 16) a thread brings
// 16 channels side by side and the threads of a head find their pairs in shared memory (channel by channel from memory a prompt of 32 K tokens, 90 of 128 channels turned, took 1172 us; now 201).
// For a cache in 8 or 4 bits the turned keys and the values wait in shared memory in fp32, and threads of 32 channels of a
// row quantise them: one rounding from what was turned.
//
// Bound by HBM on prompts (32 K tokens of 40 + 8 + 8 heads of 128, half of each turned: 158 us, 940 MB at 6.0 TB/s; into a cache of 8 or 4 bits, whose rows wait between two barriers, 174 and 169 us,
// 5.0 TB/s), by the launch and the chain position -> angle -> data on a pass's drafts.
#include <math.h>

#include <algorithm>

#include "fp4_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 64;       // of q, k and v together, a CTA's share of a token
constexpr int kMaxTokens = 8;    // ... and how many tokens it takes; half as many where heads wait in shared memory
// Of shared memory for rows that are to be quantised, with what else there is below 48 KB.  8 K tokens of 32 + 8 + 8 heads of 128 into an 8-bit cache: 48 us with the four tokens
// that fit, 51 with two, 67 with one.
constexpr int kRowBytes = 36 << 10;
constexpr int kPadded = kFp4Group + 4;  // floats that 32 channels take there: threads next to each other, a group each, read different banks

struct RopeArgs {
  double turns[LR_ROPE_MAX_DIM / 2];
  double amplitude;
  int32_t pairs, interleaved;  // pairs that are turned
  int32_t q_heads, kv_heads, q0;  // q0: 0, or q_heads where there are no queries: the first head of the row [q | k | v] that is looked at
  const int32_t *positions;
  const uint16_t *q, *k, *v;
  uint16_t *q_out;
  int64_t q_stride, k_stride, v_stride;
  const int64_t *slots;
  int64_t n_slots;
  int32_t n_tokens, tokens;  // of the call, of a CTA
  int32_t *status;
  uint8_t *pool[2], *scale[2];
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  uint32_t u;
  memcpy(&u, &t, 4);
  return u;
}
// Cosine and sine of an angle in turns, times an amplitude.  The series of |x| <= pi / 4 end at x^10 and x^11: 2^-31 off at the most.
__device__ __forceinline__ float2 cos_sin(double turns, double amplitude) {
  const double fours = 4.0 * turns, whole = rint(fours), x = (fours - whole) * 1.5707963267948966, y = x * x;
  const double c = 1.0 + y * (-1.0 / 2 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 + y * (-1.0 / 3628800)))));
  const double s = x * (1.0 + y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880 + y * (-1.0 / 39916800))))));
  const float cs = (float)(c * amplitude), sn = (float)(s * amplitude);
  const int quarters = (int)whole;  // below 2^31: a frequency is one radian a position at the most
  const float a = (quarters & 1) != 0 ? -sn : cs, b = (quarters & 1) != 0 ? cs : sn;
  return (quarters & 2) != 0 ? make_float2(-a, -b) : make_float2(a, b);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// kKind: of the cache.  kVector: the pairs of every thread start on 16 bytes.
template <int kD, int kKind, bool kVector>
__global__ void __launch_bounds__(kThreads, 4)  // (three of them without being asked: 4 % more for a prompt of 32 K tokens)
rope_write_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int kLanes = kD / 16;  // threads a head
  constexpr int kRow = kD / kFp4Group * kPadded;
  extern __shared__ __align__(16) float s_rows[];  // [token][K or V row of this CTA][kRow], of a cache in 8 or 4 bits
  constexpr int kTokens = kVector ? kMaxTokens : kMaxTokens / 2;
  __shared__ float4 s_turn[kTokens][4 * kLanes];  // [pairs 2i, 2i + 1 of a part][part]: cosine and sine of either; if not kVector of pair after pair
  __shared__ __align__(16) uint16_t s_head[kVector ? 1 : kThreads / kLanes][kD + 8];  // of heads whose pairs do not start on 16 bytes; the four of a warp in different banks
  __shared__ int64_t s_row[kMaxTokens];  // of the token's first head in the pools; -1: none
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the projection may be the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int t0 = blockIdx.x * a.tokens, n = min(a.tokens, a.n_tokens - t0);
  const int all = a.q_heads + 2 * a.kv_heads, h0 = a.q0 + blockIdx.y * kHeads, heads = min(kHeads, all - h0);
  const int rows0 = max(h0, a.q_heads), rows = max(h0 + heads - rows0, 0);  // K and V among them
  // A thread has the eight pairs of part `threadIdx.x % kLanes` of one or two heads, kStep apart, of every token; where there are fewer heads than that, of every so many tokens.
  constexpr int kStep = kThreads / kLanes, kMine = kHeads / kStep > 0 ? kHeads / kStep : 1;
  const int part = threadIdx.x % kLanes, p0 = part * 8, seat = threadIdx.x / kLanes, wide = min(heads, kStep), stride = kStep / wide, t_first = seat / wide;
  struct Mine {
    const uint16_t *src;  // of the token that is asked for next
    int64_t src_step;
    int32_t off;          // of the head in a row of q_out (channels), or of K or V in a page (rows)
    int32_t row;          // among the rows that are quantised
    bool live, is_q, is_v, turned, apart;
    uint32_t r[8];
  } mine[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    Mine &x = mine[u];
    const int h = seat % wide + u * kStep, head = h0 + h;
    x.live = h < heads && t_first < stride;
    x.is_q = head < a.q_heads;
    x.is_v = head >= a.q_heads + a.kv_heads;
    x.turned = !x.is_v && p0 < a.pairs;
    x.apart = kVector && x.turned && a.interleaved == 0;
    const int kv = x.is_v ? head - a.q_heads - a.kv_heads : head - a.q_heads;
    const int64_t step = x.is_q ? a.q_stride : x.is_v ? a.v_stride : a.k_stride;
    x.src = (x.is_q ? a.q : x.is_v ? a.v : a.k) + (t0 + t_first) * step + (x.is_q ? head : kv) * kD;
    x.src_step = step * stride;
    x.off = x.is_q ? head * kD : kv * kPage;
    x.row = head - rows0;
  }
  // channels of the 8 pairs: c and d and the seven behind them where the halves of what is turned lie apart, else the 16 from c on
  auto load = [&](Mine &x) {
    const int c = x.apart ? p0 : 2 * p0, d = x.apart ? p0 + a.pairs : c + 8;
    const uint4 u = __ldcg(reinterpret_cast<const uint4 *>(x.src + c)), w = __ldcg(reinterpret_cast<const uint4 *>(x.src + d));
    x.r[0] = u.x, x.r[1] = u.y, x.r[2] = u.z, x.r[3] = u.w, x.r[4] = w.x, x.r[5] = w.y, x.r[6] = w.z, x.r[7] = w.w;
    x.src += x.src_step;
  };
  auto finish = [&](Mine &it, int t) {
    const int64_t at_row = s_row[t];
    if (!it.is_q && at_row < 0) return;
    const int c = it.apart ? p0 : 2 * p0, d = it.apart ? p0 + a.pairs : c + 8;
    float x[8], y[8];
    uint32_t (&r)[8] = it.r;  // as they lie; what is not turned is not touched (a NaN keeps its bits)
    const bool as_bf16 = kKind == LR_KV_BF16 || it.is_q;
    auto at = [](int ch) { return ch / kFp4Group * kPadded + ch % kFp4Group; };
    float *const row = as_bf16 ? nullptr : s_rows + (t * rows + it.row) * kRow;
    if (it.apart) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[2 * j] = low(r[j]), x[2 * j + 1] = high(r[j]), y[2 * j] = low(r[4 + j]), y[2 * j + 1] = high(r[4 + j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = low(r[j]), y[j] = high(r[j]);
    }
    if (kVector && it.turned) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 e2 = s_turn[t][i * kLanes + part];  // of two pairs
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int j = 2 * i + k;
          const float cs = k == 0 ? e2.x : e2.z, sn = k == 0 ? e2.y : e2.w, to = x[j] * cs - y[j] * sn, other = fmaf(x[j], sn, y[j] * cs);
          if (p0 + j < a.pairs) {
            x[j] = to;
            y[j] = other;
            if (!it.apart) r[j] = bf16_pair(to, other);
          }
        }
      }
      if (it.apart) {  // all of them are turned
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = bf16_pair(x[2 * j], x[2 * j + 1]), r[4 + j] = bf16_pair(y[2 * j], y[2 * j + 1]);
      }
    }
    // the pairs of a head whose halves lie anywhere, by its threads: pair after pair from where the head waits
    const unsigned of_head = ((1u << kLanes) - 1u) << (threadIdx.x % 32 / kLanes * kLanes);
    auto turn_all = [&](auto get, auto set) {
      __syncwarp(of_head);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = part + j * kLanes;
        if (i < a.pairs) {
          const float2 e = reinterpret_cast<const float2 *>(s_turn[t])[i];
          const float xi = get(i), yi = get(i + a.pairs);
          set(i, xi * e.x - yi * e.y);
          set(i + a.pairs, fmaf(xi, e.y, yi * e.x));
        }
      }
      __syncwarp(of_head);
    };
    if (as_bf16) {
      if (!kVector && !it.is_v) {
        uint16_t *const head = s_head[kVector ? 0 : seat];
        uint4 *const own = reinterpret_cast<uint4 *>(head + c);
        own[0] = make_uint4(r[0], r[1], r[2], r[3]);
        own[1] = make_uint4(r[4], r[5], r[6], r[7]);
        turn_all([&](int ch) { return low(head[ch]); }, [&](int ch, float to) { head[ch] = (uint16_t)bf16_pair(to, to); });
        const uint4 u = own[0], w = own[1];
        r[0] = u.x, r[1] = u.y, r[2] = u.z, r[3] = u.w, r[4] = w.x, r[5] = w.y, r[6] = w.z, r[7] = w.w;
      }
      uint16_t *dst = it.is_q ? a.q_out + (int64_t)(t0 + t) * a.q_heads * kD + it.off : reinterpret_cast<uint16_t *>(a.pool[it.is_v ? 1 : 0]) + (at_row + it.off) * kD;
      *reinterpret_cast<uint4 *>(dst + c) = make_uint4(r[0], r[1], r[2], r[3]);
      *reinterpret_cast<uint4 *>(dst + d) = make_uint4(r[4], r[5], r[6], r[7]);
    } else {
      float4 *to_c = reinterpret_cast<float4 *>(row + at(c)), *to_d = reinterpret_cast<float4 *>(row + at(d));
      if (it.apart) {
        to_c[0] = make_float4(x[0], x[1], x[2], x[3]), to_c[1] = make_float4(x[4], x[5], x[6], x[7]);
        to_d[0] = make_float4(y[0], y[1], y[2], y[3]), to_d[1] = make_float4(y[4], y[5], y[6], y[7]);
      } else {
        to_c[0] = make_float4(x[0], y[0], x[1], y[1]), to_c[1] = make_float4(x[2], y[2], x[3], y[3]);
        to_d[0] = make_float4(x[4], y[4], x[5], y[5]), to_d[1] = make_float4(x[6], y[6], x[7], y[7]);
      }
      if (!kVector && !it.is_v) turn_all([&](int ch) { return row[at(ch)]; }, [&](int ch, float to) { row[at(ch)] = to; });
    }
  };
  // the first token's rows are on their way while the angles are worked out
#pragma unroll
  for (int u = 0; u < kMine; ++u)
    if (mine[u].live && t_first < n) load(mine[u]);
#pragma unroll 1
  for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
    const int t = i / a.pairs, p = i - t * a.pairs;
    const float2 e = cos_sin((double)__ldcg(a.positions + t0 + t) * a.turns[p], a.amplitude);
    // two neighbouring pairs of every part side by side: a thread takes them at once, and its neighbours' lie behind
    if constexpr (kVector) reinterpret_cast<float2 *>(&s_turn[t][(p % 8 / 2) * kLanes + p / 8])[p % 2] = e;
    else reinterpret_cast<float2 *>(s_turn[t])[p] = e;
  }
  if (threadIdx.x < n) {
    const int64_t slot = __ldcg(reinterpret_cast<const long long *>(a.slots) + t0 + threadIdx.x);
    s_row[threadIdx.x] = cache_row(slot, a.n_slots, a.kv_heads, 0, t0 + threadIdx.x, blockIdx.y == 0 ? a.status : nullptr);
  }
  __syncthreads();
  for (int t = t_first; t < n; t += stride) {
#pragma unroll
    for (int u = 0; u < kMine; ++u)
      if (mine[u].live) {
        Mine &x = mine[u];
        Mine now = x;  // (its rows; those of the next token are asked for before they are looked at)
        if (t + stride < n) load(x);
        finish(now, t);
      }
  }
  if constexpr (kKind != LR_KV_BF16) {
    __syncthreads();
    constexpr int kParts = kD / kFp4Group;  // threads a row, 32 channels each
    const int work = n * rows * kParts, loops = (work + kThreads - 1) / kThreads;
    for (int l = 0; l < loops; ++l) {  // (whole warps: a row's threads ask one another)
      const int i = l * kThreads + threadIdx.x, part = i % kParts, r = i / kParts, t = r / max(rows, 1), head = rows0 + r - t * rows;
      const bool live = i < work && s_row[t] >= 0;
      float x[kFp4Group];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < kFp4Group; j += 4) {
        const float4 f = live ? *reinterpret_cast<const float4 *>(s_rows + r * kRow + part * kPadded + j) : make_float4(0.f, 0.f, 0.f, 0.f);
        x[j] = f.x, x[j + 1] = f.y, x[j + 2] = f.z, x[j + 3] = f.w;
#pragma unroll
        for (int m = 0; m < 4; ++m) top = max(top, __float_as_uint(x[j + m]) & 0x7FFFFFFFu);
      }
      uint32_t most = top;  // of the row
#pragma unroll
      for (int o = kParts / 2; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
      if (!live) continue;
      const bool fine = most < 0x7F800000u;
      const int side = head >= a.q_heads + a.kv_heads ? 1 : 0, kv = head - a.q_heads - side * a.kv_heads;
      const int64_t at = s_row[t] + kv * kPage;
      if constexpr (kKind == LR_KV_FP4) {
        const int byte = fp4_byte(top);
        const float by = scale_down(byte);
        const uint4 codes = make_uint4(fp4_codes(x, by), fp4_codes(x + 8, by), fp4_codes(x + 16, by), fp4_codes(x + 24, by));
        reinterpret_cast<uint4 *>(a.pool[side] + at * (kD / 2))[part] = fine ? codes : make_uint4(0, 0, 0, 0);
        a.scale[side][at * kParts + part] = (uint8_t)(fine ? (uint32_t)byte : kFp4NanScale);
      } else {
        const int byte = fp8_byte(most);
        const float by = scale_down(byte);
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = fp8_codes(x + 4 * j, by);
        uint4 *dst = reinterpret_cast<uint4 *>(a.pool[side] + at * kD) + part * 2;
        dst[0] = fine ? make_uint4(w[0], w[1], w[2], w[3]) : make_uint4(0, 0, 0, 0);
        dst[1] = fine ? make_uint4(w[4], w[5], w[6], w[7]) : make_uint4(0, 0, 0, 0);
        if (part == 0) a.scale[side][at] = (uint8_t)(fine ? (uint32_t)byte : kFp8NanScale);
      }
    }
  }
}

template <int kD, int kKind>
int launch(const RopeArgs &a, bool vector, dim3 grid, size_t smem, cudaStream_t s) {
  return cuda_fail(launch_dependent(vector ? rope_write_kernel<kD, kKind, true> : rope_write_kernel<kD, kKind, false>, grid, dim3(kThreads), smem, s, a),
                   "rope_write_kernel launch");
}

}  // namespace

int launch_rope_write(lr_ctx *ctx, const lr_rope *rope, const lr_kv_cache &c, const RopeWrite &w, cudaStream_t s) {
  const lr_model &m = ctx->model;
  RopeArgs a = {};
  if (rope != nullptr) {
    a.pairs = rope->rot_dim / 2;
    a.interleaved = rope->interleaved;
    a.amplitude = rope->amplitude;
    std::copy(rope->turns, rope->turns + a.pairs, a.turns);
  }
  a.q_heads = m.n_q_heads;
  a.kv_heads = m.n_kv_heads;
  a.q0 = w.q != nullptr ? 0 : m.n_q_heads;
  a.positions = w.positions;
  a.q = reinterpret_cast<const uint16_t *>(w.q);
  a.k = reinterpret_cast<const uint16_t *>(w.k);
  a.v = reinterpret_cast<const uint16_t *>(w.v);
  a.q_out = reinterpret_cast<uint16_t *>(w.q_out);
  a.q_stride = w.q_stride;
  a.k_stride = w.k_stride;
  a.v_stride = w.v_stride;
  a.slots = w.slots;
  a.n_slots = c.n_pages * kPage;
  a.n_tokens = w.n_tokens;
  a.status = w.status;
  a.pool[0] = reinterpret_cast<uint8_t *>(c.k_d);
  a.pool[1] = reinterpret_cast<uint8_t *>(c.v_d);
  a.scale[0] = c.k_scale_d;
  a.scale[1] = c.v_scale_d;
  const int heads = m.n_q_heads + 2 * m.n_kv_heads - a.q0, share = std::min(heads, kHeads), chunks = (heads + kHeads - 1) / kHeads;
  const int rows = c.kind == LR_KV_BF16 ? 0 : std::min(share, 2 * m.n_kv_heads);
  const int row_bytes = rows * (m.head_dim / kFp4Group) * kPadded * 4;  // of a token
  const bool vector = a.interleaved != 0 || a.pairs % 8 == 0;
  const int most = vector ? kMaxTokens : kMaxTokens / 2;
  a.tokens = 1;
  while (2 * a.tokens <= most && w.n_tokens / (2 * a.tokens) * (int64_t)chunks >= 8 * ctx->sm_count && 2 * a.tokens * row_bytes <= kRowBytes) a.tokens *= 2;
  const size_t smem = (size_t)a.tokens * row_bytes;
  const dim3 grid((unsigned)((w.n_tokens + a.tokens - 1) / a.tokens), (unsigned)chunks);
  if (chunks > 65535) {
    set_error("lr_rope_write: too many heads");
    return LR_EUNSUPPORTED;
  }
  ctx->launches++;
  if (m.head_dim == 128) {
    if (c.kind == LR_KV_BF16) return launch<128, LR_KV_BF16>(a, vector, grid, smem, s);
    if (c.kind == LR_KV_FP8) return launch<128, LR_KV_FP8>(a, vector, grid, smem, s);
    return launch<128, LR_KV_FP4>(a, vector, grid, smem, s);
  }
  if (c.kind == LR_KV_BF16) return launch<64, LR_KV_BF16>(a, vector, grid, smem, s);
  if (c.kind == LR_KV_FP8) return launch<64, LR_KV_FP8>(a, vector, grid, smem, s);
  return launch<64, LR_KV_FP4>(a, vector, grid, smem, s);
}

}  // namespace lr
