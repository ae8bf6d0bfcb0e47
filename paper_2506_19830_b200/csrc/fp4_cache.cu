// K and V rows into the 4-bit cache and back.
//
// A row is (token, K or V, KV head): head_dim bf16 that become head_dim / 2 bytes of e2m1 codes and a scale byte for every 32 channels.  A group's scale is the smallest
// power of two that keeps its largest magnitude within 6, the largest code: nothing saturates, so that the channels that decide a score are off by the code's rounding
// alone.  It follows from the exponent of that magnitude and one comparison of its fraction, the products with its inverse are exact, and a code is one rounding.
//
// Bound by HBM on long prompts (32 K tokens of 8 heads of 128: written in 29 us, read in 31, 170 MB either way, 5.8 and 5.5 TB/s), by the chain slot -> address -> data and
// the launch on a pass's drafts.  A thread has 16 channels of K and of V of one (token, head): four 16-byte loads in flight, half a group: the largest magnitude takes one
// shuffle more than its own channels.  On the way back it has 8 channels in each half of a row, so that its 16-byte stores and its neighbours' make whole lines.
#include <algorithm>

#include "fp4_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void floats8(uint4 a, float (&x)[8]) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint32_t top2(uint4 a) {  // largest magnitudes of the low and the high halves, as bits
  const uint32_t m = 0x7FFF7FFFu;
  return __vmaxu2(__vmaxu2(a.x & m, a.y & m), __vmaxu2(a.z & m, a.w & m));
}

template <int kD>
__global__ void __launch_bounds__(kThreads)
fp4_write_kernel(CacheRows w, const uint16_t *__restrict__ k, const uint16_t *__restrict__ v, uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                 uint8_t *__restrict__ k_scale, uint8_t *__restrict__ v_scale) {
  constexpr int kLanes = kD / 16;  // threads a row
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the projection may be the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int part = threadIdx.x % kLanes;
  int64_t token;
  int head;
  w.split(row, token, head);
  const int64_t at = row < w.n_rows ? cache_row(__ldcg(reinterpret_cast<const long long *>(w.slots) + token), w.n_slots, w.heads, head, token, w.status) : -1;
  uint4 x[2][2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    x[side][0] = x[side][1] = make_uint4(0, 0, 0, 0);
    if (at >= 0) {
      const uint16_t *src = (side != 0 ? v + token * w.v_stride : k + token * w.k_stride) + head * kD + part * 16;
      x[side][0] = __ldcg(reinterpret_cast<const uint4 *>(src));
      x[side][1] = __ldcg(reinterpret_cast<const uint4 *>(src) + 1);
    }
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const uint32_t two = __vmaxu2(top2(x[side][0]), top2(x[side][1]));
    uint32_t top = max(two & 0xFFFFu, two >> 16);
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));  // of the group
    uint32_t all = top;
#pragma unroll
    for (int o = kLanes / 2; o > 1; o >>= 1) all = max(all, __shfl_xor_sync(0xFFFFFFFFu, all, o));
    const bool fine = all < 0x7F80u;
    const int byte = fp4_byte(top << 16);
    const float by = scale_down(byte);
    float lo[8], hi[8];
    floats8(x[side][0], lo);
    floats8(x[side][1], hi);
    const uint2 codes = make_uint2(fp4_codes(lo, by), fp4_codes(hi, by));
    if (at >= 0) {
      reinterpret_cast<uint2 *>((side != 0 ? v_pool : k_pool) + at * (kD / 2))[part] = fine ? codes : make_uint2(0, 0);
      if ((part & 1) == 0) (side != 0 ? v_scale : k_scale)[at * (kD / kFp4Group) + part / 2] = (uint8_t)(fine ? (uint32_t)byte : kFp4NanScale);
    }
  }
}

template <int kD>
__global__ void __launch_bounds__(kThreads)
fp4_read_kernel(CacheRows w, uint16_t *__restrict__ k, uint16_t *__restrict__ v, const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                const uint8_t *__restrict__ k_scale, const uint8_t *__restrict__ v_scale) {
  constexpr int kLanes = kD / 16;  // threads a row, 8 channels in each half of it
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const int part = threadIdx.x % kLanes;
  int64_t token;
  int head;
  w.split(row, token, head);
  if (row >= w.n_rows) return;
  const int64_t at = cache_row(__ldcg(reinterpret_cast<const long long *>(w.slots) + token), w.n_slots, w.heads, head, token, w.status);
  if (at < 0) return;
  uint32_t c[2][2], byte[2][2];
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int word = part + h * kLanes;
      c[side][h] = __ldcg(reinterpret_cast<const uint32_t *>((side != 0 ? v_pool : k_pool) + at * (kD / 2)) + word);
      byte[side][h] = ld_scale((side != 0 ? v_scale : k_scale) + at * (kD / kFp4Group) + word / 4);
    }
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      reinterpret_cast<uint4 *>((side != 0 ? v + token * w.v_stride : k + token * w.k_stride) + head * kD)[part + h * kLanes] =
          fp4_values(c[side][h], byte[side][h]);
}

}  // namespace

int launch_fp4_move(lr_ctx *ctx, const lr_fp4_cache &c, bool write, void *k, int64_t k_stride, void *v, int64_t v_stride, const int64_t *slots,
                    int32_t n_tokens, int32_t *status, cudaStream_t s) {
  const lr_model &m = ctx->model;
  const CacheRows w = {slots, (int64_t)n_tokens * m.n_kv_heads, c.n_pages * kPage, k_stride, v_stride, m.n_kv_heads, status};
  const int64_t grid = (w.n_rows * (m.head_dim / 16) + kThreads - 1) / kThreads;
  if (grid > 0x7FFFFFFF) {
    set_error("%s: too many rows in one call", write ? "lr_fp4_write" : "lr_fp4_read");
    return LR_EUNSUPPORTED;
  }
  auto *kp = reinterpret_cast<uint16_t *>(k), *vp = reinterpret_cast<uint16_t *>(v);
  auto *kc = reinterpret_cast<uint8_t *>(c.k_d), *vc = reinterpret_cast<uint8_t *>(c.v_d);
  ctx->launches++;
  if (write)
    return cuda_fail(launch_dependent(m.head_dim == 128 ? fp4_write_kernel<128> : fp4_write_kernel<64>, dim3((unsigned)grid), dim3(kThreads), 0, s, w, kp, vp,
                                      kc, vc, c.k_scale_d, c.v_scale_d),
                     "fp4_write_kernel launch");
  return cuda_fail(launch_dependent(m.head_dim == 128 ? fp4_read_kernel<128> : fp4_read_kernel<64>, dim3((unsigned)grid), dim3(kThreads), 0, s, w, kp, vp, kc,
                                    vc, c.k_scale_d, c.v_scale_d),
                   "fp4_read_kernel launch");
}

}  // namespace lr
