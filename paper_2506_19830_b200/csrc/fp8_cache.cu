// K and V rows into the 8-bit cache and back.
//
// A row is (token, K or V, KV head): head_dim bf16 that become head_dim e4m3 codes and one scale byte.  The largest magnitude of a
// row is found on its bf16 bits (for non-negative numbers their order is that of the integers, infinities and NaN at the top), and as the
// scale is a power of two it follows from the exponent and one comparison of the fraction: no division, and the products x 2^-e are
// exact, so a code is one rounding of its value.
//
// Bound by HBM on long prompts, by the chain slot -> address -> data and the launch on a pass's drafts.  A thread has 16 channels of K and of V of one
// (token, head): four 16-byte loads in flight and two 16-byte stores, a row is 8 neighbouring threads (4 with head size 64): the maximum takes
// three shuffles, and the rows of a token, which lie side by side in the projection's output, are read in whole lines.  On the way back a thread has 8
// channels in each half of a row, so that its 16-byte stores and its neighbours' make whole lines.
#include <algorithm>

#include "fp8_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256;

// |x| of two bf16 numbers, as integers
__device__ __forceinline__ uint32_t abs2(uint32_t x) { return x & 0x7FFF7FFFu; }

__device__ __forceinline__ uint2 codes8(uint4 a, float by) {  // eight bf16 values times a power of two
  const float x[8] = {__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xFFFF0000u), __uint_as_float(a.y << 16), __uint_as_float(a.y & 0xFFFF0000u),
                      __uint_as_float(a.z << 16), __uint_as_float(a.z & 0xFFFF0000u), __uint_as_float(a.w << 16), __uint_as_float(a.w & 0xFFFF0000u)};
  return make_uint2(fp8_codes(x, by), fp8_codes(x + 4, by));
}

template <int kD>
__global__ void __launch_bounds__(kThreads)
fp8_write_kernel(CacheRows w, const uint16_t *__restrict__ k, const uint16_t *__restrict__ v, uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                 uint8_t *__restrict__ k_scale, uint8_t *__restrict__ v_scale) {
  constexpr int kLanes = kD / 16;  // threads a row
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the projection may be the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
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
      x[side][0] = __ldg(reinterpret_cast<const uint4 *>(src));
      x[side][1] = __ldg(reinterpret_cast<const uint4 *>(src) + 1);
    }
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const uint4 a = x[side][0], b = x[side][1];
    const uint32_t two =
        __vmaxu2(__vmaxu2(__vmaxu2(abs2(a.x), abs2(a.y)), __vmaxu2(abs2(a.z), abs2(a.w))), __vmaxu2(__vmaxu2(abs2(b.x), abs2(b.y)), __vmaxu2(abs2(b.z), abs2(b.w))));
    uint32_t top = max(two & 0xFFFFu, two >> 16);  // bits of the largest magnitude
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const bool fine = top < 0x7F80u;
    const int byte = fp8_byte(top << 16);
    const float by = scale_down(byte);
    const uint2 lo = codes8(a, by), hi = codes8(b, by);
    const uint4 c = make_uint4(lo.x, lo.y, hi.x, hi.y);
    if (at >= 0) {
      reinterpret_cast<uint4 *>((side != 0 ? v_pool : k_pool) + at * kD)[part] = fine ? c : make_uint4(0, 0, 0, 0);
      if (part == 0) (side != 0 ? v_scale : k_scale)[at] = (uint8_t)(fine ? (uint32_t)byte : kFp8NanScale);
    }
  }
}

__device__ __forceinline__ uint32_t pack2(float2 x, float by) {  // exact: a power of two times at most four bits
  __nv_bfloat162 t = __floats2bfloat162_rn(x.x * by, x.y * by);
  uint32_t u;
  memcpy(&u, &t, 4);
  return u;
}

template <int kD>
__global__ void __launch_bounds__(kThreads)
fp8_read_kernel(CacheRows w, uint16_t *__restrict__ k, uint16_t *__restrict__ v, const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                const uint8_t *__restrict__ k_scale, const uint8_t *__restrict__ v_scale) {
  constexpr int kLanes = kD / 16;  // threads a row, 8 channels in each half of it
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int part = threadIdx.x % kLanes;
  if (row >= w.n_rows) return;
  int64_t token;
  int head;
  w.split(row, token, head);
  const int64_t at = cache_row(__ldcg(reinterpret_cast<const long long *>(w.slots) + token), w.n_slots, w.heads, head, token, w.status);
  if (at < 0) return;
  uint2 c[2][2];
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int h = 0; h < 2; ++h) c[side][h] = __ldcg(reinterpret_cast<const uint2 *>((side != 0 ? v_pool : k_pool) + at * kD) + part + h * kLanes);
  const float by[2] = {fp8_scale(ld_scale(k_scale + at)), fp8_scale(ld_scale(v_scale + at))};
#pragma unroll
  for (int side = 0; side < 2; ++side)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 q = c[side][h];
      reinterpret_cast<uint4 *>((side != 0 ? v + token * w.v_stride : k + token * w.k_stride) + head * kD)[part + h * kLanes] =
          make_uint4(pack2(fp8_float2(q.x & 0xFFFFu), by[side]), pack2(fp8_float2(q.x >> 16), by[side]), pack2(fp8_float2(q.y & 0xFFFFu), by[side]),
                     pack2(fp8_float2(q.y >> 16), by[side]));
    }
}

}  // namespace

int launch_fp8_move(lr_ctx *ctx, const lr_fp8_cache &c, bool write, void *k, int64_t k_stride, void *v, int64_t v_stride, const int64_t *slots,
                    int32_t n_tokens, int32_t *status, cudaStream_t s) {
  const lr_model &m = ctx->model;
  const CacheRows w = {slots, (int64_t)n_tokens * m.n_kv_heads, c.n_pages * kPage, k_stride, v_stride, m.n_kv_heads, status};
  const int64_t grid = (w.n_rows * (m.head_dim / 16) + kThreads - 1) / kThreads;
  if (grid > 0x7FFFFFFF) {
    set_error("%s: too many rows in one call", write ? "lr_fp8_write" : "lr_fp8_read");
    return LR_EUNSUPPORTED;
  }
  auto *kp = reinterpret_cast<uint16_t *>(k), *vp = reinterpret_cast<uint16_t *>(v);
  auto *kc = reinterpret_cast<uint8_t *>(c.k_d), *vc = reinterpret_cast<uint8_t *>(c.v_d);
  ctx->launches++;
  if (write)
    return cuda_fail(launch_dependent(m.head_dim == 128 ? fp8_write_kernel<128> : fp8_write_kernel<64>, dim3((unsigned)grid), dim3(kThreads), 0, s, w, kp, vp,
                                      kc, vc, c.k_scale_d, c.v_scale_d),
                     "fp8_write_kernel launch");
  return cuda_fail(launch_dependent(m.head_dim == 128 ? fp8_read_kernel<128> : fp8_read_kernel<64>, dim3((unsigned)grid), dim3(kThreads), 0, s, w, kp, vp, kc,
                                    vc, c.k_scale_d, c.v_scale_d),
                   "fp8_read_kernel launch");
}

}  // namespace lr
