// K and V rows into the 8-bit cache and back.
//
// A row is (token, K or V, KV head): head_dim bf16 that become head_dim e4m3 codes and one scale byte.  The largest magnitude of a
// row is found on its bf16 bits (for non-negative numbers their order is that of the integers, infinities and NaN at the top), and as the
// scale is a power of two it follows from the exponent and one comparison of the fraction: no division, and the products x 2^-e are
// exact, so a code is one rounding of its value.
//
// Bound by HBM on long prompts, by the chain slot -> address -> data and the launch on a pass's drafts.  A thread has 16 channels, two
// 16-byte loads and one 16-byte store (or the other way round), a row is 8 neighbouring threads (4 with head size 64): the maximum
// takes three shuffles, and the rows of a token, which lie side by side in the projection's output, are read in whole lines.
#include <algorithm>

#include "fp8_cache.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256;

struct Fp8Rows {  // the rows of a call
  const int64_t *slots;
  int64_t n_rows;      // n_tokens * sides * heads
  int64_t n_slots;     // of the cache
  int64_t k_stride, v_stride;
  int32_t heads;
  int32_t *status;
};

struct Fp8Row {
  int64_t token, at;  // at: (page * heads + head) * 16 + place, the row's number in a pool; -1: nothing to do
  int32_t head;
  bool v;
};

__device__ __forceinline__ Fp8Row fp8_row(const Fp8Rows &w, int64_t row) {
  Fp8Row r;
  const int32_t per = 2 * w.heads;
  r.token = row / per;
  const int32_t side = (int32_t)(row - r.token * per);
  r.v = side >= w.heads;
  r.head = r.v ? side - w.heads : side;
  const int64_t slot = w.slots[r.token];
  r.at = -1;
  if (slot >= 0 && slot < w.n_slots) r.at = ((slot / kPage) * w.heads + r.head) * kPage + slot % kPage;
  else if (slot >= 0 && w.status != nullptr) {
    w.status[0] = LR_EBOUNDS;
    w.status[1] = (int32_t)r.token;
  }
  return r;
}

// |x| of two bf16 numbers, as integers
__device__ __forceinline__ uint32_t abs2(uint32_t x) { return x & 0x7FFF7FFFu; }

__device__ __forceinline__ uint32_t codes4(uint32_t a, uint32_t b, float by) {  // four bf16 values times a power of two, as e4m3
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r)
      : "f"(__uint_as_float(a << 16) * by), "f"(__uint_as_float(a & 0xFFFF0000u) * by), "f"(__uint_as_float(b << 16) * by),
        "f"(__uint_as_float(b & 0xFFFF0000u) * by));
  return r;
}

template <int kD>
__global__ void __launch_bounds__(kThreads)
fp8_write_kernel(Fp8Rows w, const uint16_t *__restrict__ k, const uint16_t *__restrict__ v, uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                 uint8_t *__restrict__ k_scale, uint8_t *__restrict__ v_scale) {
  constexpr int kLanes = kD / 16;  // threads a row
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the projection may be the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int part = threadIdx.x % kLanes;
  Fp8Row r;
  r.at = -1;
  if (row < w.n_rows) r = fp8_row(w, row);
  uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (r.at >= 0) {
    const uint16_t *src = (r.v ? v + r.token * w.v_stride : k + r.token * w.k_stride) + r.head * kD + part * 16;
    x[0] = __ldg(reinterpret_cast<const uint4 *>(src));
    x[1] = __ldg(reinterpret_cast<const uint4 *>(src) + 1);
  }
  const uint32_t two = __vmaxu2(__vmaxu2(__vmaxu2(abs2(x[0].x), abs2(x[0].y)), __vmaxu2(abs2(x[0].z), abs2(x[0].w))),
                                __vmaxu2(__vmaxu2(abs2(x[1].x), abs2(x[1].y)), __vmaxu2(abs2(x[1].z), abs2(x[1].w))));
  uint32_t top = max(two & 0xFFFFu, two >> 16);  // bits of the largest magnitude
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  if (r.at < 0) return;
  const bool fine = top < 0x7F80u;
  // top = (1 + m / 128) 2^E: E - 8 brings it below 512, one more where that is above 448 = 1.75 x 256
  const int byte = max((int)(top >> 7) - 8 + ((top & 0x7Fu) > 0x60u ? 1 : 0), kFp8LeastScale);
  const float by = __uint_as_float((uint32_t)(254 - byte) << 23);  // 2^(127 - byte)
  const uint4 c = make_uint4(codes4(x[0].x, x[0].y, by), codes4(x[0].z, x[0].w, by), codes4(x[1].x, x[1].y, by), codes4(x[1].z, x[1].w, by));
  reinterpret_cast<uint4 *>((r.v ? v_pool : k_pool) + r.at * kD)[part] = fine ? c : make_uint4(0, 0, 0, 0);
  if (part == 0) (r.v ? v_scale : k_scale)[r.at] = (uint8_t)(fine ? (uint32_t)byte : kFp8NanScale);
}

__device__ __forceinline__ uint32_t pack2(float2 x, float by) {  // exact: a power of two times at most four bits
  __nv_bfloat162 t = __floats2bfloat162_rn(x.x * by, x.y * by);
  uint32_t u;
  memcpy(&u, &t, 4);
  return u;
}

template <int kD>
__global__ void __launch_bounds__(kThreads)
fp8_read_kernel(Fp8Rows w, uint16_t *__restrict__ k, uint16_t *__restrict__ v, const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                const uint8_t *__restrict__ k_scale, const uint8_t *__restrict__ v_scale) {
  constexpr int kLanes = kD / 16;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;
  const int part = threadIdx.x % kLanes;
  if (row >= w.n_rows) return;
  const Fp8Row r = fp8_row(w, row);
  if (r.at < 0) return;
  const uint4 c = __ldg(reinterpret_cast<const uint4 *>((r.v ? v_pool : k_pool) + r.at * kD) + part);
  const float by = fp8_scale(__ldg((r.v ? v_scale : k_scale) + r.at));
  const uint32_t q[4] = {c.x, c.y, c.z, c.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = pack2(fp8_float2(q[i] & 0xFFFFu), by);
    o[2 * i + 1] = pack2(fp8_float2(q[i] >> 16), by);
  }
  uint4 *dst = reinterpret_cast<uint4 *>((r.v ? v + r.token * w.v_stride : k + r.token * w.k_stride) + r.head * kD + part * 16);
  dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
  dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

}  // namespace

int launch_fp8_move(lr_ctx *ctx, const lr_fp8_cache &c, bool write, void *k, int64_t k_stride, void *v, int64_t v_stride, const int64_t *slots,
                    int32_t n_tokens, int32_t *status, cudaStream_t s) {
  const lr_model &m = ctx->model;
  const Fp8Rows w = {slots, (int64_t)n_tokens * 2 * m.n_kv_heads, c.n_pages * kPage, k_stride, v_stride, m.n_kv_heads, status};
  const int lanes = m.head_dim / 16;
  const int64_t grid = (w.n_rows * lanes + kThreads - 1) / kThreads;
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
