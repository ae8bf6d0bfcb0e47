// Whole pages copied from one place of a cache to another, in every layer's pools by one launch.
//
// A page of a layer is one page of each of its pools -- K, V and, in 8 or 4 bits, their scales -- taken as one run of 16-byte units; a CTA copies a part of one pair's
// run, every thread kUnits of them at once.  Bound by HBM: a page is read and written once (four layers of bf16 pages, 718 MB
// read and written: 221 us, 6.5 TB/s; forks of 64 K tokens in four layers of 8 heads of 128: 327 us in bf16, 170 in 8 bits, 96 in 4 bits, of 332, 168 and 88 at the copy rate).  In 4 bits
// such a page is 1088 units, and every second CTA has 64 of them.
#include <algorithm>

#include "lr_common.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 4;         // 16-byte units a thread has in flight
constexpr int kMaxCaches = 32;    // layers in one launch: their pointers are the kernel's arguments (2.6 KB, which take the host a microsecond more than those of one)

struct Pools {
  uint4 *p[4];  // K, V, scales of K, scales of V
};
template <int kCaches>
struct CopyArgs {
  Pools src[kCaches], dst[kCaches];
  int64_t src_pages[kCaches], dst_pages[kCaches];
  int32_t codes, scales;  // units of a page in a pool of K or V, and in one of scales
  int32_t parts;          // CTAs a pair
  int32_t n_pairs;
};

template <int kCaches>
__global__ void __launch_bounds__(kThreads)
copy_pages_kernel(const __grid_constant__ CopyArgs<kCaches> a, const int32_t *__restrict__ src_pages, const int32_t *__restrict__ dst_pages, int32_t *__restrict__ status) {
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the pages may come from the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int pair = blockIdx.x / a.parts, part = blockIdx.x % a.parts, c = blockIdx.y;
  const int64_t from = __ldcg(src_pages + pair), to = __ldcg(dst_pages + pair);
  if (from < 0 || to < 0) return;
  if (from >= a.src_pages[c] || to >= a.dst_pages[c]) {
    if (threadIdx.x == 0 && status != nullptr) {
      status[0] = LR_EBOUNDS;
      status[1] = pair;
    }
    return;
  }
  const int total = 2 * (a.codes + a.scales);
  uint4 x[kUnits];
  uint4 *dst[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int i = (part * kUnits + u) * kThreads + threadIdx.x;
    dst[u] = nullptr;
    if (i < total) {
      const bool code = i < 2 * a.codes;
      const int size = code ? a.codes : a.scales, j = code ? i : i - 2 * a.codes, second = j >= size ? 1 : 0, pool = (code ? 0 : 2) + second;
      const int at = j - second * size;
      x[u] = __ldcg(a.src[c].p[pool] + from * size + at);
      dst[u] = a.dst[c].p[pool] + to * size + at;
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
    if (dst[u] != nullptr) *dst[u] = x[u];
}

}  // namespace

int launch_copy_pages(lr_ctx *ctx, const lr_kv_cache *src, const lr_kv_cache *dst, int32_t n_caches, const int32_t *src_pages, const int32_t *dst_pages,
                      int32_t n_pairs, int32_t *status, cudaStream_t s) {
  const lr_model &m = ctx->model;
  const int64_t rows = (int64_t)m.n_kv_heads * kPage;
  const int kind = src[0].kind;
  const int64_t codes = rows * (kind == LR_KV_BF16 ? m.head_dim * 2 : kind == LR_KV_FP8 ? m.head_dim : m.head_dim / 2) / 16;
  const int64_t scales = kind == LR_KV_BF16 ? 0 : rows * (kind == LR_KV_FP8 ? 1 : m.head_dim / 32) / 16;
  const int64_t parts = (2 * (codes + scales) + kThreads * kUnits - 1) / (kThreads * kUnits);
  if (2 * (codes + scales) > (1 << 30) || parts * n_pairs > 0x7FFFFFFF) {
    set_error("lr_copy_pages: too many pages in one call");
    return LR_EUNSUPPORTED;
  }
  auto launch = [&](auto a, int c0, int n) {
    for (int c = 0; c < n; ++c) {
      const lr_kv_cache &from = src[c0 + c], &to = dst[c0 + c];
      a.src[c] = {{(uint4 *)from.k_d, (uint4 *)from.v_d, (uint4 *)from.k_scale_d, (uint4 *)from.v_scale_d}};
      a.dst[c] = {{(uint4 *)to.k_d, (uint4 *)to.v_d, (uint4 *)to.k_scale_d, (uint4 *)to.v_scale_d}};
      a.src_pages[c] = from.n_pages;
      a.dst_pages[c] = to.n_pages;
    }
    a.codes = (int32_t)codes;
    a.scales = (int32_t)scales;
    a.parts = (int32_t)parts;
    a.n_pairs = n_pairs;
    ctx->launches++;
    return cuda_fail(launch_dependent(copy_pages_kernel<(int)(sizeof(a.src) / sizeof(Pools))>, dim3((unsigned)(parts * n_pairs), (unsigned)n), dim3(kThreads), 0, s, a, src_pages,
                                      dst_pages, status),
                     "copy_pages_kernel launch");
  };
  for (int c0 = 0; c0 < n_caches; c0 += kMaxCaches) {
    const int n = std::min(kMaxCaches, n_caches - c0);
    if (int rc = n == 1 ? launch(CopyArgs<1>{}, c0, n) : launch(CopyArgs<kMaxCaches>{}, c0, n)) return rc;
  }
  return LR_OK;
}

}  // namespace lr
