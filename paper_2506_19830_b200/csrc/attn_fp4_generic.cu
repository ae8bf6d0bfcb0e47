// CUDA-core nested-prefix attention over the 4-bit cache: the path for shapes the tensor-core kernel does not take, and an on-device
// cross-check of it.  One warp per (query row, query head), 32 keys at a time: a lane scores one key -- the dot products of 32 channels with
// their codes, each times the group's scale -- the warp combines them with shuffle reductions into a running (max, sum) in fp32, and the lanes then share the value
// rows, head_dim/32 channels each.  Everything is fp32 up to the output.  A key whose row of K or V stands for NaN has a score that is no number, and
// with it the row's sum.
#include "fp4_cache.cuh"

namespace lr {

namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32)
attn_fp4_generic_kernel(DevBatch d, const uint16_t *__restrict__ q, const uint8_t *__restrict__ kpool, const uint8_t *__restrict__ vpool,
                        const uint8_t *__restrict__ kscale, const uint8_t *__restrict__ vscale, uint16_t *__restrict__ out, float *__restrict__ lse,
                        float scale_log2) {
  constexpr int EPL = D / 32;  // output channels per lane
  __shared__ float sq[kWarps][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t wg = (int64_t)blockIdx.x * kWarps + warp;
  if (wg >= (int64_t)d.n_q_rows * d.n_q_heads) return;
  const int row = (int)(wg / d.n_q_heads), h = (int)(wg % d.n_q_heads), kv = h / d.group;

  int lo = 0, hi = d.n_branch - 1;  // branch of this row: largest b with cu_q[b] <= row
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (d.cu_q[mid] <= row) lo = mid; else hi = mid - 1;
  }
  const int b = lo;
  const int i = row - d.cu_q[b], q_len = d.cu_q[b + 1] - d.cu_q[b];
  const int s0 = d.req_span_off[d.br_req[b]], n_seg = d.req_span_off[d.br_req[b] + 1] - s0 - 1;
  const int node = d.span_tin[s0 + d.br_depth[b]];  // depth-first number of the node the branch continues
  const int tail_vis = d.br_own_len[b] - q_len + i + 1;  // the query sees itself

  const uint16_t *qp = q + ((int64_t)row * d.n_q_heads + h) * D;
  for (int e = lane; e < D; e += 32) sq[warp][e] = __uint_as_float((uint32_t)qp[e] << 16);
  __syncwarp();

  float m = -INFINITY, l = 0.f, acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;

  for (int sp = 0; sp <= n_seg + 1; ++sp) {  // prefix, the segments the node descends from (index order), tail
    if (sp <= n_seg && (node < d.span_tin[s0 + sp] || node > d.span_last[s0 + sp])) continue;
    const int slot0 = (sp <= n_seg) ? d.span_slot[s0 + sp] : d.br_own_slot[b];
    const int len = (sp <= n_seg) ? d.span_len[s0 + sp] : tail_vis;
    for (int t0 = 0; t0 < len; t0 += 32) {
      const int t = t0 + lane;
      bool valid = t < len;
      int64_t at = 0;  // the key's row in the pools
      if (valid) {
        int64_t page = d.page_ids[slot0 + t / kPage];
        if (page < 0 || page >= d.n_pool_pages) {  // never dereference a page outside the pool
          d.status[0] = kDevBounds;
          d.status[1] = 110;
          page = 0;
          valid = false;
        }
        at = (page * d.n_kv_heads + kv) * kPage + (t % kPage);
      }
      float s = -INFINITY;
      if (valid) {
        s = 0.f;
#pragma unroll
        for (int g = 0; g < D / kFp4Group; ++g) {
          const uint4 kk = __ldcg(reinterpret_cast<const uint4 *>(kpool + at * (D / 2)) + g);
          const uint32_t w[4] = {kk.x, kk.y, kk.z, kk.w};
          float a0 = 0.f, a1 = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float *qq = &sq[warp][g * kFp4Group + j * 8];
            float x[8];
            fp4_floats(w[j], x);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              a0 = fmaf(qq[i], x[i], a0);
              a1 = fmaf(qq[i + 1], x[i + 1], a1);
            }
          }
          const uint32_t vb = ld_scale(vscale + at * (D / kFp4Group) + g);
          s = fmaf(a0 + a1, fp8_scale(vb == kFp4NanScale ? kFp4NanScale : ld_scale(kscale + at * (D / kFp4Group) + g)), s);
        }
        s *= scale_log2;
      }
      const float bm = warp_max(s);  // (a NaN score is not the largest: it comes back through the sum)
      const float m_new = fmaxf(m, bm);
      const float ref = m_new > -INFINITY ? m_new : 0.f;
      const float p = valid ? exp2f(s - ref) : 0.f;
      const float corr = m > -INFINITY ? exp2f(m - ref) : 0.f;
      l = l * corr + warp_sum(p);
#pragma unroll
      for (int e = 0; e < EPL; ++e) acc[e] *= corr;
      const unsigned live = __ballot_sync(0xFFFFFFFFu, valid);
      const int n = min(32, len - t0);
      for (int j = 0; j < n; ++j) {
        const float pj = __shfl_sync(0xFFFFFFFFu, p, j);
        const int64_t aj = __shfl_sync(0xFFFFFFFFu, (long long)at, j);
        if (!((live >> j) & 1u)) continue;
        // the lane's channels lane * EPL .. + EPL - 1 of their word of eight
        const uint32_t vv = __ldcg(reinterpret_cast<const uint32_t *>(vpool + aj * (D / 2)) + lane * EPL / 8);
        const float by = pj * fp8_scale(ld_scale(vscale + aj * (D / kFp4Group) + lane * EPL / kFp4Group));
        float x[8];
        fp4_floats(vv, x);
        const int first = lane * EPL % 8;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          float y = x[e];
#pragma unroll
          for (int f = EPL; f < 8; f += EPL)
            if (first == f) y = x[f + e];
          acc[e] = fmaf(by, y, acc[e]);
        }
      }
      m = m_new;
    }
  }
  const float inv = 1.f / l;
  uint16_t *op = out + ((int64_t)row * d.n_q_heads + h) * D + lane * EPL;
#pragma unroll
  for (int e = 0; e < EPL; e += 2) {
    __nv_bfloat162 o2 = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
    *reinterpret_cast<uint32_t *>(op + e) = *reinterpret_cast<uint32_t *>(&o2);
  }
  if (lse != nullptr && lane == 0) lse[(int64_t)row * d.n_q_heads + h] = (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

int launch_attn_fp4_generic(lr_plan *p, const void *q, const lr_fp4_cache &c, void *out, float *lse, float scale, cudaStream_t s) {
  const DevBatch &d = p->dev;
  const int64_t warps = (int64_t)d.n_q_rows * d.n_q_heads;
  const unsigned grid = (unsigned)((warps + kWarps - 1) / kWarps);
  p->ctx->launches++;
  return cuda_fail(launch_dependent(d.head_dim == 128 ? attn_fp4_generic_kernel<128> : attn_fp4_generic_kernel<64>, dim3(grid), dim3(kWarps * 32), 0, s, d,
                                    reinterpret_cast<const uint16_t *>(q), reinterpret_cast<const uint8_t *>(c.k_d), reinterpret_cast<const uint8_t *>(c.v_d),
                                    c.k_scale_d, c.v_scale_d, reinterpret_cast<uint16_t *>(out), lse, scale * 1.4426950408889634f),
                   "attn_fp4_generic_kernel launch");
}

}  // namespace lr
