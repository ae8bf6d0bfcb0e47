// Stochastic token-level acceptance of drafts that a draft model sampled: the target's rows P and the drafter's rows Q.
//
// Two kernels.  drafted_stats_kernel streams all rows of both matrices once, a warp a chunk at a time, and leaves the pairs (M_c, S_c)
// of the chunks (accept_stats.cuh): bound by HBM.  drafted_walk_kernel takes a cluster of eight CTAs a branch:
//   1. its warps take the branch's rows in turn: the pairs of a row of P and of Q into (m, Z), P(d), Q(d), and whether the draft is
//      refused, u Q(d) >= P(d).  A warp remembers its first refused row; the smallest of all is the row the walk stops at, and its (m, Z) come from the
//      warp that has them.  A branch of fewer rows than a CTA has warps is gone through by every CTA alone, a longer one by all together and a cluster
//      barrier;
//   2. the weights max(0, P - Q) over that row (or P, behind a full match): a CTA sums an eighth of the vocabulary, 256 tokens a step,
//      the sums of the steps staying in shared memory.  Their total and the inverse CDF need all CTAs' sums: a cluster barrier;
//   3. the CTA whose share holds u_final * total finds the step from the sums, then the token by computing the step's weights again.
// The second read of the stop rows mostly hits L2.  As one CTA a branch the walk over 152 K tokens would keep 3 to 55 SMs busy for
// ten microseconds; a cluster has the reductions without a trip through global memory or a launch of their own.
// Weights are fp32; the sums of steps, CTAs and the scan for the token are in 64 bits and of fixed order: same inputs, same outputs.
//
// Measured, 152 K tokens: 65 branches of up to 16 drafts 84 us, of which the stream over the rows is 70 (its bytes at the copy rate: 58); 3 branches 17 us, bound by
// the walk's chain of trips to memory.  Weights two at a time in packed fp32 and CTAs of 1024 threads where there are SMs for them brought the
// first from 107 and the second from 26.
#include <algorithm>

#include "accept_stats.cuh"

namespace lr {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCtasPerSm = 4;
constexpr int kCluster = 8;
constexpr int kTokens = 256;       // a step: 8 tokens a lane
constexpr int kMaxSteps = 4096;    // of a CTA: 16 KB of sums
constexpr int kAhead = 2;          // steps a warp has in flight: with more the weights spill (64 registers for four CTAs an SM)

struct Rows {  // a matrix of logits, and log2(e) / T
  const uint16_t *logits;
  int64_t stride;
  float k_log2;
};

// ---- cluster ---------------------------------------------------------------------------
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank) {  // the address of a shared variable in another CTA of the cluster
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ int32_t ld_cluster_i32(uint32_t a) {
  int32_t v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t a) { return __int_as_float(ld_cluster_i32(a)); }
__device__ __forceinline__ double ld_cluster_f64(uint32_t a) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
  return v;
}

__global__ void __launch_bounds__(kThreads, kCtasPerSm)
drafted_stats_kernel(Rows p, Rows q, uint32_t n_rows, int32_t vocab, uint32_t n_chunks, int steps, uint32_t total, float2 *__restrict__ stats) {
  const int lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the logits may come from the kernel launched just before
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5); unit < total; unit += gridDim.x * kWarps) {
    const uint32_t row = unit / n_chunks;
    const bool drafter = row >= n_rows;
    const uint16_t *rp = drafter ? q.logits + (int64_t)(row - n_rows) * q.stride : p.logits + (int64_t)row * p.stride;
    const float2 pair = chunk_pair(rp, vocab, (int32_t)(unit - row * n_chunks) * steps * (kStep / 8) + lane, steps, drafter ? q.k_log2 : p.k_log2);
    if (lane == 0) stats[unit] = pair;
  }
}

struct RowSum {  // softmax statistics of a row: largest logit, 1 / sum exp((x - m) / T) (0 for a row of -inf)
  float m, inv;
};

// by a whole warp, from the chunk pairs in order.  The pairs come from the kernel before.
struct RowPairs {
  float2 v[kMaxChunks / 32];
  __device__ __forceinline__ void load(const float2 *st, int n_chunks, int lane) {
#pragma unroll
    for (int k = 0; k < kMaxChunks / 32; ++k) v[k] = k * 32 + lane < n_chunks ? ld_behind_wait(st + k * 32 + lane) : make_float2(-INFINITY, 0.f);
  }
  __device__ __forceinline__ RowSum sum(float k_log2) const {
    float m = -INFINITY, z = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxChunks / 32; ++k) m = fmaxf(m, v[k].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
#pragma unroll
    for (int k = 0; k < kMaxChunks / 32; ++k)
      if (v[k].y > 0.f) z += v[k].y * exp2f((v[k].x - m) * k_log2);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, o);
    return RowSum{m, z > 0.f ? 1.0f / z : 0.f};
  }
};

__device__ __forceinline__ float share(float x, RowSum r, float k_log2) {  // the probability of a logit
  return x > -INFINITY ? exp2f((x - r.m) * k_log2) * r.inv : 0.f;
}

struct Stop {  // the row a warp would stop at
  int32_t i;
  RowSum p, q;
};

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// The rows the final token is drawn from, and their weights.
struct Weights {
  const uint16_t *pr, *qr;  // qr: null for P alone
  RowSum p, q;
  float kp, kq;
  int32_t vocab;
  __device__ __forceinline__ void alone() {  // P without Q
    qr = nullptr;
    q = RowSum{0.f, 0.f};
  }
  __device__ __forceinline__ void load(int32_t vi, uint4 &a, uint4 &b) const {  // eight logits of each; -inf behind the last
    b = make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
    if (vi < (vocab >> 3)) {
      a = __ldg(reinterpret_cast<const uint4 *>(pr) + vi);
      if (qr != nullptr) b = __ldg(reinterpret_cast<const uint4 *>(qr) + vi);
    } else {
      a = tail(pr, vi);
      if (qr != nullptr) b = tail(qr, vi);
    }
  }
  __device__ __forceinline__ uint4 tail(const uint16_t *row, int32_t vi) const {
    uint32_t t[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int32_t e = vi * 8 + 2 * j;
      t[j] = (e < vocab ? (uint32_t)row[e] : 0xFF80u) | (e + 1 < vocab ? (uint32_t)row[e + 1] : 0xFF80u) << 16;
    }
    return make_uint4(t[0], t[1], t[2], t[3]);
  }
  // max(0, P - Q) of two tokens; Q's row may be all -inf (load) with q = {0, 0}.  x - m is exact near the maximum, whatever the logits' size; a NaN of P falls to the
  // maximum with 0.  Below 2^-126 of the largest there is no weight.
  __device__ __forceinline__ float2 weight2(uint32_t a, uint32_t b) const {
    const float2 x = mul2(add2(make_float2(bf_lo(a), bf_hi(a)), make_float2(-p.m, -p.m)), make_float2(kp, kp));
    const float2 y = mul2(add2(make_float2(denan(bf_lo(b)), denan(bf_hi(b))), make_float2(-q.m, -q.m)), make_float2(kq, kq));
    // (not as one fused operation: where the rows are equal the difference has to be 0, not what a rounding left)
    const float2 w = add2(mul2(make_float2(ex2_approx(x.x), ex2_approx(x.y)), make_float2(p.inv, p.inv)),
                          mul2(make_float2(ex2_approx(y.x), ex2_approx(y.y)), make_float2(-q.inv, -q.inv)));
    return make_float2(fmaxf(w.x, 0.f), fmaxf(w.y, 0.f));
  }
  __device__ __forceinline__ float mass(const uint4 &a, const uint4 &b) const {  // of the eight tokens of a vector
    const float2 w = add2(add2(weight2(a.x, b.x), weight2(a.y, b.y)), add2(weight2(a.z, b.z), weight2(a.w, b.w)));
    return w.x + w.y;
  }
  __device__ __forceinline__ void weigh(const uint4 &a, const uint4 &b, float (&w)[8]) const {  // one by one
    const float2 t[4] = {weight2(a.x, b.x), weight2(a.y, b.y), weight2(a.z, b.z), weight2(a.w, b.w)};
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = (j & 1) != 0 ? t[j / 2].y : t[j / 2].x;
  }
};

__device__ __forceinline__ double shfl_up_f64(double x, int o) {
  return __hiloint2double(__shfl_up_sync(0xFFFFFFFFu, __double2hiint(x), o), __shfl_up_sync(0xFFFFFFFFu, __double2loint(x), o));
}
__device__ __forceinline__ double shfl_f64(double x, int l) {
  return __hiloint2double(__shfl_sync(0xFFFFFFFFu, __double2hiint(x), l), __shfl_sync(0xFFFFFFFFu, __double2loint(x), l));
}
__device__ __forceinline__ double warp_sum_f64(double x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    x += __hiloint2double(__shfl_xor_sync(0xFFFFFFFFu, __double2hiint(x), o), __shfl_xor_sync(0xFFFFFFFFu, __double2loint(x), o));
  return x;
}

// Where the running sum of a warp's 32 weights first exceeds `target`, having been `before` ahead of them: the lane, or -1; `before` moves to
// the sum ahead of that lane (or behind all).  `last`: the last lane that has any weight, or -1.
__device__ __forceinline__ int find_lane(double w, double target, double &before, int &last, int lane) {
  double t = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double y = shfl_up_f64(t, o);
    if (lane >= o) t += y;
  }
  t += before;
  const unsigned some = __ballot_sync(0xFFFFFFFFu, w > 0.0), hit = __ballot_sync(0xFFFFFFFFu, w > 0.0 && t > target);
  last = some != 0u ? 31 - __clz(some) : -1;
  if (hit == 0u) {
    before = shfl_f64(t, 31);
    return -1;
  }
  const int l = __ffs(hit) - 1;
  before = shfl_f64(t - w, l);
  return l;
}

// cluster b of kCluster CTAs: branch b.  per_step: tokens of a step, kTokens or a multiple; steps: of a CTA.
template <int kWalk>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kWalk, 1024 / kWalk)
drafted_walk_kernel(Rows tp, Rows tq, int32_t vocab, const float2 *stats, int32_t n_rows, int n_chunks, int32_t per_step, int32_t steps,
                    const int32_t *__restrict__ draft_ids, const int32_t *__restrict__ cu_draft, const float *__restrict__ u_accept,
                    const float *__restrict__ u_final, int32_t *__restrict__ n_accept, int32_t *__restrict__ final_id, float *__restrict__ p_draft,
                    float *__restrict__ q_draft) {
  constexpr int kTeam = kWalk / 32;
  extern __shared__ float s_step[];  // [steps]: the weight of each step of this CTA
  __shared__ Stop s_stop[kTeam];
  __shared__ double s_total[2];      // this CTA's weight, of either attempt
  __shared__ Stop s_at;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x / kCluster, rank = blockIdx.x % kCluster;
  // Only the statistics come from the kernel launched just before, and that kernel let this one start when everything older
  // had finished: all else is fetched while it drains.
  const int32_t d0 = cu_draft[b], L = cu_draft[b + 1] - d0, r0 = d0 + b;
  const float u_fin = u_final[b];

  // ---- 1. the rows of the branch
  Stop mine;
  mine.i = 0x7FFFFFFF;
  mine.p = mine.q = RowSum{0.f, 0.f};
  bool waited = false;
  const bool few = L < kTeam;  // every CTA looks at all rows itself, which saves the wait for the others
  for (int32_t i = (few ? 0 : rank * kTeam) + warp; i <= L; i += kCluster * kTeam) {
    float xd = -INFINITY, yd = -INFINITY, u = 0.f;
    if (i < L) {
      const int32_t d = draft_ids[d0 + i];
      u = u_accept[d0 + i];
      if (d >= 0 && d < vocab) {
        xd = denan(bf_lo((uint32_t)tp.logits[(int64_t)(r0 + i) * tp.stride + d]));
        yd = denan(bf_lo((uint32_t)tq.logits[(int64_t)(d0 + i) * tq.stride + d]));
      }
    }
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    waited = true;
    RowPairs a, c;
    a.load(stats + (int64_t)(r0 + i) * n_chunks, n_chunks, lane);
    if (i < L) c.load(stats + ((int64_t)n_rows + d0 + i) * n_chunks, n_chunks, lane);
    Stop row;
    row.i = i;
    row.p = a.sum(tp.k_log2);
    row.q = RowSum{0.f, 0.f};
    bool refused = true;  // the row behind the last draft
    if (i < L) {
      row.q = c.sum(tq.k_log2);
      const float p = share(xd, row.p, tp.k_log2), q = share(yd, row.q, tq.k_log2);
      refused = !(u * q < p);
      if (lane == 0 && !(few && rank != 0)) {
        if (p_draft != nullptr) p_draft[d0 + i] = p;
        if (q_draft != nullptr) q_draft[d0 + i] = q;
      }
    }
    if (refused && mine.i == 0x7FFFFFFF) mine = row;
  }
  if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (lane == 0) s_stop[warp] = mine;
  if (few) __syncthreads();
  else cluster_barrier();
  if (warp == 0) {  // the first refused row of the cluster's warps
    int32_t best = 0x7FFFFFFF;
    uint32_t at = 0;
    const int warps = few ? kTeam : kCluster * kTeam;  // of this CTA alone, or of all
#pragma unroll
    for (int k = 0; k < kCluster * kTeam / 32; ++k) {
      const int w = k * 32 + lane;
      if (w < warps) {
        const uint32_t from = in_cta(&s_stop[w % kTeam], few ? rank : w / kTeam);
        const int32_t i = ld_cluster_i32(from);
        if (i < best) {
          best = i;
          at = from;
        }
      }
    }
    const int32_t n = __reduce_min_sync(0xFFFFFFFFu, best);
    if (best == n) {  // one lane: a row is one warp's, and a warp is looked at once
      s_at.i = n;
      s_at.p.m = ld_cluster_f32(at + 4);
      s_at.p.inv = ld_cluster_f32(at + 8);
      s_at.q.m = ld_cluster_f32(at + 12);
      s_at.q.inv = ld_cluster_f32(at + 16);
    }
  }
  __syncthreads();
  const int32_t n = s_at.i;
  Weights wt;
  wt.vocab = vocab;
  wt.pr = tp.logits + (int64_t)(r0 + n) * tp.stride;
  wt.qr = tq.logits + (int64_t)(d0 + n) * tq.stride;
  wt.p = s_at.p;
  wt.q = s_at.q;
  if (n == L || !(wt.q.inv > 0.f)) wt.alone();  // behind a full match, and where Q's row is all -inf
  wt.kp = tp.k_log2;
  wt.kq = tq.k_log2;
  const int sub = per_step / kTokens;

  // ---- 2. the weights, once more from P alone where P - Q leaves nothing
  for (int attempt = 0;; ++attempt) {
    const int32_t s0 = rank * steps;
    for (int32_t at = warp; at < steps; at += kTeam * kAhead) {
      float sum[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) sum[k] = 0.f;
      for (int j = 0; j < sub; ++j) {
        uint4 x[kAhead], y[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int64_t vi = ((int64_t)(s0 + at + k * kTeam) * sub + j) * 32 + lane;
          x[k] = y[k] = make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
          if (at + k * kTeam < steps && vi * 8 < vocab) wt.load((int32_t)vi, x[k], y[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) sum[k] += wt.mass(x[k], y[k]);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], o);
        if (lane == 0 && at + k * kTeam < steps) s_step[at + k * kTeam] = sum[k];
      }
    }
    __syncthreads();
    if (warp == 0) {
      double t = 0.0;
      for (int32_t s = lane; s < steps; s += 32) t += (double)s_step[s];
      t = warp_sum_f64(t);
      if (lane == 0) s_total[attempt] = t;
    }
    cluster_barrier();
    // every warp of every CTA finds the same: the CTAs' weights, whose share holds the target
    const double t = lane < kCluster ? ld_cluster_f64(in_cta(&s_total[attempt], lane)) : 0.0;
    const double total = warp_sum_f64(t);
    if (!(total > 0.0) && attempt == 0) {
      wt.alone();
      continue;
    }
    // ---- 3. the token
    const double target = (double)u_fin * total;
    double before = 0.0;
    int last;
    int owner = find_lane(t, target, before, last, lane);
    const bool past = owner < 0;  // rounding pushed the target past the end: the last token with any weight
    if (past) owner = max(last, 0);
    if (rank == owner && warp == 0) {
      const double goal = past ? 1e300 : target;
      // the step: a lane's share of them, then one by one
      const int32_t each = (steps + 31) / 32, first = lane * each, end = min(first + each, steps);
      double own = 0.0;
      for (int32_t s = first; s < end; ++s) own += (double)s_step[s];
      int l = find_lane(own, goal, before, last, lane);
      const bool late = l < 0;
      if (late) {
        l = max(last, 0);
        before = 0.0;  // (any: the last token with a weight is looked for)
      }
      int32_t step = first;
      double ahead = before, cum = before;
      bool hit = false;
      for (int32_t s = first; s < end; ++s) {
        const double w = (double)s_step[s];
        if (!hit && w > 0.0) {
          step = s;
          ahead = cum;
          cum += w;
          hit = !late && cum > goal;
        }
      }
      step = __shfl_sync(0xFFFFFFFFu, step, l);
      before = shfl_f64(ahead, l);
      int32_t token = 0;  // nothing has any weight: a row of -inf
      bool found = false;
      for (int j = 0; j < sub && !found; ++j) {
        const int64_t vi = ((int64_t)(s0 + step) * sub + j) * 32 + lane;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 0.f;
        if (vi * 8 < vocab) {
          uint4 x, y;
          wt.load((int32_t)vi, x, y);
          wt.weigh(x, y, w);
        }
        double mass = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) mass += (double)w[e];
        l = find_lane(mass, late ? 1e300 : goal, before, last, lane);
        found = l >= 0;
        if (!found) l = last;
        if (l >= 0) {  // within that lane's eight
          double cum = before;
          int pick = -1, end = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (w[e] > 0.f) {
              end = e;
              cum += (double)w[e];
              if (pick < 0 && found && cum > goal) pick = e;
            }
          if (pick < 0) pick = end;
          token = __shfl_sync(0xFFFFFFFFu, (int32_t)(vi * 8) + pick, l);
        }
      }
      if (lane == 0) {
        n_accept[b] = n;
        final_id[b] = token;
      }
    }
    break;
  }
  cluster_barrier();  // nobody leaves while another CTA may still read its sums
}

}  // namespace

size_t accept_drafted_scratch_bytes(int32_t vocab, int32_t n_rows) { return 2 * accept_sample_scratch_bytes(vocab, n_rows); }

int launch_accept_drafted(lr_ctx *ctx, const void *logits, int64_t stride, const void *draft_logits, int64_t draft_stride, const int32_t *drafts,
                          const int32_t *cu_draft, int32_t n_branch, int32_t n_rows, float temperature, float draft_temperature, const float *u_accept,
                          const float *u_final, int32_t *n_accept, int32_t *final_id, float *p_draft, float *q_draft, void *scratch, cudaStream_t s) {
  if (n_rows > 65535) {
    set_error("lr_accept_sample_drafted: more than 65535 logits rows in one call");
    return LR_EUNSUPPORTED;
  }
  const int32_t vocab = ctx->model.vocab;
  const int chunk = chunk_steps(vocab), n_chunks = (int)(((int64_t)vocab + (int64_t)chunk * kStep - 1) / ((int64_t)chunk * kStep));
  const Rows p = {reinterpret_cast<const uint16_t *>(logits), stride, log2_scale(temperature)};
  const Rows q = {reinterpret_cast<const uint16_t *>(draft_logits), draft_stride, log2_scale(draft_temperature)};
  auto *st = reinterpret_cast<float2 *>(scratch);
  const uint32_t total = ((uint32_t)n_rows + (uint32_t)(n_rows - n_branch)) * (uint32_t)n_chunks;  // at most 2 * 65535 * kMaxChunks
  const unsigned grid = std::min((total + kWarps - 1) / kWarps, (uint32_t)(ctx->sm_count * kCtasPerSm));
  int64_t per_step = kTokens, steps;
  for (;; per_step *= 2) {
    steps = ((vocab + per_step - 1) / per_step + kCluster - 1) / kCluster;
    if (steps <= kMaxSteps) break;
  }
  ctx->launches += 2;
  if (int rc = cuda_fail(launch_dependent(drafted_stats_kernel, dim3(grid), dim3(kThreads), 0, s, p, q, (uint32_t)n_rows, vocab, (uint32_t)n_chunks, chunk,
                                          total, st),
                         "drafted_stats_kernel launch"))
    return rc;
  // With an SM for each CTA a CTA of 1024 threads has all of its share of a row on its way at once; more CTAs share SMs, four of 256 each.
  const bool wide = (int64_t)n_branch * kCluster <= ctx->sm_count;
  return cuda_fail(launch_dependent(wide ? drafted_walk_kernel<1024> : drafted_walk_kernel<256>, dim3((unsigned)n_branch * kCluster), dim3(wide ? 1024 : 256), (size_t)steps * sizeof(float), s, p, q, vocab, st,
                                    n_rows, n_chunks, (int32_t)per_step, (int32_t)steps, drafts, cu_draft, u_accept, u_final, n_accept, final_id, p_draft,
                                    q_draft),
                   "drafted_walk_kernel launch");
}

}  // namespace lr
