// af_draft_verify: drafted tokens against the target's distribution, from given uniforms.
//
// Two launches.  The first reads rows of logits once, in slices, for the maximum and the sum of exponentials (fp32).  The
// second decides request by request which drafts pass and draws the token after them.
//
// What has to be exact is whole numbers: a comparison u q < p, and the place of u C among running sums C_v of up to
// 10^5 terms, where fp32 would be off by as much as many terms are large.  So a comparison whose sides are within 1e-5 is
// made again from sums in 64 bits, and a draw's sums are in 64 bits throughout.
#include <cooperative_groups.h>

#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCluster = 8;                        // CTAs that draw for one request
constexpr float kNoMax = -INFINITY;
constexpr double kResidualFloor = 0x1p-30;         // a residual with less mass than this is drawn from the target itself

struct RowPart {                                   // a slice of a row: max z, sum exp((z - m) / tau), place of the maximum
  float m, s;
  int32_t at, pad;
};
struct Shape {
  int slices, positions;                           // slices of a row; max_draft + 1
};

__device__ __forceinline__ float load(const LogitRows& x, int64_t row, int v) {
  const int64_t i = row * x.pitch + v;
  return x.type == AF_F32 ? __ldg(static_cast<const float*>(x.p) + i)
                          : __bfloat162float(static_cast<const __nv_bfloat16*>(x.p)[i]);
}

// Drafts of request r: rows [first, first + n) of the drafts, [first + r, first + r + n] of the target.
struct Span { int first, n; bool ok; };
__device__ __forceinline__ Span span_of(const VerifyCall& c, int r) {
  const int a = __ldg(c.cu + r), b = __ldg(c.cu + r + 1);
  const bool ok = a >= 0 && a <= b && b <= c.D && b - a <= c.max_draft;
  return {ok ? a : 0, ok ? b - a : 0, ok};
}

__device__ __forceinline__ RowPart join(const RowPart& a, const RowPart& b, float scale) {
  RowPart o;
  const bool first = a.m > b.m || (a.m == b.m && a.at < b.at);
  o.m = first ? a.m : b.m;
  o.at = first ? a.at : b.at;
  // a part without mass adds nothing (its maximum may be -inf); a NaN stays
  o.s = (a.s == 0.f ? 0.f : a.s * ex2f((a.m - o.m) * scale)) + (b.s == 0.f ? 0.f : b.s * ex2f((b.m - o.m) * scale));
  return o;
}

__device__ RowPart row_part(const LogitRows& x, int64_t row, int lo, int hi, float scale) {
  RowPart a{kNoMax, 0.f, 0x7fffffff, 0};
  for (int v = lo + threadIdx.x; v < hi; v += kThreads) {
    const float z = load(x, row, v);
    if (z > a.m) {
      a.s = a.s == 0.f ? 0.f : a.s * ex2f((a.m - z) * scale);
      a.m = z;
      a.at = v;
    }
    if (z != kNoMax) a.s += ex2f((z - a.m) * scale);         // a NaN, and infinity less itself, make the sum NaN
  }
  __shared__ RowPart part[kWarps];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    RowPart b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
    b.at = __shfl_xor_sync(0xffffffffu, a.at, o);
    a = join(a, b, scale);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
  __syncthreads();
  a = part[0];
  for (int w = 1; w < kWarps; ++w) a = join(a, part[w], scale);
  return a;
}

__global__ void __launch_bounds__(kThreads) verify_rows_kernel(const VerifyCall c, const Shape shape, float scale, RowPart* target_parts,
                                                               RowPart* draft_parts) {
  wait_for_predecessor();
  let_successor_start();
  const int slice = (int)(blockIdx.x % shape.slices), unit = (int)(blockIdx.x / shape.slices);
  const int r = unit % c.R, i = unit / c.R;
  const Span sp = span_of(c, r);
  if (!sp.ok || i > sp.n) return;
  const int lo = (int)((int64_t)c.V * slice / shape.slices), hi = (int)((int64_t)c.V * (slice + 1) / shape.slices);
  const int64_t row = sp.first + r + i;
  const RowPart t = row_part(c.target, row, lo, hi, scale);
  if (threadIdx.x == 0) target_parts[row * shape.slices + slice] = t;
  if (c.draft.p && i < sp.n) {
    const RowPart d = row_part(c.draft, sp.first + i, lo, hi, scale);
    if (threadIdx.x == 0) draft_parts[(int64_t)(sp.first + i) * shape.slices + slice] = d;
  }
}

// A row's distribution from its parts: maximum, its place, and the sum in 64 bits of the parts' sums.
struct Row { float m; int32_t at; double s; };
__device__ __forceinline__ bool good(const Row& x) { return fabsf(x.m) < INFINITY && x.s > 0.0 && x.s < 1e300; }
// Called by a whole warp.
__device__ Row warp_row(const RowPart* parts, int slices, double inv_tau) {
  const int lane = threadIdx.x & 31;
  Row x{kNoMax, 0x7fffffff, 0.0};
  for (int i = lane; i < slices; i += 32) {
    const float m = __ldcg(&parts[i].m);
    const int32_t at = __ldcg(&parts[i].at);
    if (m > x.m || (m == x.m && at < x.at)) { x.m = m; x.at = at; }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m = __shfl_xor_sync(0xffffffffu, x.m, o);
    const int32_t at = __shfl_xor_sync(0xffffffffu, x.at, o);
    if (m > x.m || (m == x.m && at < x.at)) { x.m = m; x.at = at; }
  }
  for (int i = lane; i < slices; i += 32) {
    const float m = __ldcg(&parts[i].m), s = __ldcg(&parts[i].s);
    if (s != 0.f) x.s += (double)s * exp(((double)m - (double)x.m) * inv_tau);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
  return x;
}

__device__ __forceinline__ double weight(const LogitRows& x, int64_t row, int v, float m, double inv_tau) {
  return exp(((double)load(x, row, v) - (double)m) * inv_tau);
}
// Sum over the block, in a fixed order; every thread gets it.
__device__ double block_sum(double a, double* warp_sums) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = a;
  __syncthreads();
  double all = 0.0;
  for (int w = 0; w < kWarps; ++w) all += warp_sums[w];
  return all;
}
__device__ double exact_sum(const LogitRows& x, int64_t row, int lo, int hi, float m, double inv_tau, double* warp_sums) {
  double a = 0.0;
  for (int v = lo + threadIdx.x; v < hi; v += kThreads) a += weight(x, row, v, m, inv_tau);
  return block_sum(a, warp_sums);
}

// A cluster per request.
__global__ void __launch_bounds__(kThreads) verify_draw_kernel(const VerifyCall c, const Shape shape, float scale,
                                                               const RowPart* target_parts, const RowPart* draft_parts,
                                                               unsigned int* d_err) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ double s_warp[kWarps], s_sum[4];                 // s_sum: this CTA's shares, read by the cluster
  __shared__ double s_thread[kThreads];
  __shared__ Row s_target, s_draft;
  wait_for_predecessor();
  let_successor_start();
  const int r = (int)blockIdx.x / kCluster, rank = (int)blockIdx.x % kCluster;
  const int warp = threadIdx.x >> 5;
  const Span sp = span_of(c, r);
  const bool leader = rank == 0 && threadIdx.x == 0;
  if (leader) {
    unsigned int bad = sp.ok ? 0 : AF_DEVERR_CU_SEQLENS;
    if (r == 0 && __ldg(c.cu) != 0) bad |= AF_DEVERR_CU_SEQLENS;
    if (r == c.R - 1 && __ldg(c.cu + c.R) != c.D) bad |= AF_DEVERR_CU_SEQLENS;
    if (bad) atomicOr(d_err, bad);
    if (!sp.ok) c.n_emitted[r] = 0;
  }
  if (!sp.ok) return;                                         // the whole cluster
  const bool greedy = c.temperature == 0.f;
  const double inv_tau = greedy ? 1.0 : 1.0 / (double)c.temperature;
  const int64_t base = sp.first + r;
  const int lo = (int)((int64_t)c.V * rank / kCluster), hi = (int)((int64_t)c.V * (rank + 1) / kCluster);

  // ---- which drafts pass: every CTA of the cluster finds out by itself
  int i = 0;
  bool has_row = true;
  Row t{}, q{};
  for (;; ++i) {
    __syncthreads();
    if (warp == 0) {
      const Row x = warp_row(target_parts + (base + i) * shape.slices, shape.slices, inv_tau);
      if (threadIdx.x == 0) s_target = x;
    } else if (warp == 1 && c.draft.p && i < sp.n) {
      const Row x = warp_row(draft_parts + (int64_t)(sp.first + i) * shape.slices, shape.slices, inv_tau);
      if (threadIdx.x == 32) s_draft = x;
    }
    __syncthreads();
    t = s_target;
    has_row = good(t);
    if (!has_row) break;
    if (i == sp.n) break;
    const int x = __ldg(c.draft_ids + sp.first + i);
    const bool id_ok = x >= 0 && x < c.V;
    if (!id_ok && leader) atomicOr(d_err, AF_DEVERR_TARGET_RANGE);
    bool pass;
    if (greedy) {
      pass = x == t.at;
    } else {
      if (c.draft.p) {
        q = s_draft;
        has_row = good(q);
        if (!has_row) break;
      }
      pass = false;
      if (id_ok) {
        const double u = (double)__ldg(c.u_accept + sp.first + i);
        const double pw = weight(c.target, base + i, x, t.m, inv_tau), qw = c.draft.p ? weight(c.draft, sp.first + i, x, q.m, inv_tau) : 1.0;
        double left = u * qw * t.s, right = pw * (c.draft.p ? q.s : 1.0);      // u q < p, times both sums
        if (fabs(left - right) <= 1e-5 * fabs(right)) {
          t.s = exact_sum(c.target, base + i, 0, c.V, t.m, inv_tau, s_warp);
          if (c.draft.p) q.s = exact_sum(c.draft, sp.first + i, 0, c.V, q.m, inv_tau, s_warp);
          left = u * qw * t.s;
          right = pw * (c.draft.p ? q.s : 1.0);
        }
        pass = left < right;
      }
    }
    if (!pass) break;
    if (leader) {
      c.token[base + i] = x;
      if (c.logp) c.logp[base + i] = (float)(((double)load(c.target, base + i, x) - (double)t.m) * inv_tau - log(t.s));
    }
  }
  if (leader) {
    for (int j = i + 1; j <= sp.n; ++j) {
      c.token[base + j] = -1;
      if (c.logp) c.logp[base + j] = 0.f;
    }
    c.n_emitted[r] = has_row ? i + 1 : i;
    if (!has_row) {
      atomicOr(d_err, AF_DEVERR_DISTRIBUTION);
      c.token[base + i] = -1;
      if (c.logp) c.logp[base + i] = __int_as_float(0x7fc00000);
    }
    if (has_row && greedy) {
      c.token[base + i] = t.at;
      if (c.logp) c.logp[base + i] = (float)-log(t.s);
    }
  }
  if (!has_row || greedy) return;                             // the whole cluster

  // ---- the token after them, from row base + i
  const bool rejected = i < sp.n, dense = rejected && c.draft.p != nullptr;
  const int cut = rejected && !dense ? __ldg(c.draft_ids + sp.first + i) : -1;
  double p_unit = 1.0, q_unit = 1.0;                          // dense: 1 / sums
  double row_sum = 0.0;                                       // of the target's weights
  if (dense) {
    const double a = exact_sum(c.target, base + i, lo, hi, t.m, inv_tau, s_warp);
    const double b = exact_sum(c.draft, sp.first + i, lo, hi, q.m, inv_tau, s_warp);
    if (threadIdx.x == 0) { s_sum[0] = a; s_sum[1] = b; }
    cluster.sync();
    double sum_q = 0.0;
    for (int k = 0; k < kCluster; ++k) {
      row_sum += *cluster.map_shared_rank(&s_sum[0], k);
      sum_q += *cluster.map_shared_rank(&s_sum[1], k);
    }
    p_unit = 1.0 / row_sum;
    q_unit = 1.0 / sum_q;
  }
  // a thread's stretch of the CTA's share
  const int mine_lo = lo + (int)((int64_t)(hi - lo) * threadIdx.x / kThreads), mine_hi = lo + (int)((int64_t)(hi - lo) * (threadIdx.x + 1) / kThreads);
  bool plain = !rejected;                                     // drawn from the target itself
  auto mass = [&](int v) {
    double w = weight(c.target, base + i, v, t.m, inv_tau) * p_unit;
    if (!plain && dense) w = fmax(w - weight(c.draft, sp.first + i, v, q.m, inv_tau) * q_unit, 0.0);
    if (!plain && v == cut) w = 0.0;
    return w;
  };
  double before, total;
  for (;;) {
    double a = 0.0, whole = 0.0;
    for (int v = mine_lo; v < mine_hi; ++v) {
      const double w = mass(v);
      a += w;
      if (!dense) whole += v == cut ? weight(c.target, base + i, v, t.m, inv_tau) : w;
    }
    __syncthreads();
    s_thread[threadIdx.x] = a;
    __syncthreads();
    if (threadIdx.x == 0) {
      double run = 0.0;
      for (int k = 0; k < kThreads; ++k) { const double x = s_thread[k]; s_thread[k] = run; run += x; }
      s_sum[2] = run;
    }
    whole = block_sum(whole, s_warp);
    if (threadIdx.x == 0) s_sum[3] = whole;
    cluster.sync();
    before = total = 0.0;
    double all = 0.0;
    for (int k = 0; k < kCluster; ++k) {
      if (k == rank) before = total;
      total += *cluster.map_shared_rank(&s_sum[2], k);
      all += *cluster.map_shared_rank(&s_sum[3], k);
    }
    cluster.sync();                                           // s_sum is read by all before it is written again, or its CTA ends
    if (!dense) row_sum = all;
    if (plain || (dense ? total : total / row_sum) > kResidualFloor) break;
    plain = true;                                             // next to nothing is left: the target itself
  }
  // the thread whose stretch holds the first v with C_v > u C
  const double u = (double)fminf(fmaxf(__ldg(c.u_sample + r), 0.f), 1.f - 0x1p-24f), goal = u * total;
  const double start = before + s_thread[threadIdx.x];
  const double end = before + (threadIdx.x + 1 < kThreads ? s_thread[threadIdx.x + 1] : s_sum[2]);
  if (start <= goal && goal < end) {
    double at = start;
    int y = mine_lo;
    for (int v = mine_lo; v < mine_hi; ++v) {
      const double w = mass(v);
      if (w > 0.0) y = v;                                     // the last with mass, if rounding leaves the goal beyond the stretch
      at += w;
      if (at > goal) break;
    }
    c.token[base + i] = y;
    if (c.logp) c.logp[base + i] = (float)(((double)load(c.target, base + i, y) - (double)t.m) * inv_tau - log(row_sum));
  }
}

// Slices of a row: enough CTAs for every SM's warps, of 2048 logits at least.
Shape shape_of(int32_t R, int32_t V, int32_t max_draft, int sm_count) {
  const int64_t units = (int64_t)R * (max_draft + 1), want = ((int64_t)sm_count * 8 + units - 1) / units, most = V / 2048;
  const int64_t slices = want < most ? want : most;
  return {(int)(slices < 1 ? 1 : slices), max_draft + 1};
}

}  // namespace

// Rows in several slices are few: fewer than 16 parts per SM in all, and as many of the drafts.  So smaller calls of any
// kind fit in what a larger one needs.
size_t verify_workspace_bytes(int32_t R, int32_t D, int sm_count) {
  const size_t whole_rows = (size_t)R + 2 * (size_t)D, sliced = (size_t)sm_count * 32;
  return (whole_rows > sliced ? whole_rows : sliced) * sizeof(RowPart);
}

af_status launch_draft_verify(af_ctx* ctx, const VerifyCall& c, cudaStream_t s) {
  const af_status st = ws_grow(ctx->verify_ws, verify_workspace_bytes(c.R, c.D, ctx->sm_count));
  if (st != AF_OK) return st;
  const Shape shape = shape_of(c.R, c.V, c.max_draft, ctx->sm_count);
  RowPart* const target_parts = static_cast<RowPart*>(ctx->verify_ws.p);
  RowPart* const draft_parts = target_parts + ((size_t)c.R + c.D) * shape.slices;
  const float scale = c.temperature == 0.f ? kLog2e : kLog2e / c.temperature;
  const int64_t blocks = (int64_t)c.R * shape.positions * shape.slices;
  if (launch_overlapped(verify_rows_kernel, (unsigned)blocks, kThreads, 0, s, c, shape, scale, target_parts, draft_parts) != cudaSuccess)
    return AF_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = (unsigned)c.R * kCluster;
  cfg.blockDim = kThreads;
  cfg.stream = s;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_draw_kernel, c, shape, scale, (const RowPart*)target_parts, (const RowPart*)draft_parts,
                            ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
