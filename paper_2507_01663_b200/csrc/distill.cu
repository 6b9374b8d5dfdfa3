// af_distill_loss: divergence between a teacher's and the student's log-probs of K listed ids per token,
// and its gradient in the student's log-probs, in one pass (8 bytes read and 4 written per slot: HBM-bound).
//
// kG lanes of a warp share a row and hold kElems of its slots each, so a row's sums and maxima are a few
// shuffles inside the group and every value is read once.  At full bandwidth an SM takes about two slots
// per clock, which leaves some 60 thread instructions for each: eight slots per lane keep the shuffles of up
// to five row reductions at a few instructions per slot.  A CTA walks a contiguous range of rows, so a
// token's sequence (its weight in the mean) is nearly always the previous one's.
// Row sums are taken in fp32 over at most 256 terms in a fixed tree, the batch's in fp64 in a fixed order:
// results are bit-reproducible.
#include "common.cuh"
#include "device_util.cuh"

namespace af {
namespace {

constexpr int kThreads = 256;
constexpr int kElems = 8;                  // slots per lane
constexpr int kNumSums = 3;                // weighted loss, teacher mass, student mass
constexpr float kTailFloor = 1.f / 65536.f;

struct DistillWs {                         // the header and blocks of the policy loss's reduction workspace
  unsigned int ticket;
  unsigned int pad[15];
};
__device__ __forceinline__ double* ws_partial(DistillWs* ws, int block) {
  return reinterpret_cast<double*>(ws + 1) + (size_t)block * 4;
}

template <int kG>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = kG / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int kG>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = kG / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

template <int kVec>
__device__ __forceinline__ void load_slots(const float* __restrict__ p, float* v) {
  if constexpr (kVec == 4) {
    const float4 q = __ldcs(reinterpret_cast<const float4*>(p));
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else if constexpr (kVec == 2) {
    const float2 q = __ldg(reinterpret_cast<const float2*>(p));
    v[0] = q.x; v[1] = q.y;
  } else {
    v[0] = __ldg(p);
  }
}
template <int kVec>
__device__ __forceinline__ void store_slots(float* p, const float* v) {
  if constexpr (kVec == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  else if constexpr (kVec == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  else *p = v[0];
}

// The divergence of one row and its gradient: lane `lane` of the group holds the slots lt / lq (absent ones
// and those past K with lt = -inf).  Returns the row's loss (all lanes); g receives dloss/dlq; tm and sm gain
// the lane's share of the teacher's and the student's mass.
template <int kSupport, int kG>
__device__ __forceinline__ float row_divergence(const float (&lt)[kElems], const float (&lq)[kElems], bool forward,
                                                float tau, float inv_tau, float (&g)[kElems], float& tm, float& sm) {
  if constexpr (kSupport == 1) {
    // a = softmax(lt / tau), b = softmax(lq / tau) over the present slots; d = log a - log b
    float ma = -INFINITY, mb = -INFINITY;
#pragma unroll
    for (int i = 0; i < kElems; ++i) {
      ma = fmaxf(ma, lt[i]);
      mb = lt[i] == -INFINITY ? mb : fmaxf(mb, lq[i]);
    }
    ma = group_max<kG>(ma);
    mb = group_max<kG>(mb);
    if (ma == -INFINITY) {          // no slot is present (uniform in the group; the other reductions use no lane of it)
      ma = 0.f; mb = 0.f;
    }
    const float c = kLog2e * inv_tau;
    float a[kElems], za = 0.f, zb = 0.f;
#pragma unroll
    for (int i = 0; i < kElems; ++i) {
      const bool on = lt[i] != -INFINITY;
      a[i] = on ? ex2f((lt[i] - ma) * c) : 0.f;
      g[i] = on ? ex2f((lq[i] - mb) * c) : 0.f;
      za += a[i];
      zb += g[i];
      if (tau != 1.f && on) { tm += ex2f(lt[i] * kLog2e); sm += ex2f(lq[i] * kLog2e); }
    }
    if (tau == 1.f) { tm = fmaf(ex2f(ma * kLog2e), za, tm); sm = fmaf(ex2f(mb * kLog2e), zb, sm); }
    za = group_sum<kG>(za);
    zb = group_sum<kG>(zb);
    const float ia = za > 0.f ? 1.f / za : 0.f, ib = zb > 0.f ? 1.f / zb : 0.f;
    const float shift = za > 0.f ? fmaf(mb - ma, inv_tau, logf(zb * ia)) : 0.f;   // log of the ratio of the sums
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < kElems; ++i) {
      const float d = fmaf(lt[i] - lq[i], inv_tau, shift);
      const float b = g[i] * ib;
      a[i] *= ia;
      if (forward) {
        loss += a[i] > 0.f ? a[i] * d : 0.f;
        g[i] = tau * (b - a[i]);
      } else {
        loss -= b > 0.f ? b * d : 0.f;
        a[i] = d;
        g[i] = tau * b;
      }
    }
    loss = group_sum<kG>(loss);
    if (!forward) {
#pragma unroll
      for (int i = 0; i < kElems; ++i) g[i] = g[i] > 0.f ? g[i] * (-a[i] - loss) : 0.f;
    }
    return tau * tau * loss;
  } else {
    float loss = 0.f, ps = 0.f, qs = 0.f;
    float q[kElems];
#pragma unroll
    for (int i = 0; i < kElems; ++i) {
      const bool on = lt[i] != -INFINITY;
      const float p = on ? ex2f(lt[i] * kLog2e) : 0.f;
      q[i] = on ? ex2f(lq[i] * kLog2e) : 0.f;
      const float gap = lt[i] - lq[i];
      ps += p;
      qs += q[i];
      if (forward) {
        loss += p > 0.f ? p * gap : 0.f;
        g[i] = -p;
      } else {
        loss -= q[i] > 0.f ? q[i] * gap : 0.f;
        g[i] = q[i] > 0.f ? q[i] * (1.f - gap) : 0.f;
      }
    }
    tm += ps;
    sm += qs;
    if constexpr (kSupport == 2) {
      // one more outcome holds what the listed ones leave of either distribution
      ps = group_sum<kG>(ps);
      qs = group_sum<kG>(qs);
      const float q_left = 1.f - qs;
      const float pr = fmaxf(1.f - ps, kTailFloor), qr = fmaxf(q_left, kTailFloor);
      const bool free = q_left > kTailFloor;
      const float ratio = logf(pr / qr);
      const float slope = !free ? 0.f : forward ? pr / qr : ratio - 1.f;
#pragma unroll
      for (int i = 0; i < kElems; ++i) g[i] = fmaf(q[i], slope, g[i]);
      return group_sum<kG>(loss) + (forward ? pr * ratio : -qr * ratio);
    }
    return group_sum<kG>(loss);
  }
}

template <int kSupport, int kG, int kVec>
__global__ void __launch_bounds__(kThreads) distill_loss_kernel(
    const float* __restrict__ cand_logp, const float* __restrict__ teacher_logp, const int32_t* __restrict__ cu, int B,
    int T, int t0, int rows, int K, af_distill_params prm, af_distill_out* __restrict__ out,
    float* __restrict__ token_loss, float* __restrict__ dcand, DistillWs* ws, unsigned int* d_err) {
  constexpr int kRows = kThreads / kG;              // rows of a CTA's step
  const int sub = threadIdx.x / kG, lane = threadIdx.x % kG;
  const float tau = prm.temperature, inv_tau = 1.f / prm.temperature;
  const bool forward = prm.divergence == 0;
  const float w_all = prm.agg_mode == 0 ? (B > 0 ? prm.loss_scale / (float)B : 0.f)
                                        : (T > 0 ? prm.loss_scale / (float)T : 0.f);
  if (out)      // as in the policy loss: entries out of order raise the flag, nothing is indexed by them
    for (int q = blockIdx.x * kThreads + threadIdx.x; q < B; q += gridDim.x * kThreads)
      if (__ldg(cu + q) > __ldg(cu + q + 1)) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);

  const int steps = (rows + kRows - 1) / kRows;
  const int begin = (int)(((int64_t)steps * blockIdx.x) / gridDim.x);
  const int end = (int)(((int64_t)steps * (blockIdx.x + 1)) / gridDim.x);
  double sum_loss = 0.0, sum_t = 0.0, sum_s = 0.0;
  int seq_beg = 0, seq_end = 0;                     // the sequence of the previous row
  float w = w_all;
  for (int step = begin; step < end; ++step) {
    const int row = step * kRows + sub;
    const bool live = row < rows;                   // a group's lanes agree; all stay for the shuffles
    const float* lt_row = teacher_logp + (size_t)row * K;
    const float* lq_row = cand_logp + (size_t)row * K;
    float lt[kElems], lq[kElems], g[kElems];
#pragma unroll
    for (int i = 0; i < kElems / kVec; ++i) {
      const int k = (i * kG + lane) * kVec;
      if (live && k < K) {
        load_slots<kVec>(lt_row + k, lt + i * kVec);
        load_slots<kVec>(lq_row + k, lq + i * kVec);
      } else {
#pragma unroll
        for (int v = 0; v < kVec; ++v) { lt[i * kVec + v] = -INFINITY; lq[i * kVec + v] = 0.f; }
      }
    }
    if (prm.agg_mode == 0 && live) {
      const int t = t0 + row;
      if (t < seq_beg || t >= seq_end) {
        const int j = find_seq(cu, B, t);
        seq_beg = __ldg(cu + j);
        seq_end = __ldg(cu + j + 1);
        w = w_all * __frcp_rn((float)(seq_end - seq_beg));
      }
    }
    float tm = 0.f, sm = 0.f;
    const float loss = row_divergence<kSupport, kG>(lt, lq, forward, tau, inv_tau, g, tm, sm);
    if (live) {
      sum_t += (double)tm;
      sum_s += (double)sm;
      if (lane == 0) {
        sum_loss += (double)w * (double)loss;
        if (token_loss) token_loss[row] = loss;
      }
      if (dcand) {
        float* dst = dcand + (size_t)row * K;
#pragma unroll
        for (int i = 0; i < kElems / kVec; ++i) {
          const int k = (i * kG + lane) * kVec;
          if (k < K) {
#pragma unroll
            for (int v = 0; v < kVec; ++v) g[i * kVec + v] = lt[i * kVec + v] == -INFINITY ? 0.f : g[i * kVec + v] * w;
            store_slots<kVec>(dst + k, g + i * kVec);
          }
        }
      }
    }
  }
  if (!out) return;

  __shared__ double s_part[kThreads / 32][kNumSums];
  __shared__ int s_last;
  double v[kNumSums] = {sum_loss, sum_t, sum_s};
  const int wlane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int q = 0; q < kNumSums; ++q)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[q] += __shfl_xor_sync(0xffffffffu, v[q], o);
  if (wlane == 0)
    for (int q = 0; q < kNumSums; ++q) s_part[warp][q] = v[q];
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 0; q < kNumSums; ++q) {
      double t = 0.0;
      for (int i = 0; i < kThreads / 32; ++i) t += s_part[i][q];
      ws_partial(ws, blockIdx.x)[q] = t;
    }
    __threadfence();
    s_last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  if (warp == 0) {
    double tot[kNumSums] = {0.0, 0.0, 0.0};
    for (int b = wlane; b < (int)gridDim.x; b += 32)
      for (int q = 0; q < kNumSums; ++q) tot[q] += __ldcg(ws_partial(ws, b) + q);
#pragma unroll
    for (int q = 0; q < kNumSums; ++q)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) tot[q] += __shfl_xor_sync(0xffffffffu, tot[q], o);
    if (wlane == 0) {
      af_distill_out r;
      r.loss = (float)tot[0];
      r.teacher_mass = T > 0 ? (float)(tot[1] / (double)T) : 0.f;
      r.student_mass = T > 0 ? (float)(tot[2] / (double)T) : 0.f;
      r.reserved = 0;
      r.n_tokens = T;
      *out = r;
      if (__ldg(cu) != 0 || __ldg(cu + B) != T) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
      ws->ticket = 0;        // ready for the next call on this stream
    }
  }
}

struct DistillCall {
  const float* cand_logp;
  const float* teacher_logp;
  const int32_t* cu;
  int B, T, t0, rows, K;
  af_distill_params prm;
  af_distill_out* out;
  float* token_loss;
  float* dcand;
  DistillWs* ws;
  unsigned int* d_err;
  int sm_count;
};

template <int kSupport, int kG, int kVec>
cudaError_t launch_rows(const DistillCall& c, cudaStream_t s) {
  const int per_step = kThreads / kG;
  const int steps = (c.rows + per_step - 1) / per_step;
  const int most = c.sm_count * 8;                 // the workspace holds eight blocks' sums per SM
  const int blocks = steps < 1 ? 1 : steps < most ? steps : most;
  distill_loss_kernel<kSupport, kG, kVec><<<blocks, kThreads, 0, s>>>(
      c.cand_logp, c.teacher_logp, c.cu, c.B, c.T, c.t0, c.rows, c.K, c.prm, c.out, c.token_loss, c.dcand, c.ws, c.d_err);
  return cudaGetLastError();
}
// Rows that start on 16 bytes (K a multiple of 4) are read four slots at a time, even ones two.
template <int kSupport, int kG>
cudaError_t launch_group(const DistillCall& c, int vec, cudaStream_t s) {
  if (vec == 4) return launch_rows<kSupport, kG, 4>(c, s);
  if (vec == 2) return launch_rows<kSupport, kG, 2>(c, s);
  return launch_rows<kSupport, kG, 1>(c, s);
}
// The smallest group whose lanes hold the row with kElems slots each.
template <int kSupport>
cudaError_t launch_support(const DistillCall& c, int vec, cudaStream_t s) {
  if (c.K <= kElems) return launch_group<kSupport, 1>(c, vec, s);
  if (c.K <= 2 * kElems) return launch_group<kSupport, 2>(c, vec, s);
  if (c.K <= 4 * kElems) return launch_group<kSupport, 4>(c, vec, s);
  if (c.K <= 8 * kElems) return launch_group<kSupport, 8>(c, vec, s);
  if (c.K <= 16 * kElems) return launch_group<kSupport, 16>(c, vec, s);
  return launch_group<kSupport, 32>(c, vec, s);
}

}  // namespace

cudaError_t launch_distill_loss(const float* cand_logp, const float* teacher_logp, const int32_t* cu, int32_t B,
                                int64_t T, int64_t t0, int64_t rows, int32_t K, const af_distill_params& p,
                                af_distill_out* out, float* token_loss, float* dcand, void* ws, unsigned int* d_err,
                                int sm_count, cudaStream_t s) {
  auto all_aligned = [&](uintptr_t bytes) {
    return ((reinterpret_cast<uintptr_t>(cand_logp) | reinterpret_cast<uintptr_t>(teacher_logp) |
             reinterpret_cast<uintptr_t>(dcand)) & (bytes - 1)) == 0;
  };
  const int vec = K % 4 == 0 && all_aligned(16) ? 4 : K % 2 == 0 && all_aligned(8) ? 2 : 1;
  const DistillCall c{cand_logp, teacher_logp, cu, B, (int)T, (int)t0, (int)rows, K, p, out, token_loss, dcand,
                      static_cast<DistillWs*>(ws), d_err, sm_count};
  switch (p.support) {
    case 0: return launch_support<0>(c, vec, s);
    case 1: return launch_support<1>(c, vec, s);
    default: return launch_support<2>(c, vec, s);
  }
}

}  // namespace af
