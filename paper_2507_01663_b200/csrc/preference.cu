// af_preference_loss: paired sequence log ratios -> preference loss and its gradient per token.
//
//   S_j = sum over the tokens of sequence j of (logp - ref);  x_p = beta (n_c S_c - n_r S_r) - margin;
//   l_p = f(x_p) + nll_coef * mean(-logp over the chosen);    dlogp is constant over a sequence.
//
// 8 (or 4, without reference) bytes read and 4 written per token: HBM-bound, in two passes with the pairs in
// between, since a token's gradient needs its pair's sums.
//   1. sums    a warp per slice of 256 tokens: eight tokens per lane in registers, one warp reduction per
//              sequence that meets the slice.  A sequence inside one slice is done; one that crosses slice
//              borders leaves a piece per slice (16 bytes per 256 tokens), at most one coming in (head) and one
//              going out (tail), so pieces need no counters and their order is fixed.
//   2. pairs   a few lanes per pair add the pieces, evaluate the loss and write the two sequences' coefficients.
//   3. fill    a warp per slice again: the coefficient of each token's sequence.
// All sums are fp64 (thousands of near-cancelling terms, and the card has the rate: two additions per token)
// and taken in a fixed order, so results are bit-reproducible.
#include "common.cuh"
#include "device_util.cuh"

namespace af {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSlice = 256;                 // tokens of a warp's slice: two groups of 4 per lane, 128 apart
constexpr int kNumSums = 6;                 // loss, pair loss, nll, accuracy, chosen score, rejected score

struct PrefWs {                             // device views into the workspace
  double2* seq;                             // [B] sums of the sequences that lie inside one slice: S, sum of logp
  double2* head;                            // [slices] piece of the sequence that comes into the slice
  double2* tail;                            // [slices] piece of the sequence that starts in it and goes on
  float* coef;                              // [B] dloss/dlogp of a sequence's tokens
  double* partial;                          // [pair blocks][kNumSums]
};

int64_t slices_of(int64_t T) { return (T + kSlice - 1) / kSlice; }
constexpr int kMaxPairBlocks = 1024;

PrefWs carve(void* ws, int32_t B, int64_t T) {
  PrefWs w;
  w.seq = static_cast<double2*>(ws);
  w.head = w.seq + B;
  w.tail = w.head + slices_of(T);
  w.partial = reinterpret_cast<double*>(w.tail + slices_of(T));
  w.coef = reinterpret_cast<float*>(w.partial + (size_t)kMaxPairBlocks * kNumSums);
  return w;
}

// Token of slot i (0..7) of a lane: group i / 4 starts 128 tokens after the first.
__device__ __forceinline__ int slot_token(int base, int lane, int i) { return base + (i >> 2) * 128 + lane * 4 + (i & 3); }

// The lane's eight values of a column; zeros past the end.
__device__ __forceinline__ void load_slice(const float* __restrict__ p, int base, int lane, int T, bool vec, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int t = slot_token(base, lane, 4 * q);
    if (vec && t + 4 <= T) {
      const float4 x = __ldcs(reinterpret_cast<const float4*>(p + t));
      v[4 * q] = x.x; v[4 * q + 1] = x.y; v[4 * q + 2] = x.z; v[4 * q + 3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * q + i] = t + i < T ? __ldg(p + t + i) : 0.f;
    }
  }
}

// Calls f(j, beg, end) for every non-empty sequence that meets tokens [base, last), in order.  Uniform over the
// warp; ends whatever cu holds.
template <class F>
__device__ __forceinline__ void for_sequences(const int32_t* __restrict__ cu, int B, int base, int last, int lane, F f) {
  int t = base;
  int j = find_seq_warp(cu, B, t, lane);
  for (;;) {
    const int beg = __ldg(cu + j), end = __ldg(cu + j + 1);
    f(j, beg, end);
    if (end >= last || end <= t || j + 1 >= B) return;
    t = end;
    ++j;
    if (__ldg(cu + j + 1) <= t) j = find_seq_warp(cu, B, t, lane);      // a pile of empty sequences
  }
}

__global__ void __launch_bounds__(kThreads) pref_sums_kernel(
    const float* __restrict__ logp, const float* __restrict__ ref, const int32_t* __restrict__ cu, int B, int T,
    PrefWs ws, int vec) {
  const int lane = threadIdx.x & 31;
  const int slice = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int base = slice * kSlice;
  if (base >= T) return;
  const int last = T - base < kSlice ? T : base + kSlice;
  float lp[8], rf[8];
  load_slice(logp, base, lane, T, vec != 0, lp);
  if (ref) load_slice(ref, base, lane, T, vec != 0, rf);
  for_sequences(cu, B, base, last, lane, [&](int j, int beg, int end) {
    double s = 0.0, l = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = slot_token(base, lane, i);
      if (t >= beg && t < end) {
        l += (double)lp[i];
        if (ref) s += (double)lp[i] - (double)rf[i];
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      l += __shfl_xor_sync(0xffffffffu, l, o);
      if (ref) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    if (lane == 0) {
      const double2 v = make_double2(ref ? s : l, l);
      if (beg < base) ws.head[slice] = v;
      else if (end > last) ws.tail[slice] = v;
      else ws.seq[j] = v;
    }
  });
}

// Sums of one sequence, by kLanes lanes together (all get the result; every lane of the warp takes part).
// beg and end lie in [0, T].
template <int kLanes>
__device__ __forceinline__ double2 sequence_sum(const PrefWs& ws, int j, int beg, int end, int lane) {
  double s = 0.0, l = 0.0;
  if (end > beg) {
    const int first = beg / kSlice, final = (end - 1) / kSlice;
    if (first == final) {
      if (lane == 0) { const double2 v = ws.seq[j]; s = v.x; l = v.y; }
    } else {
      for (int i = first + lane; i <= final; i += kLanes) {
        const double2 v = i == first ? ws.tail[i] : ws.head[i];
        s += v.x; l += v.y;
      }
    }
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    l += __shfl_xor_sync(0xffffffffu, l, o);
  }
  return make_double2(s, l);
}

template <int kLanes>
__global__ void __launch_bounds__(kThreads) pref_pairs_kernel(
    const int32_t* __restrict__ cu, int B, int T, af_preference_params prm, PrefWs ws,
    af_preference_out* __restrict__ out, float* __restrict__ pair_loss, float* __restrict__ seq_score,
    unsigned int* ticket, unsigned int* d_err) {
  constexpr int kPairs = kThreads / kLanes;
  const int P = B / 2;
  const int lane = threadIdx.x % kLanes;
  for (int q = blockIdx.x * kThreads + threadIdx.x; q < B; q += gridDim.x * kThreads)
    if (__ldg(cu + q) > __ldg(cu + q + 1)) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
  const double beta = (double)prm.beta, w = P > 0 ? (double)prm.loss_scale / (double)P : 0.0;
  double sum[kNumSums] = {};
  for (int p0 = blockIdx.x * kPairs; p0 < P; p0 += gridDim.x * kPairs) {
    const int p = p0 + threadIdx.x / kLanes;
    const bool live = p < P;
    const int c = !live ? 0 : prm.pair_layout ? p : 2 * p, r = !live ? 0 : prm.pair_layout ? P + p : 2 * p + 1;
    // clamped: a cu_seqlens out of order is flagged, but must not index anything
    const int cb = min(max(__ldg(cu + c), 0), T), ce = min(max(__ldg(cu + c + 1), 0), T);
    const int rb = min(max(__ldg(cu + r), 0), T), re = min(max(__ldg(cu + r + 1), 0), T);
    const double2 sc = sequence_sum<kLanes>(ws, c, cb, live ? ce : cb, lane);
    const double2 sr = sequence_sum<kLanes>(ws, r, rb, live ? re : rb, lane);
    if (!live || lane != 0) continue;
    const double per_c = 1.0 / (double)(ce > cb ? ce - cb : 1), per_r = 1.0 / (double)(re > rb ? re - rb : 1);
    const double n_c = prm.length_norm ? per_c : 1.0, n_r = prm.length_norm ? per_r : 1.0;
    const double score_c = beta * sc.x * n_c, score_r = beta * sr.x * n_r;
    const double x = score_c - score_r - (double)prm.margin;
    double l, slope;
    if (prm.kind == 0) {
      const double eps = (double)prm.label_smoothing;
      l = log1p(exp(-fabs(x))) + (x < 0.0 ? -x : 0.0) + (eps > 0.0 ? eps * x : 0.0);
      slope = eps - 1.0 / (1.0 + exp(x));
    } else if (prm.kind == 1) {
      const double y = (x - 0.5) / beta;
      l = y * y;
      slope = 2.0 * y / beta;
    } else {
      l = x < 1.0 ? 1.0 - x : x >= 1.0 ? 0.0 : x;        // a NaN stays one
      slope = x < 1.0 ? -1.0 : 0.0;
    }
    const double nll = -sc.y * per_c, nll_coef = (double)prm.nll_coef;
    const double whole = nll_coef != 0.0 ? l + nll_coef * nll : l;
    ws.coef[c] = (float)(w * (slope * beta * n_c - nll_coef * per_c));
    ws.coef[r] = (float)(-w * slope * beta * n_r);
    if (pair_loss) pair_loss[p] = (float)whole;
    if (seq_score) { seq_score[c] = (float)score_c; seq_score[r] = (float)score_r; }
    sum[0] += whole; sum[1] += l; sum[2] += nll;
    sum[3] += score_c > score_r ? 1.0 : 0.0;
    sum[4] += score_c; sum[5] += score_r;
  }

  __shared__ double s_part[kWarps][kNumSums];
  __shared__ int s_last;
  const int wlane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncwarp();
#pragma unroll
  for (int q = 0; q < kNumSums; ++q)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], o);
  if (wlane == 0)
    for (int q = 0; q < kNumSums; ++q) s_part[warp][q] = sum[q];
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int q = 0; q < kNumSums; ++q) {
      double t = 0.0;
      for (int i = 0; i < kWarps; ++i) t += s_part[i][q];
      ws.partial[(size_t)blockIdx.x * kNumSums + q] = t;
    }
    __threadfence();
    s_last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  if (warp == 0) {
    double tot[kNumSums] = {};
    for (int b = wlane; b < (int)gridDim.x; b += 32)
      for (int q = 0; q < kNumSums; ++q) tot[q] += __ldcg(ws.partial + (size_t)b * kNumSums + q);
#pragma unroll
    for (int q = 0; q < kNumSums; ++q)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) tot[q] += __shfl_xor_sync(0xffffffffu, tot[q], o);
    if (wlane == 0) {
      const double inv = P > 0 ? 1.0 / (double)P : 0.0;
      af_preference_out r;
      r.loss = (float)(w * tot[0]);
      r.pair_loss = (float)(inv * tot[1]);
      r.nll = (float)(inv * tot[2]);
      r.accuracy = (float)(inv * tot[3]);
      r.chosen_score = (float)(inv * tot[4]);
      r.rejected_score = (float)(inv * tot[5]);
      r.n_pairs = P;
      *out = r;
      if (__ldg(cu) != 0 || __ldg(cu + B) != T) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
      *ticket = 0;           // ready for the next call on this stream
    }
  }
}

__global__ void __launch_bounds__(kThreads) pref_fill_kernel(const int32_t* __restrict__ cu, int B, int T, PrefWs ws,
                                                             float* __restrict__ dlogp, int vec) {
  const int lane = threadIdx.x & 31;
  const int base = (blockIdx.x * kWarps + (threadIdx.x >> 5)) * kSlice;
  if (base >= T) return;
  const int last = T - base < kSlice ? T : base + kSlice;
  float g[8] = {};
  for_sequences(cu, B, base, last, lane, [&](int j, int beg, int end) {
    const float c = __ldg(ws.coef + j);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = slot_token(base, lane, i);
      if (t >= beg && t < end) g[i] = c;
    }
  });
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int t = slot_token(base, lane, 4 * q);
    if (vec && t + 4 <= T) {
      __stcs(reinterpret_cast<float4*>(dlogp + t), make_float4(g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) if (t + i < T) dlogp[t + i] = g[4 * q + i];
    }
  }
}

}  // namespace

size_t preference_workspace_bytes(int32_t B, int64_t T) {
  return (size_t)B * (sizeof(double2) + sizeof(float)) + (size_t)slices_of(T) * 2 * sizeof(double2) +
         (size_t)kMaxPairBlocks * kNumSums * sizeof(double);
}

cudaError_t launch_preference_loss(const float* logp, const float* ref_logp, const int32_t* cu, int32_t B, int64_t T,
                                   const af_preference_params& p, af_preference_out* out, float* pair_loss,
                                   float* seq_score, float* dlogp, void* ws_mem, void* loss_ws, unsigned int* d_err,
                                   int sm_count, cudaStream_t s) {
  auto al = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  const PrefWs ws = carve(ws_mem, B, T);
  const unsigned slice_blocks = (unsigned)((slices_of(T) + kWarps - 1) / kWarps);
  if (T > 0) {
    pref_sums_kernel<<<slice_blocks, kThreads, 0, s>>>(logp, ref_logp, cu, B, (int)T, ws, al(logp) && al(ref_logp));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  // eight lanes per pair while sequences have few pieces, a warp beyond 4096 tokens on average
  const int P = B / 2;
  const int lanes = B > 0 && T / B > 4096 ? 32 : 8;
  const int wanted = (P + kThreads / lanes - 1) / (kThreads / lanes);
  int most = sm_count * 4 < kMaxPairBlocks ? sm_count * 4 : kMaxPairBlocks;
  const int blocks = wanted < 1 ? 1 : wanted < most ? wanted : most;
  unsigned int* ticket = static_cast<unsigned int*>(loss_ws);      // the reductions' ticket of this context
  if (lanes == 8)
    pref_pairs_kernel<8><<<blocks, kThreads, 0, s>>>(cu, B, (int)T, p, ws, out, pair_loss, seq_score, ticket, d_err);
  else
    pref_pairs_kernel<32><<<blocks, kThreads, 0, s>>>(cu, B, (int)T, p, ws, out, pair_loss, seq_score, ticket, d_err);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || T == 0 || !dlogp) return e;
  pref_fill_kernel<<<slice_blocks, kThreads, 0, s>>>(cu, B, (int)T, ws, dlogp, al(dlogp));
  return cudaGetLastError();
}

}  // namespace af
