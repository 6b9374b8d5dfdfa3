// af_distill_update: scoring of the listed candidates, distillation loss and backward of one packed
// micro-batch in one call, token block by token block.
//
// As in af_policy_update a block's fp32 logits stay in scratch between the two places that need them, so
// that the backward does not compute them again (two of eight T d V products less):
//   per block   1. Z = H_blk W^T (promoted accumulation) with the online-softmax statistics; Z is stored;
//               2. one warp per token: lse, entropy, and the listed log-probs picked from Z;
//               3. the loss kernel on the block's rows: d loss / d cand_logp;
//               4. one CTA per token: dZ in bf16 (reads 4 V, writes 2 V bytes per token);
//               5. dH_blk = dZ W and, unless the head is frozen, dW += dZ^T H_blk.
//   at the end  the record over all tokens, by the loss kernel (in step 3 when one block holds the batch).
// Measured: 8192 tokens, 3584 x 152064, K = 64, bf16 d_W 22.4-23.1 ms; 32768 tokens (four blocks) 94-97 ms; 1195 tokens,
// 256 x 4096 59 us, seven launches; dZ from the logits moves its 6 bytes per logit at 6.3 TB/s (4100 rows of 152064: 0.59 ms).
#include "candidate.cuh"

#include <algorithm>

namespace af {
namespace {

constexpr int kThreads = 256;

// One CTA per token row of the block and range of columns (one range, unless the rows are too few to fill the device: 29
// rows of 152064 take 45 us that way, 9 in ranges).  The dense part -G q_v goes out first; the listed columns are then
// written over it, rounded once from fp32: sum of the gradients that name the column, minus G q.
__global__ void __launch_bounds__(kThreads) dz_candidates_kernel(
    const float* __restrict__ z, __nv_bfloat16* __restrict__ dz, int V, const int32_t* __restrict__ cand,
    const float* __restrict__ g, const float* __restrict__ cand_logp, const float* __restrict__ lse, int K, int range) {
  __shared__ int s_id[AF_MAX_CANDIDATES];
  __shared__ float s_g[AF_MAX_CANDIDATES];
  __shared__ double s_sum[kThreads / 32];
  wait_for_predecessor();
  let_successor_start();
  const size_t row = blockIdx.x;
  const int k = threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int id = -1;
  float mine = 0.f;
  if (k < K) {
    id = __ldg(cand + row * K + k);
    if (id >= V) id = -1;
    if (id >= 0) mine = __ldg(g + row * K + k);
    s_id[k] = id;
    s_g[k] = mine;
  }
  double sum = (double)mine;      // 64 bits: the gradients of a renormalised list cancel
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) sum += s_sum[w];
  const float G = (float)sum;
  const float nl = -__ldg(lse + row) * kLog2e;
  const float4* zr = reinterpret_cast<const float4*>(z + row * V);
  uint4* out = reinterpret_cast<uint4*>(dz + row * V);
  const int begin = blockIdx.y * range, end = V - begin < range ? V : begin + range;     // range % 8 == 0
  for (int c8 = begin / 8 + threadIdx.x; c8 * 8 < end; c8 += kThreads) {      // 8 columns per thread per step
    const float4 a = __ldcs(zr + 2 * c8), b = __ldcs(zr + 2 * c8 + 1);
    float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = -G * ex2f(fmaf(v[i], kLog2e, nl));
    out[c8] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                         pack_bf16x2(v[6], v[7]));
  }
  float total = 0.f, q = 0.f;
  if (id < begin || id >= end) id = -1;                         // another CTA's
  if (id >= 0) {
    for (int i = 0; i < K; ++i) total += s_id[i] == id ? s_g[i] : 0.f;   // the same order for every slot naming id
    q = ex2f(__ldg(cand_logp + row * K + k) * kLog2e);
  }
  __syncthreads();                                              // the dense part is written
  if (id >= 0) dz[row * V + id] = __float2bfloat16_rn(fmaf(-G, q, total));
}

}  // namespace

af_status reserve_distill_update(af_ctx* ctx, int64_t T, int32_t K, int32_t V) {
  const int64_t Tc = backward_token_block(ctx, T);
  const af_status st = ws_grow(ctx->zlog, (size_t)Tc * V * 4);
  return st != AF_OK ? st : ws_grow(ctx->distill_ws, (size_t)Tc * K * sizeof(float));
}

af_status launch_distill_update(af_ctx* ctx, const void* hidden, const void* W, const int32_t* cand,
                                const float* teacher_logp, const int32_t* cu_seqlens, int32_t B, int64_t T, int32_t K,
                                int32_t d, int32_t V, const af_distill_params& params, af_distill_out* out,
                                float* cand_logp, float* entropy, float* lse, float* token_loss, float* dcand,
                                void* d_hidden, const HeadGradient& head, cudaStream_t s) {
  af_status st;
  if (T == 0) {
    if ((st = head_gradient_of_nothing(ctx, head, d, V, s)) != AF_OK) return st;
  } else {
    if ((st = reserve_head_gradient(ctx, T, d, V, head.d_W && head.type == AF_BF16)) != AF_OK) return st;
    if ((st = reserve_distill_update(ctx, T, K, V)) != AF_OK) return st;
  }
  const int64_t Tc = backward_token_block(ctx, T);
  const bool one_block = T > 0 && T <= Tc;
  const __nv_bfloat16* H = static_cast<const __nv_bfloat16*>(hidden);
  __nv_bfloat16* dz = static_cast<__nv_bfloat16*>(ctx->dz.p);
  float* zlog = static_cast<float*>(ctx->zlog.p);
  for (int64_t t0 = 0; t0 < T; t0 += Tc) {
    const int64_t tc = (T - t0) < Tc ? (T - t0) : Tc;
    float* lq = cand_logp + t0 * K;
    float* g = dcand ? dcand + t0 * K : static_cast<float*>(ctx->distill_ws.p);
    st = launch_candidate_logprob_z(ctx, H + t0 * d, W, cand + t0 * K, tc, K, d, V, lq, entropy ? entropy + t0 : nullptr,
                                    lse + t0, zlog, s);
    if (st != AF_OK) return st;
    if (launch_distill_loss(lq, teacher_logp + t0 * K, cu_seqlens, B, T, t0, tc, K, params, one_block ? out : nullptr,
                            one_block ? token_loss : nullptr, g, ctx->loss_ws.p, ctx->d_err, ctx->sm_count,
                            s) != cudaSuccess)
      return AF_ERR_CUDA;
    // ranges of at least 2048 columns, as many as it takes for four CTAs per SM
    const int64_t ranges = std::min<int64_t>((4 * (int64_t)ctx->sm_count + tc - 1) / tc, (V + 2047) / 2048);
    const int range = (int)(((V + ranges - 1) / ranges + 7) / 8 * 8);
    if (launch_overlapped(dz_candidates_kernel, dim3((unsigned)tc, (unsigned)((V + range - 1) / range)), kThreads, 0, s, zlog, dz, V,
                          cand + t0 * K, g, lq, lse + t0, K, range) != cudaSuccess)
      return AF_ERR_CUDA;
    st = launch_head_products(ctx, H + t0 * d, W, dz, tc, d, V, static_cast<__nv_bfloat16*>(d_hidden) + t0 * d, head,
                              t0 == 0, t0 + Tc >= T, s);
    if (st != AF_OK) return st;
  }
  if (one_block) return AF_OK;
  return launch_distill_loss(cand_logp, teacher_logp, cu_seqlens, B, T, 0, T, K, params, out, token_loss, nullptr,
                             ctx->loss_ws.p, ctx->d_err, ctx->sm_count, s) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
