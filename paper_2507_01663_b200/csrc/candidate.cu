// af_candidate_logprob: log-probs of K listed vocabulary ids per token -- the LM-head GEMM with the
// online log-softmax of af_token_logprob, whose epilogue also hands out the listed logits.
//
//   z_tv = h_t . w_v;   lse_t = log sum_v e^{z_tv};   cand_logp[t,k] = z_{t, cand[t,k]} - lse_t
//
// Bound: tensor cores for batches (2 T d V), the stream of W for single tokens (2 d V bytes).  The
// lists cost next to nothing on top: each row's list is sorted into keys once (4 bytes per slot), and
// a thread of the epilogue, which owns a row and sweeps the vocabulary upwards, compares one key with
// the end of its columns per 32 of them.  Fetching the K rows of W again for K dot products instead
// would move 2 K d bytes per token (0.46 MB at K = 64, d = 3584: a tenth of the GEMM's time).
//
// Measured at d = 3584, V = 152064: 8192 tokens, K = 64, 7.1-7.2 ms (1.25 PFLOP/s in a stream of calls under the power cap);
// 64 tokens, K = 20, 187-198 us on several B200s (5.8-5.5 TB/s of W).
//
// The accumulation is promoted to round-to-nearest every kPromoteBlocks K blocks (see umma.cuh).
#include "candidate.cuh"
#include "gemm_launch.cuh"

namespace af {
namespace {

// K = 512 per part.  8192 x 3584 x 152064: 7529 us at 256, 6902 at 512, 6692 at 896, 6495 without parts; the error of lse
// is 3.2e-7 at 512 and 5.8e-7 at 896.
constexpr int kPromoteBlocks = 8;

struct CandidateState {
  float m, s, u;
  const uint32_t* keys;                 // this row's sorted list
  int next;                             // first entry not behind the sweep
  uint32_t key;                         // that entry
};

// kStoreZ: write the fp32 logits of the tile (one token block of the fused update, which picks from them
// later); otherwise the listed logits go to cand_z as the sweep passes them.
template <bool kStoreZ>
struct CandidateEpi {
  struct Params {
    const uint32_t* keys;   // [T, K] sorted (not kStoreZ)
    float* cand_z;          // [T, K] (not kStoreZ)
    float4* partial;        // [T, parts]: m, s, u of every part
    float* z;               // [T, V] (kStoreZ)
    int T, V, K, parts;
  };
  using State = CandidateState;
  static constexpr bool kStaged = kStoreZ;
  static __device__ __forceinline__ void unit_begin(State& st, const Params& p, int row, int col0) {
    st.m = -INFINITY; st.s = 0.f; st.u = 0.f;
    st.key = kNoCandidate;
    if constexpr (!kStoreZ) {
      if (row < p.T) {
        st.keys = p.keys + (size_t)row * p.K;
        st.next = first_candidate(st.keys, p.K, col0);
        st.key = candidate_at(st.keys, p.K, st.next);
      }
    }
  }
  static __device__ __forceinline__ void tile(State& st, const Params& p, int row, int col0, int cols,
                                              float (&a)[umma::kPromoteCols], uint8_t* stage) {
    constexpr int kCols = umma::kPromoteCols;
    if (col0 >= p.V) return;
    if constexpr (kStoreZ) {
      // a lane has a row's 128 values; stored that way, an instruction would write 16 bytes to each of 32 rows.  By
      // way of shared memory it writes four whole 128-byte lines (32 x 32 values at a time; slot q of row r sits at
      // q ^ (r & 7), so that neither side meets bank conflicts)
      const int lane = threadIdx.x & 31;
      float4* const st4 = reinterpret_cast<float4*>(stage);
#pragma unroll
      for (int c = 0; c < kCols; c += 32) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          st4[lane * 8 + (q ^ (lane & 7))] = make_float4(a[c + 4 * q], a[c + 4 * q + 1], a[c + 4 * q + 2], a[c + 4 * q + 3]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = i * 4 + (lane >> 3), q = lane & 7;
          const int zr = row - lane + r, zc = col0 + c + 4 * q;
          if (zr < p.T && zc < p.V)           // V % 8 == 0 here: whole float4s, 16-byte aligned
            __stcs(reinterpret_cast<float4*>(p.z + (size_t)zr * p.V + zc), st4[r * 8 + (q ^ (r & 7))]);
        }
        __syncwarp();
      }
    } else {
      // entries of the other column half that the sweep has passed by
      while ((int)(st.key >> 8) < col0) { ++st.next; st.key = candidate_at(st.keys, p.K, st.next); }
#pragma unroll
      for (int c = 0; c < kCols; c += 32) {
        const int end = col0 + (c + 32 < cols ? c + 32 : cols);
        while ((int)(st.key >> 8) < end) {
          const int j = (int)(st.key >> 8) - (col0 + c);
          float z = a[c];
#pragma unroll
          for (int i = 1; i < 32; ++i) z = i == j ? a[c + i] : z;
          p.cand_z[(size_t)row * p.K + (st.key & 255u)] = z;
          ++st.next;
          st.key = candidate_at(st.keys, p.K, st.next);
        }
      }
    }
    if (col0 + kCols > p.V || cols < kCols) {   // columns >= V hold zero-fill, columns past the tile's width nothing
      const int n = p.V - col0 < cols ? p.V - col0 : cols;
#pragma unroll
      for (int j = 0; j < kCols; ++j) if (j >= n) a[j] = -1.0e30f;
    }
    float mx[4] = {a[0], a[1], a[2], a[3]};
#pragma unroll
    for (int j = 4; j < kCols; ++j) mx[j & 3] = fmaxf(mx[j & 3], a[j]);
    const float m_new = fmaxf(st.m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
    const float sc = ex2f((st.m - m_new) * kLog2e);             // 0 on the first tile (m = -inf)
    const float nm = -m_new * kLog2e;
    float s[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};   // short sums first: less rounding
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      const float e = ex2f(fmaf(a[j], kLog2e, nm));
      s[j & 3] += e;
      u[j & 3] = fmaf(e, a[j], u[j & 3]);
    }
    st.m = m_new;
    st.s = fmaf(st.s, sc, (s[0] + s[1]) + (s[2] + s[3]));
    st.u = fmaf(st.u, sc, (u[0] + u[1]) + (u[2] + u[3]));
  }
  static __device__ __forceinline__ void unit_end(State& st, const Params& p, int row, int part) {
    if (row < p.T) p.partial[(size_t)row * p.parts + part] = make_float4(st.m, st.s, st.u, 0.f);
  }
};

// ---- the lists -> sorted keys -------------------------------------------------------------------------
// One warp per token, kE entries per lane (entry i = e * 32 + lane), bitonic network.
template <int kE>
__global__ void __launch_bounds__(256) sort_candidates_kernel(
    const int32_t* __restrict__ cand, const float* __restrict__ g, int64_t rows, int K, int V,
    uint32_t* __restrict__ keys, float* __restrict__ gsum) {
  wait_for_predecessor();
  let_successor_start();
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int lane = threadIdx.x & 31;
  uint32_t x[kE];
  double sum = 0.0;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const int k = e * 32 + lane;
    x[e] = kNoCandidate;
    if (k < K) {
      const int id = __ldg(cand + row * K + k);
      if (id >= 0 && id < V) {
        x[e] = ((uint32_t)id << 8) | (uint32_t)k;
        if (g) sum += (double)__ldg(g + row * K + k);
      }
    }
  }
  if (g) {     // 64 bits: the gradients of a renormalised list cancel in this sum
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) gsum[row] = (float)sum;
  }
#pragma unroll
  for (int size = 2; size <= 32 * kE; size <<= 1) {
#pragma unroll
    for (int stride = size >> 1; stride > 0; stride >>= 1) {
      if (stride >= 32) {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const int o = e ^ (stride >> 5);
          if (o > e) {
            const bool up = ((e * 32) & size) == 0;          // size > 32 here: the lane does not decide
            const uint32_t lo = x[e] < x[o] ? x[e] : x[o], hi = x[e] < x[o] ? x[o] : x[e];
            x[e] = up ? lo : hi;
            x[o] = up ? hi : lo;
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, x[e], stride);
          const bool up = ((e * 32 + lane) & size) == 0, low = (lane & stride) == 0;
          x[e] = (up == low) ? (x[e] < other ? x[e] : other) : (x[e] < other ? other : x[e]);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    const int k = e * 32 + lane;
    if (k < K) keys[row * K + k] = x[e];
  }
}

// ---- partial softmax states -> lse, entropy; listed logits -> log-probs ----------------------------------
// One warp per token.  kFromZ: the listed logits are picked from the stored logits z [rows, V] here.
template <bool kFromZ>
__global__ void __launch_bounds__(256) finish_candidates_kernel(
    const float4* __restrict__ partial, int parts, const int32_t* __restrict__ cand, const float* __restrict__ z,
    int64_t rows, int K, int V, float* __restrict__ cand_logp, float* __restrict__ entropy,
    float* __restrict__ lse_out, unsigned int* d_err) {
  wait_for_predecessor();
  let_successor_start();
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int lane = threadIdx.x & 31;
  const float4* q = partial + row * parts;
  float M = -INFINITY;
  for (int i = lane; i < parts; i += 32) M = fmaxf(M, __ldg(q + i).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  float s = 0.f, u = 0.f;
  for (int i = lane; i < parts; i += 32) {
    const float4 c = __ldg(q + i);
    // a part whose columns all lie past the vocabulary's end never began: (-inf, 0, 0)
    const float w = c.x == -INFINITY ? 0.f : ex2f((c.x - M) * kLog2e);
    s = fmaf(c.y, w, s);
    u = fmaf(c.z, w, u);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    u += __shfl_xor_sync(0xffffffffu, u, o);
  }
  const float lse = M + logf(s);
  if (lane == 0) {
    if (lse_out) lse_out[row] = lse;
    if (entropy) entropy[row] = lse - u / s;
  }
  for (int k = lane; k < K; k += 32) {
    const int id = __ldg(cand + row * K + k);
    float lq;
    if (id >= 0 && id < V) {
      lq = (kFromZ ? __ldg(z + (size_t)row * V + id) : cand_logp[row * K + k]) - lse;
    } else if (id < 0) {
      lq = -INFINITY;                                          // an unused slot
    } else {
      lq = __int_as_float(0x7fc00000);
      atomicOr(d_err, AF_DEVERR_TARGET_RANGE);
    }
    cand_logp[row * K + k] = lq;
  }
}

}  // namespace

cudaError_t launch_sort_candidates(const int32_t* cand, const float* g, int64_t rows, int32_t K, int32_t V,
                                   uint32_t* keys, float* gsum, cudaStream_t s) {
  const unsigned blocks = (unsigned)((rows + 7) / 8);
  auto kernel = K <= 32 ? sort_candidates_kernel<1> : K <= 64 ? sort_candidates_kernel<2>
              : K <= 128 ? sort_candidates_kernel<4> : sort_candidates_kernel<8>;
  return launch_overlapped(kernel, blocks, 256, 0, s, cand, g, rows, K, V, keys, gsum);
}

// How the scoring GEMM is cut: vocabulary ranges per row tile, columns of a tile, CTA pairs or single CTAs.
// Up to 128 tokens it is the stream of W, and the MMAs should not stand in its way: a pair multiplies 256 rows of
// hidden states whatever their number, a single CTA 128, and the tile's width is free to share the columns out evenly
// (152064 columns on 148 SMs: 5 tiles of 208 for 4.94; on 74 pairs 9 tiles of 256 for 8.03).  64 tokens of 3584 over
// 152064 words: 183 us against 228 on pairs (191 with tiles of 256); 17 tokens 209 against 242; 64 tokens of 5120, 255
// against 326.  From there on the rule of af_token_logprob holds, except that it stops at 32 ranges, too few for one or
// two row tiles.
struct CandidateTiling {
  int splits, bn;
  bool single;
};
static CandidateTiling candidate_tiling(const af_ctx* ctx, int64_t T, int32_t d, int32_t V, bool store_z) {
  const int64_t m_tiles = (T + umma::kPairBM - 1) / umma::kPairBM;
  const int n_tiles = (V + umma::kBN - 1) / umma::kBN;
  if (ctx->v_splits == 0 && T <= umma::kBM && !store_z) {
    int bn = umma::kBN;
    int64_t least = INT64_MAX;
    for (int b = umma::kBN; b >= 128; b -= 16) {
      const int64_t tiles = (V + b - 1) / b, columns = (tiles + ctx->sm_count - 1) / ctx->sm_count * b;   // of the busiest SM
      if (columns < least) { least = columns; bn = b; }
    }
    const int tiles = (V + bn - 1) / bn;
    return CandidateTiling{ctx->sm_count < tiles ? ctx->sm_count : tiles, bn, true};
  }
  const int workers = ctx->sm_count / 2 > 0 ? ctx->sm_count / 2 : 1;
  int S;
  if (ctx->v_splits == 0 && m_tiles * 32 < workers) {
    S = (int)(workers / m_tiles);
  } else {
    const int die0_pairs = ctx->die_aware && ctx->die0_sms > 0 ? ctx->die0_sms / 2 : 0;
    S = logprob_pick_splits(T, d, V, ctx->sm_count, true, ctx->v_splits, die0_pairs);
  }
  return CandidateTiling{S < n_tiles ? S : n_tiles, umma::kBN, false};
}

static size_t candidate_partial_bytes(const af_ctx* ctx, int64_t max_T, int32_t d, int32_t V) {
  const int64_t S = candidate_tiling(ctx, max_T, d, V, true).splits;
  // smaller batches may pick up to 8 ranges whatever their size, and more only while there are at most 8
  // units per pair (one unit = 256 rows of two parts) or one per SM (128 rows)
  const int64_t need = (S > 8 ? S : 8) * 2 * max_T;
  const int64_t small = (int64_t)(ctx->sm_count / 2 + 1) * 8 * 2 * umma::kPairBM;
  return (size_t)(need > small ? need : small) * sizeof(float4);
}

// Logits of `T` rows (kStoreZ) or their listed ones, and the partial softmax states; *parts: states per row.
static af_status candidate_gemm(af_ctx* ctx, const void* hidden, const void* W, int64_t T, int32_t d, int32_t V,
                                int32_t K, const uint32_t* keys, float* cand_z, float* z, int* parts,
                                cudaStream_t s) {
  const Operand Hop{hidden, (uint64_t)T, (uint64_t)d, (uint64_t)d * 2};
  const Operand Wop{W, (uint64_t)V, (uint64_t)d, (uint64_t)d * 2};
  GemmEnv env = unpaced_if_cached(gemm_env(ctx), Hop, Wop);
  if (T <= umma::kPairBM) env.tile_clock = nullptr;   // one row tile: every pair reads its own part of W, none shares
  const CandidateTiling tiling = candidate_tiling(ctx, T, d, V, z != nullptr);
  const int S = tiling.splits;
  *parts = 2 * S;
  af_status st = ws_grow(ctx->partial, (size_t)*parts * (size_t)T * sizeof(float4));
  if (st != AF_OK) return st;
  float4* partial = static_cast<float4*>(ctx->partial.p);
  if (z) {
    CandidateEpi<true>::Params ep{nullptr, nullptr, partial, z, (int)T, V, K, *parts};
    return run_gemm_promoted<CandidateEpi<true>, kPromoteBlocks>(env, Hop, Wop, S, ep, s);
  }
  CandidateEpi<false>::Params ep{keys, cand_z, partial, nullptr, (int)T, V, K, *parts};
  if (tiling.single) return run_gemm_promoted_single<CandidateEpi<false>, kPromoteBlocks>(env, Hop, Wop, S, tiling.bn, ep, s);
  return run_gemm_promoted<CandidateEpi<false>, kPromoteBlocks>(env, Hop, Wop, S, ep, s);
}

// Workspace of the one-pass kernel: softmax states in `partial`, logits in `cand_keys`.
static af_status reserve_stream(af_ctx* ctx, int64_t T, int32_t V) {
  const af_status st = ws_grow(ctx->partial, (size_t)T * ctx->sm_count * sizeof(float4));
  return st != AF_OK ? st : ws_grow(ctx->cand_keys, (size_t)T * V * sizeof(float));
}
af_status reserve_candidate_logprob(af_ctx* ctx, int64_t max_T, int32_t K, int32_t d, int32_t V) {
  af_status st = ws_grow(ctx->partial, candidate_partial_bytes(ctx, max_T, d, V));
  if (st == AF_OK) st = ws_grow(ctx->cand_keys, (size_t)max_T * K * sizeof(uint32_t));
  if (st == AF_OK) st = reserve_stream(ctx, max_T < kStreamTokens ? max_T : kStreamTokens, V);
  return st;
}

af_status launch_candidate_logprob(af_ctx* ctx, const void* hidden, const void* W, const int32_t* cand, int64_t T,
                                   int32_t K, int32_t d, int32_t V, float* cand_logp, float* entropy, float* lse,
                                   cudaStream_t s) {
  if (ctx->v_splits == 0 && stream_fits(T, d)) {
    const af_status fits = reserve_stream(ctx, T, V);
    if (fits != AF_OK) return fits;
    const StreamCall c{hidden, W, cand, (int)T, K, d, V, static_cast<float*>(ctx->cand_keys.p),
                       static_cast<float4*>(ctx->partial.p), cand_logp, entropy, lse,
                       static_cast<unsigned int*>(ctx->loss_ws.p), ctx->d_err};      // the reductions' ticket of this context
    return launch_candidate_stream(c, ctx->sm_count, s);
  }
  af_status st = ws_grow(ctx->cand_keys, (size_t)T * K * sizeof(uint32_t));
  if (st != AF_OK) return st;
  uint32_t* keys = static_cast<uint32_t*>(ctx->cand_keys.p);
  if (launch_sort_candidates(cand, nullptr, T, K, V, keys, nullptr, s) != cudaSuccess) return AF_ERR_CUDA;
  int parts = 0;
  if ((st = candidate_gemm(ctx, hidden, W, T, d, V, K, keys, cand_logp, nullptr, &parts, s)) != AF_OK) return st;
  return launch_overlapped(finish_candidates_kernel<false>, (unsigned)((T + 7) / 8), 256, 0, s,
                           static_cast<const float4*>(ctx->partial.p), parts, cand, nullptr, T, K, V, cand_logp, entropy, lse,
                           ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

af_status launch_candidate_logprob_z(af_ctx* ctx, const void* hidden, const void* W, const int32_t* cand, int64_t T,
                                     int32_t K, int32_t d, int32_t V, float* cand_logp, float* entropy, float* lse,
                                     float* z, cudaStream_t s) {
  if (ctx->v_splits == 0 && stream_fits(T, d)) {
    const af_status fits = ws_grow(ctx->partial, (size_t)T * ctx->sm_count * sizeof(float4));
    if (fits != AF_OK) return fits;
    const StreamCall c{hidden, W, cand, (int)T, K, d, V, z, static_cast<float4*>(ctx->partial.p), cand_logp, entropy, lse,
                       static_cast<unsigned int*>(ctx->loss_ws.p), ctx->d_err};
    return launch_candidate_stream(c, ctx->sm_count, s);
  }
  int parts = 0;
  const af_status st = candidate_gemm(ctx, hidden, W, T, d, V, K, nullptr, nullptr, z, &parts, s);
  if (st != AF_OK) return st;
  return launch_overlapped(finish_candidates_kernel<true>, (unsigned)((T + 7) / 8), 256, 0, s,
                           static_cast<const float4*>(ctx->partial.p), parts, cand, z, T, K, V, cand_logp, entropy, lse,
                           ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
