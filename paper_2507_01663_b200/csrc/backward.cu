// af_policy_loss_backward: gradient of the policy loss through log-softmax and the LM head.
//
// Tokens are processed in blocks of Tc rows.  Per block, three tensor-core GEMMs built on the
// same tcgen05 main loop:
//   1. recompute  Z = H_blk W^T  (both operands K-major) and turn it, in the epilogue, into
//        dZ = g_t (1{v = y_t} - exp(z - lse_t))   (bf16), written once as dZ [Tc, V];
//   2. dH_blk = dZ * W        A = dZ [Tc,V] K-major,  B = W [V,d] read MN-major   -> bf16 [Tc, d];
//   3. dW^T  += H_blk^T * dZ  A = H_blk [Tc,d] and B = dZ [Tc,V], both read MN-major; the tile is
//                             computed as [d, V] and stored transposed into fp32 dW [V, d].
// No operand is ever transposed in memory.  The scratch is one block of dZ; [T,V] is never
// materialised and the scratch does not grow with T.
//
// Epilogues hold one output row per lane (the TMEM load shape); storing that directly would write
// 16 bytes to each of 32 different rows per instruction.  The dZ and dH epilogues therefore pass
// their 32x32 chunk through a private, XOR-swizzled shared-memory buffer and store whole 64-byte
// row segments, eight rows per instruction.  The dW product is laid out the other way round: its
// accumulator rows run along d, the contiguous dimension of dW, so 32 lanes holding the same
// vocabulary row write 128 consecutive bytes without any staging.  That orientation also gives the
// product the forward's memory behaviour: the H_blk panels of the row tiles in flight stay in L2
// while dZ streams past them (once per round of row tiles).
#include "candidate.cuh"
#include "device_util.cuh"
#include "gemm_launch.cuh"

namespace af {
namespace {

constexpr int kDefaultTokenBlock = 74 * 128;  // 37 pair tiles (74 CTA tiles) x 14 column tiles of d = 3584: 7 full rounds of 148 SMs


// Store a 32-row x 32-column bf16 chunk (lane L holds row L as 16 packed words) to a row-major
// bf16 matrix: rows row0.., columns col0..; rows >= M and 8-column groups past N are skipped.
// Staging layout: row r occupies 64 bytes = four 16-byte slots; slot q of row r lives at position
// q ^ ((r >> 1) & 3), which makes both the row-per-lane writes and the 8-rows-per-instruction
// reads free of bank conflicts.
__device__ __forceinline__ void store_chunk_bf16(const uint32_t (&w)[16], uint8_t* stage, int lane,
                                                 __nv_bfloat16* C, int64_t ldc, int row0, int col0,
                                                 int M, int N) {
  uint4* st = reinterpret_cast<uint4*>(stage);
#pragma unroll
  for (int q = 0; q < 4; ++q)
    st[lane * 4 + (q ^ ((lane >> 1) & 3))] = make_uint4(w[q * 4 + 0], w[q * 4 + 1], w[q * 4 + 2], w[q * 4 + 3]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + (lane >> 2), c = lane & 3;
    const uint4 v = st[r * 4 + (c ^ ((r >> 1) & 3))];
    const int grow = row0 + r, gcol = col0 + c * 8;
    if (grow < M && gcol + 8 <= N) *reinterpret_cast<uint4*>(C + (size_t)grow * ldc + gcol) = v;
  }
  __syncwarp();
}

// ---- epilogue 1: logits tile -> dZ ----------------------------------------------------------------
struct DzEpi {
  struct Params {
    const int32_t* target;  // [rows] of this block
    const float* lse;       // [rows]
    const float* g;         // [rows] dL/dlogp
    __nv_bfloat16* dz;      // [rows, V]
    int rows, V;
    int v_offset;           // vocabulary id of W's first row (0 unless W is one shard of the head)
  };
  struct State {
    float g, nl;
    int y;
  };
  static constexpr bool kStaged = true;
  static __device__ __forceinline__ void unit_begin(State& st, const Params& p, int row, int, int) {
    if (row < p.rows) {
      st.g = __ldg(p.g + row);
      st.nl = -__ldg(p.lse + row) * kLog2e;
      st.y = __ldg(p.target + row) - p.v_offset;   // outside [0, V): no column of this W matches
    } else {
      st.g = 0.f; st.nl = 0.f; st.y = -1;
    }
  }
  static __device__ __forceinline__ void chunk(State& st, const Params& p, int row, int col0,
                                               const uint32_t (&v)[32], uint8_t* stage) {
    if (col0 >= p.V) return;                       // uniform across the warp
    const int lane = threadIdx.x & 31;
    float dzv[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float prob = ex2f(fmaf(__uint_as_float(v[j]), kLog2e, st.nl));
      dzv[j] = -st.g * prob;
    }
    const int yl = st.y - col0;
    if (yl >= 0 && yl < 32) {
#pragma unroll
      for (int j = 0; j < 32; ++j) if (j == yl) dzv[j] += st.g;
    }
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(dzv[2 * j], dzv[2 * j + 1]);
    store_chunk_bf16(w, stage, lane, p.dz, p.V, row - lane, col0, p.rows, p.V);
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

// ---- epilogue 1b: logits tile -> dZ of listed candidates --------------------------------------------
// dZ_tv = sum_{k: cand[t,k] = v} g_tk - G_t exp(z_tv - lse_t),  G_t = sum_k g_tk: the softmax part is dense,
// the rest lands on the K listed columns, which the sweep meets in the order of the sorted keys.  Both are
// added in fp32 and rounded to bf16 once.  (4001 tokens at 3584 x 152064: 2.86 ms, 1.52 PFLOP/s alone.)
struct DzCandidateEpi {
  struct Params {
    const uint32_t* keys;   // [rows, K] sorted
    const float* g;         // [rows, K] in list order
    const float* gsum;      // [rows]
    const float* lse;       // [rows]
    __nv_bfloat16* dz;      // [rows, V]
    int rows, V, K;
  };
  struct State {
    float gsum, nl;
    int next;               // -1: the unit's first chunk has not been met
    uint32_t key;
  };
  static constexpr bool kStaged = true;
  static constexpr bool kHalves = true;
  static __device__ __forceinline__ void unit_begin(State& st, const Params& p, int row, int, int) {
    st.next = -1;
    st.key = kNoCandidate;
    if (row < p.rows) {
      st.gsum = __ldg(p.gsum + row);
      st.nl = -__ldg(p.lse + row) * kLog2e;
    } else {
      st.gsum = 0.f; st.nl = 0.f;
    }
  }
  static __device__ __forceinline__ void chunk(State& st, const Params& p, int row, int col0,
                                               const uint32_t (&v)[32], uint8_t* stage) {
    if (col0 >= p.V) return;                       // uniform across the warp
    const int lane = threadIdx.x & 31;
    const uint32_t* keys = p.keys + (size_t)row * p.K;      // read for rows < p.rows only
    if (st.next < 0) {
      st.next = 0;
      if (row < p.rows) {
        st.next = first_candidate(keys, p.K, col0);
        st.key = candidate_at(keys, p.K, st.next);
      }
    }
    float dzv[32];
#pragma unroll
    for (int j = 0; j < 32; ++j)
      dzv[j] = -st.gsum * ex2f(fmaf(__uint_as_float(v[j]), kLog2e, st.nl));
    while ((int)(st.key >> 8) < col0) { ++st.next; st.key = candidate_at(keys, p.K, st.next); }   // another warp's columns
    while ((int)(st.key >> 8) < col0 + 32) {
      const int j = (int)(st.key >> 8) - col0;
      const float g = __ldg(p.g + (size_t)row * p.K + (st.key & 255u));
#pragma unroll
      for (int i = 0; i < 32; ++i) dzv[i] += i == j ? g : 0.f;
      ++st.next;
      st.key = candidate_at(keys, p.K, st.next);
    }
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(dzv[2 * j], dzv[2 * j + 1]);
    __syncwarp();
    store_chunk_bf16(w, stage, lane, p.dz, p.V, row - lane, col0, p.rows, p.V);
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

// ---- epilogue 2: accumulator tile -> bf16 matrix ------------------------------------------------
struct StoreBf16Epi {
  struct Params {
    __nv_bfloat16* C;
    int64_t ldc;
    int M, N;
  };
  struct State {};
  static constexpr bool kStaged = true;
  static __device__ __forceinline__ void unit_begin(State&, const Params&, int, int, int) {}
  static __device__ __forceinline__ void chunk(State&, const Params& p, int row, int col0,
                                               const uint32_t (&v)[32], uint8_t* stage) {
    if (col0 >= p.N) return;
    const int lane = threadIdx.x & 31;
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
    store_chunk_bf16(w, stage, lane, p.C, p.ldc, row - lane, col0, p.M, p.N);
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

// ---- epilogue 3: accumulator tile [m, n] -> fp32 matrix C[n, m] (store or add) ------------------
// Lane L holds row m = row0 + L; for a fixed column n the 32 lanes address 32 consecutive floats of
// C's row n: one coalesced 128-byte access per column.
struct StoreF32TransposedEpi {
  struct Params {
    float* C;          // [N, M] row-major
    int64_t ldc;       // elements between consecutive n
    int M, N;
    int accumulate;
  };
  struct State {};
  static constexpr bool kStaged = false;
  static __device__ __forceinline__ void unit_begin(State&, const Params&, int, int, int) {}
  static __device__ __forceinline__ void chunk(State&, const Params& p, int row, int col0,
                                               const uint32_t (&v)[32], uint8_t*) {
    if (col0 >= p.N || row >= p.M) return;
    float* dst = p.C + (size_t)col0 * p.ldc + row;
    if (col0 + 32 <= p.N) {
      if (p.accumulate) {
        float o[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = dst[(size_t)j * p.ldc];
#pragma unroll
        for (int j = 0; j < 32; ++j) dst[(size_t)j * p.ldc] = o[j] + __uint_as_float(v[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) dst[(size_t)j * p.ldc] = __uint_as_float(v[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if (col0 + j < p.N) {
          float w = __uint_as_float(v[j]);
          if (p.accumulate) w += dst[(size_t)j * p.ldc];
          dst[(size_t)j * p.ldc] = w;
        }
      }
    }
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

// ---- epilogue 3b: the same into a bf16 matrix, on top of fp32 sums of earlier blocks if there are any ----
struct StoreBf16TransposedEpi {
  struct Params {
    __nv_bfloat16* C;     // [N, M] row-major
    const float* sums;    // [N, M] sums of the earlier token blocks, or null
    int64_t ldc;
    int M, N;
  };
  struct State {};
  static constexpr bool kStaged = false;
  static constexpr bool kHalves = true;
  static __device__ __forceinline__ void unit_begin(State&, const Params&, int, int, int) {}
  static __device__ __forceinline__ void chunk(State&, const Params& p, int row, int col0,
                                               const uint32_t (&v)[32], uint8_t*) {
    if (col0 >= p.N) return;                       // uniform across the warp
    // Two lanes trade a column for a row (M = d is even), so that each stores two neighbouring values of one column: half
    // the stores.  (5000 tokens at 3584 x 19008: 1.6 ms either way, most of it products.)
    const int lane = threadIdx.x & 31;
    const bool odd = lane & 1;
    const size_t at = (size_t)(col0 + odd) * p.ldc + (row - odd);
    const bool mine = row < p.M;
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
      const float keep = __uint_as_float(odd ? v[j + 1] : v[j]);
      const float got = __shfl_xor_sync(0xffffffffu, __uint_as_float(odd ? v[j] : v[j + 1]), 1);
      float2 w = odd ? make_float2(got, keep) : make_float2(keep, got);
      if (mine && col0 + j + odd < p.N) {
        if (p.sums) {
          const float2 o = *reinterpret_cast<const float2*>(p.sums + at + (size_t)j * p.ldc);
          w.x += o.x; w.y += o.y;
        }
        *reinterpret_cast<uint32_t*>(p.C + at + (size_t)j * p.ldc) = pack_bf16x2(w.x, w.y);
      }
    }
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

}  // namespace

// The two products that consume a block of dZ [tc, V] (bf16):
//   dH_blk = dZ W:        A = dZ (K = v contiguous), B = W read MN-major (n = d contiguous, K = v rows)
//   dW^T  += H_blk^T dZ:  A = H_blk read MN-major (m = d contiguous, K = t rows), B = dZ read MN-major
//                         (n = v contiguous); tile [d, v] stored transposed into dW [V, d].  Vocabulary
//                         ranges are chosen as in the forward: the H_blk panels in flight stay in L2, dZ
//                         streams past them.
af_status launch_backward_products(af_ctx* ctx, const void* hidden_blk, const void* W, const void* dz_blk,
                                   int64_t tc, int32_t d, int32_t V, void* d_hidden_blk, float* d_W,
                                   int32_t accumulate_dW, bool last_block, cudaStream_t s) {
  const GemmEnv env = gemm_env(ctx);
  const uint64_t dB = (uint64_t)d * 2, vB = (uint64_t)V * 2;
  const Operand Hblk{hidden_blk, (uint64_t)tc, (uint64_t)d, dB};
  const Operand Wop{W, (uint64_t)V, (uint64_t)d, dB};
  const Operand dZop{dz_blk, (uint64_t)tc, (uint64_t)V, vB};
  auto dH_product = [&]() {
    StoreBf16Epi::Params p2{static_cast<__nv_bfloat16*>(d_hidden_blk), d, (int)tc, d};
    return run_gemm<StoreBf16Epi, false, true>(env, dZop, Wop, 0, p2, s);
  };
  auto dW_product = [&]() {
    StoreF32TransposedEpi::Params p3{d_W, d, d, V, accumulate_dW ? 1 : 0};
    return run_gemm<StoreF32TransposedEpi, true, true>(
        env, Hblk, dZop, logprob_pick_splits((int64_t)d, (int32_t)tc, V, ctx->sm_count, env.pair, 0, 0), p3, s);
  };
  // With a "d_W ready" event registered, the last block runs its dW product first and records the
  // event behind it: d_W is complete from there on, and whoever waits on the event (a gradient
  // all-reduce on another stream) overlaps with the block's dH product and whatever follows.
  if (last_block && ctx->dw_ready) {
    af_status st = dW_product();
    if (st != AF_OK) return st;
    if (cudaEventRecord(ctx->dw_ready, s) != cudaSuccess) return AF_ERR_CUDA;
    return dH_product();
  }
  af_status st = dH_product();
  if (st != AF_OK) return st;
  return dW_product();
}

namespace {

// ---- epilogue 2b: accumulator tile of one range of the reduction -> fp32 partial sums [part][M, N] ----------
struct StorePartialEpi {
  struct Params {
    float* P;
    int M, N;
  };
  struct State {
    float* row;
  };
  static constexpr bool kStaged = false;
  static constexpr bool kHalves = true;
  static __device__ __forceinline__ void unit_begin(State& st, const Params& p, int row, int, int part) {
    st.row = p.P + ((size_t)part * p.M + row) * p.N;
  }
  static __device__ __forceinline__ void chunk(State& st, const Params& p, int row, int col0, const uint32_t (&v)[32],
                                               uint8_t*) {
    if (row >= p.M) return;
#pragma unroll
    for (int q = 0; q < 8; ++q)        // N % 8 == 0
      if (col0 + 4 * q < p.N)
        *reinterpret_cast<uint4*>(st.row + col0 + 4 * q) = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

// ---- epilogue 3c: accumulator tile [v, d] -> d_W [V, d] in either type, by way of shared memory as whole pieces of rows ----
template <bool kF32>
struct StoreHeadEpi {
  struct Params {
    void* C;
    int M, N;
    int accumulate;       // kF32 only
  };
  struct State {};
  static constexpr bool kStaged = true;
  static constexpr bool kHalves = true;
  static __device__ __forceinline__ void unit_begin(State&, const Params&, int, int, int) {}
  static __device__ __forceinline__ void chunk(State&, const Params& p, int row, int col0, const uint32_t (&v)[32],
                                               uint8_t* stage) {
    if (col0 >= p.N) return;                       // uniform across the warp
    const int lane = threadIdx.x & 31;
    if constexpr (kF32) {
      // slot q (16 bytes) of row r sits at q ^ (r & 7): no bank conflicts on either side
      float4* const st = reinterpret_cast<float4*>(stage);
#pragma unroll
      for (int q = 0; q < 8; ++q)
        st[lane * 8 + (q ^ (lane & 7))] = make_float4(__uint_as_float(v[4 * q]), __uint_as_float(v[4 * q + 1]),
                                                      __uint_as_float(v[4 * q + 2]), __uint_as_float(v[4 * q + 3]));
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = i * 4 + (lane >> 3), q = lane & 7;
        const int grow = row - lane + r, gcol = col0 + 4 * q;
        if (grow < p.M && gcol < p.N) {            // N % 8 == 0
          float4* const to = reinterpret_cast<float4*>(static_cast<float*>(p.C) + (size_t)grow * p.N + gcol);
          float4 w = st[r * 8 + (q ^ (r & 7))];
          if (p.accumulate) {
            const float4 o = *to;
            w = make_float4(o.x + w.x, o.y + w.y, o.z + w.z, o.w + w.w);
          }
          *to = w;
        }
      }
      __syncwarp();
    } else {
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
      store_chunk_bf16(w, stage, lane, static_cast<__nv_bfloat16*>(p.C), p.N, row - lane, col0, p.M, p.N);
    }
  }
  static __device__ __forceinline__ void unit_end(State&, const Params&, int, int) {}
};

// Adds the parts in order and rounds once: 8 values per thread.
__global__ void __launch_bounds__(256) sum_parts_kernel(const float* __restrict__ P, int parts, size_t n,
                                                        __nv_bfloat16* __restrict__ out) {
  wait_for_predecessor();
  let_successor_start();
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float a[8] = {};
  for (int k = 0; k < parts; ++k) {
    const float4 x = __ldcs(reinterpret_cast<const float4*>(P + k * n + i));
    const float4 y = __ldcs(reinterpret_cast<const float4*>(P + k * n + i) + 1);
    a[0] += x.x; a[1] += x.y; a[2] += x.z; a[3] += x.w;
    a[4] += y.x; a[5] += y.y; a[6] += y.z; a[7] += y.w;
  }
  *reinterpret_cast<uint4*>(out + i) =
      make_uint4(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(a[4], a[5]), pack_bf16x2(a[6], a[7]));
}

// How dH = dZ W is cut: its reduction is the vocabulary, its tiles are few (16 x 14 for 4001 tokens of the 7B-shaped
// head), and a last round of tiles that is not full costs as much as a full one (224 tiles on 74 pairs: 4 rounds for
// 3.03).  The last `rows` row tiles are cut into `parts` ranges of K instead, as many as spread them evenly.
struct TailPlan {
  int rows, parts;
};
constexpr int kMaxTailRounds = 4;      // tiles x parts of the tail, per pair: bounds its workspace
TailPlan plan_tail(int m_tiles, int n_tiles, int k_blocks, int pairs) {
  TailPlan best{0, 1};
  const double tile_us = 0.25 * k_blocks;      // a 256 x 256 x 64 block takes a pair about 0.25 us
  double best_us = tile_us * ((m_tiles * (int64_t)n_tiles + pairs - 1) / pairs);
  for (int r = 1; r <= m_tiles && r <= pairs; ++r) {
    const int64_t rounds = ((m_tiles - r) * (int64_t)n_tiles + pairs - 1) / pairs;
    for (int k = 2; k <= 32 && k * 4 <= k_blocks; ++k) {
      const int64_t units = (int64_t)r * n_tiles * k;
      if (units > (int64_t)kMaxTailRounds * pairs) break;
      // the split launch and the sum of its parts (written and read once each), and a second GEMM launch
      const double us = tile_us * (rounds + (double)((units + pairs - 1) / pairs) / k) + 0.13 * units + (r < m_tiles ? 7.0 : 4.0);
      if (us < best_us) { best_us = us; best = TailPlan{r, k}; }
    }
  }
  return best;
}

// dH_blk = dZ W with the tail cut that way.
af_status hidden_gradient(af_ctx* ctx, const GemmEnv& env, const Operand& dZ, const Operand& W, int64_t tc, int32_t d,
                          __nv_bfloat16* d_hidden, cudaStream_t s) {
  const int pairs = env.sm_count / 2;
  const int m_tiles = (int)((tc + umma::kPairBM - 1) / umma::kPairBM), n_tiles = (d + umma::kBN - 1) / umma::kBN;
  const TailPlan tail = env.pair ? plan_tail(m_tiles, n_tiles, (int)((dZ.cols + umma::kBK - 1) / umma::kBK), pairs)
                                 : TailPlan{0, 1};
  const int64_t first = tail.rows > 0 ? (int64_t)(m_tiles - tail.rows) * umma::kPairBM : tc;   // rows before the tail
  af_status st = AF_OK;
  if (first > 0) {
    const Operand A{dZ.base, (uint64_t)first, dZ.cols, dZ.pitch_bytes};
    StoreBf16Epi::Params p{d_hidden, d, (int)first, d};
    st = run_gemm<StoreBf16Epi, false, true>(unpaced_if_cached(env, A, W), A, W, 0, p, s);
    if (st != AF_OK) return st;
  }
  if (first == tc) return AF_OK;
  const int64_t rows = tc - first;
  const size_t n = (size_t)rows * d;
  float* P = static_cast<float*>(ctx->split_k.p);
  const Operand A{static_cast<const char*>(dZ.base) + (size_t)first * dZ.pitch_bytes, (uint64_t)rows, dZ.cols, dZ.pitch_bytes};
  StorePartialEpi::Params p{P, (int)rows, d};
  if ((st = run_gemm_split_k<StorePartialEpi, false, true>(env, A, W, tail.parts, p, s)) != AF_OK) return st;
  return launch_overlapped(sum_parts_kernel, (unsigned)((n / 8 + 255) / 256), 256, 0, s, P, tail.parts, n,
                           d_hidden + (size_t)first * d) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

// Most that plan_tail may ask for, whatever the batch: a tile of partial sums per unit.
size_t split_k_bytes(int sm_count) {
  return (size_t)kMaxTailRounds * (sm_count / 2) * umma::kPairBM * umma::kBN * sizeof(float);
}

}  // namespace

// The same two products for a head whose gradient is wanted in fp32, in bf16 or not at all.  A bf16 d_W is
// rounded once: with several token blocks the earlier ones are summed in fp32 in the workspace and the last
// one's epilogue adds and rounds.
af_status launch_head_products(af_ctx* ctx, const void* hidden_blk, const void* W, const void* dz_blk, int64_t tc,
                               int32_t d, int32_t V, void* d_hidden_blk, const HeadGradient& head, bool first_block,
                               bool last_block, cudaStream_t s) {
  GemmEnv env = gemm_env(ctx);
  env.overlapped = true;
  const uint64_t dB = (uint64_t)d * 2, vB = (uint64_t)V * 2;
  const Operand Hblk{hidden_blk, (uint64_t)tc, (uint64_t)d, dB};
  const Operand Wop{W, (uint64_t)V, (uint64_t)d, dB};
  const Operand dZop{dz_blk, (uint64_t)tc, (uint64_t)V, vB};
  auto dH_product = [&]() {
    return hidden_gradient(ctx, env, dZop, Wop, tc, d, static_cast<__nv_bfloat16*>(d_hidden_blk), s);
  };
  auto dW_product = [&]() {
    // With dZ^T as the first operand a thread holds a piece of a row of d_W in place of a column, and a warp stores 16
    // bytes per lane, which is what counts for few tokens, when the product is a stream of d_W; dZ streams past once, and
    // the hidden states stay in L2 as long as they take 32 MB or less.  3584 x 152064, the whole call: 29 tokens 697 us
    // against 1106, 400 tokens 1.30 ms against 1.59, 700 tokens 1.94 against 2.38, 4001 tokens 10.1 against 10.2.
    // d_W of 29 tokens alone: 1.09 GB in 314 us, 3.5 TB/s of writes (728 us the other way round; a plain fill of the same
    // bytes takes 279 us, 3.9 TB/s).
    // Beyond that the order whose panels of hidden states take turns in L2.
    if (env.pair && first_block && last_block && tc * (int64_t)d <= (16 << 20)) {
      GemmEnv stream = env;
      stream.tile_clock = nullptr;
      if (head.type == AF_BF16)
        return run_gemm<StoreHeadEpi<false>, true, true>(stream, dZop, Hblk, 0, {head.d_W, V, d, 0}, s);
      return run_gemm<StoreHeadEpi<true>, true, true>(stream, dZop, Hblk, 0, {head.d_W, V, d, head.accumulate ? 1 : 0}, s);
    }
    const int S = logprob_pick_splits((int64_t)d, (int32_t)tc, V, ctx->sm_count, env.pair, 0, 0);
    if (head.type == AF_BF16 && last_block) {
      StoreBf16TransposedEpi::Params p3{static_cast<__nv_bfloat16*>(head.d_W),
                                        first_block ? nullptr : static_cast<const float*>(ctx->dw_sums.p), d, d, V};
      return run_gemm<StoreBf16TransposedEpi, true, true>(unpaced_if_cached(env, Hblk, dZop), Hblk, dZop, S, p3, s);
    }
    float* C = head.type == AF_BF16 ? static_cast<float*>(ctx->dw_sums.p) : static_cast<float*>(head.d_W);
    const bool add = !first_block || (head.type == AF_F32 && head.accumulate);
    StoreF32TransposedEpi::Params p3{C, d, d, V, add ? 1 : 0};
    return run_gemm<StoreF32TransposedEpi, true, true>(unpaced_if_cached(env, Hblk, dZop), Hblk, dZop, S, p3, s);
  };
  if (!head.d_W) return dH_product();
  if (last_block && ctx->dw_ready) {      // as in launch_backward_products
    af_status st = dW_product();
    if (st != AF_OK) return st;
    if (cudaEventRecord(ctx->dw_ready, s) != cudaSuccess) return AF_ERR_CUDA;
    return dH_product();
  }
  const af_status st = dH_product();
  return st != AF_OK ? st : dW_product();
}

// d_W of an empty batch, and the event that says it is complete.
af_status head_gradient_of_nothing(af_ctx* ctx, const HeadGradient& head, int32_t d, int32_t V, cudaStream_t s) {
  if (!head.d_W) return AF_OK;
  const size_t bytes = (size_t)V * d * (head.type == AF_BF16 ? 2 : 4);
  if (!head.accumulate && cudaMemsetAsync(head.d_W, 0, bytes, s) != cudaSuccess) return AF_ERR_CUDA;
  if (ctx->dw_ready && cudaEventRecord(ctx->dw_ready, s) != cudaSuccess) return AF_ERR_CUDA;
  return AF_OK;
}

// Scratch of the candidate backward: dZ of one token block and, for a bf16 d_W over several blocks, the fp32 sums.
af_status reserve_head_gradient(af_ctx* ctx, int64_t T, int32_t d, int32_t V, bool bf16_head) {
  const int64_t Tc = backward_token_block(ctx, T);
  af_status st = ws_grow(ctx->dz, (size_t)Tc * V * 2);
  if (st == AF_OK) st = ws_grow(ctx->split_k, split_k_bytes(ctx->sm_count));
  if (st == AF_OK && bf16_head && T > Tc) st = ws_grow(ctx->dw_sums, (size_t)V * d * sizeof(float));
  return st;
}

// af_candidate_logprob_backward: per token block the sorted lists and G, then dZ on the tensor cores (the
// logits recomputed) and the two products.
af_status launch_candidate_backward(af_ctx* ctx, const void* hidden, const void* W, const int32_t* cand,
                                    const float* lse, const float* g, int64_t T, int32_t K, int32_t d, int32_t V,
                                    void* d_hidden, const HeadGradient& head, cudaStream_t s) {
  if (T == 0) return head_gradient_of_nothing(ctx, head, d, V, s);
  af_status st = reserve_head_gradient(ctx, T, d, V, head.d_W && head.type == AF_BF16);
  if (st != AF_OK) return st;
  const int64_t Tc = backward_token_block(ctx, T);
  const size_t key_bytes = (size_t)Tc * K * sizeof(uint32_t);
  if ((st = ws_grow(ctx->cand_keys, key_bytes + (size_t)Tc * sizeof(float))) != AF_OK) return st;
  uint32_t* keys = static_cast<uint32_t*>(ctx->cand_keys.p);
  float* gsum = reinterpret_cast<float*>(static_cast<char*>(ctx->cand_keys.p) + key_bytes);
  __nv_bfloat16* dz = static_cast<__nv_bfloat16*>(ctx->dz.p);
  const __nv_bfloat16* H = static_cast<const __nv_bfloat16*>(hidden);
  GemmEnv env = gemm_env(ctx);
  env.overlapped = true;
  for (int64_t t0 = 0; t0 < T; t0 += Tc) {
    const int64_t tc = (T - t0) < Tc ? (T - t0) : Tc;
    if (launch_sort_candidates(cand + t0 * K, g + t0 * K, tc, K, V, keys, gsum, s) != cudaSuccess) return AF_ERR_CUDA;
    const Operand Hblk{H + t0 * d, (uint64_t)tc, (uint64_t)d, (uint64_t)d * 2};
    const Operand Wop{W, (uint64_t)V, (uint64_t)d, (uint64_t)d * 2};
    DzCandidateEpi::Params p1{keys, g + t0 * K, gsum, lse + t0, dz, (int)tc, V, K};
    // one or two row tiles: a range of W per pair, as in the scoring call (32 ranges, the most of the other rule, leave
    // pairs idle: 29 tokens at 3584 x 152064, 338 us); and one row tile shares nothing that needs pacing
    const int64_t m_tiles = (tc + umma::kPairBM - 1) / umma::kPairBM, workers = ctx->sm_count / 2;
    const int S = env.pair && ctx->v_splits == 0 && m_tiles * 32 < workers
                      ? (int)(workers / m_tiles)
                      : logprob_pick_splits(tc, d, V, ctx->sm_count, env.pair, ctx->v_splits, env.die0_pairs);
    GemmEnv dz_env = unpaced_if_cached(env, Hblk, Wop);
    if (tc <= umma::kPairBM) dz_env.tile_clock = nullptr;
    st = run_gemm<DzCandidateEpi, false, false>(dz_env, Hblk, Wop, S, p1, s);
    if (st != AF_OK) return st;
    st = launch_head_products(ctx, H + t0 * d, W, dz, tc, d, V, static_cast<__nv_bfloat16*>(d_hidden) + t0 * d, head,
                              t0 == 0, t0 + Tc >= T, s);
    if (st != AF_OK) return st;
  }
  return AF_OK;
}

// Token block of the backward (and of the fused update): a multiple of 128 rows.
int64_t backward_token_block(const af_ctx* ctx, int64_t T) {
  int64_t Tc = ctx->bwd_token_block > 0 ? ctx->bwd_token_block : kDefaultTokenBlock;
  const int64_t T_round = ((T + 127) / 128) * 128;
  if (Tc > T_round) Tc = T_round > 0 ? T_round : 128;
  return Tc;
}

af_status launch_backward(af_ctx* ctx, const void* hidden, const void* W, const int32_t* target,
                          const float* lse, const float* dlogp, int64_t T, int32_t d, int32_t V,
                          void* d_hidden, float* d_W, int32_t accumulate_dW, cudaStream_t s, int32_t v_offset) {
  const int64_t Tc = backward_token_block(ctx, T);
  const GemmEnv env = gemm_env(ctx);
  af_status st;
  if ((st = ws_grow(ctx->dz, (size_t)Tc * V * 2)) != AF_OK) return st;
  if (accumulate_dW < 0) return AF_OK;  // reserve only

  if (T == 0) {
    if (!accumulate_dW && cudaMemsetAsync(d_W, 0, (size_t)V * d * sizeof(float), s) != cudaSuccess) return AF_ERR_CUDA;
    if (ctx->dw_ready && cudaEventRecord(ctx->dw_ready, s) != cudaSuccess) return AF_ERR_CUDA;
    return AF_OK;
  }
  const __nv_bfloat16* H = static_cast<const __nv_bfloat16*>(hidden);
  __nv_bfloat16* dz = static_cast<__nv_bfloat16*>(ctx->dz.p);
  const uint64_t dB = (uint64_t)d * 2;

  bool first = true;
  for (int64_t t0 = 0; t0 < T; t0 += Tc, first = false) {
    const uint64_t tc = (uint64_t)((T - t0) < Tc ? (T - t0) : Tc);
    const Operand Hblk{H + t0 * d, tc, (uint64_t)d, dB};
    const Operand Wop{W, (uint64_t)V, (uint64_t)d, dB};
    // 1. dZ block:  Z = H_blk W^T, both K-major
    DzEpi::Params p1{target + t0, lse + t0, dlogp + t0, dz, (int)tc, V, v_offset};
    st = run_gemm<DzEpi, false, false>(env, Hblk, Wop,
                                       logprob_pick_splits((int64_t)tc, d, V, ctx->sm_count, env.pair, ctx->v_splits, env.die0_pairs), p1, s);
    if (st != AF_OK) return st;
    st = launch_backward_products(ctx, H + t0 * d, W, dz, (int64_t)tc, d, V,
                                  static_cast<__nv_bfloat16*>(d_hidden) + t0 * d, d_W,
                                  (!first || accumulate_dW) ? 1 : 0, t0 + Tc >= T, s);
    if (st != AF_OK) return st;
  }
  return AF_OK;
}

}  // namespace af
