// af_candidate_logprob for a few tokens (single-token decoding, small batches): one pass over W.
//
// With T <= 16 tokens the head is a stream of V d bf16 values, each used T times: 2 V d bytes at the memory's
// rate (166 us for the 7B-shaped head), and everything else has to stay out of the way.  A CTA takes 8 rows of W
// at a time, one stretch of memory and one bulk copy into a ring of shared-memory stages, and its eight warps split the
// sum over k.  A warp's part of the hidden states is the same for every row, so it stays in registers for the whole
// launch as fragments of mma.m16n8k16 (the tokens as M, the rows as N); the order of k inside a dot product is free, so
// a lane takes 32 consecutive bytes of its row (16 values of k) as the fragments of four MMAs.  The CTAs' tiles are
// neighbours: what is being read at one time is one stretch of W.
// Measured: 159 us for one token, 6.9 TB/s.  What else was measured for one token at the 7B-shaped head: the tcgen05 kernel
// 280 us (it fetches a 128-row tile of hidden states per stage, 127 rows of which are absent, and balances 256 rows of W
// per pair); a warp per row tile with loads to registers 182-197 us (DRAM serves 28 000 streams of a few hundred bytes at
// 5.5 TB/s); loads to registers with k split over the warps 185-600 us (a warp cannot tell more than a few loads in flight
// apart).
// Each warp's accumulators cover an eighth of k; the parts are added in fp32, rounding to nearest (see umma.cuh on
// truncation), in the order of the warps, once per kRound tiles.  What the eighths still lose to truncation is one place
// of lse (1.2e-7 of it).
// Every logit is also written to the workspace (4 V bytes per token, 0.06 % of W's each): the last CTA to finish
// joins the softmax states and picks the listed logits from there, so the lists need no sorting and the call is one
// launch.
#include "candidate.cuh"
#include "umma.cuh"

namespace af {
namespace {

constexpr int kWarps = 8;                // a ninth, to feed the ring, would leave 168 registers a thread instead of 255
constexpr int kThreads = kWarps * 32;
constexpr int kLineK = 64;               // k of a 128-byte line
constexpr int kRows = 8;                 // rows of a tile
constexpr int kRound = 4;                // tiles whose parts are joined at a time
constexpr int kMaxStages = 8;
constexpr int kRingBytes = 184 * 1024;   // beside 17 or 33 KB of parts

__device__ __forceinline__ void bulk_load(uint32_t dst_smem, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               :: "r"(dst_smem), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds_u128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
// c (16 x 8) += a (16 x 16) b (16 x 8); a row-major fragments, b column-major.
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// m = max z, s = sum 2^x, u = sum 2^x x with x = (z - m) log2 e.  u is taken about the maximum, so that the entropy,
// log s - log 2 u / s, does not come out as a small difference of two numbers of the size of the logits.
struct SoftmaxState {
  float m, s, u;
  __device__ __forceinline__ void add(float z) {
    const float m_new = fmaxf(m, z);
    const float dm = (m - m_new) * kLog2e, x = (z - m_new) * kLog2e;
    const float sc = ex2f(dm), e = ex2f(x);
    u = fmaf(fmaf(s, dm, u), sc, e * x);
    s = fmaf(s, sc, e);
    m = m_new;
  }
  // states of nothing have m = kNone (finite, so that differences stay numbers)
  __device__ __forceinline__ void join(float m2, float s2, float u2) {
    const float m_new = fmaxf(m, m2);
    const float da = (m - m_new) * kLog2e, db = (m2 - m_new) * kLog2e;
    const float a = ex2f(da), b = ex2f(db);
    u = fmaf(fmaf(s, da, u), a, fmaf(s2, db, u2) * b);
    s = fmaf(s, a, s2 * b);
    m = m_new;
  }
};
constexpr float kNone = -1.0e30f;

// kTokens: groups of 8 tokens (1 or 2); kLines: most lines of k a warp's part may have.
template <int kTokens, int kLines>
__global__ void __launch_bounds__(kThreads, 1) candidate_stream_kernel(
    const uint4* __restrict__ H, const char* __restrict__ W, const int32_t* __restrict__ cand, int T, int K, int d, int V,
    int stages, float* __restrict__ z, float4* __restrict__ partial, float* __restrict__ cand_logp,
    float* __restrict__ entropy, float* __restrict__ lse_out, unsigned int* ticket, unsigned int* d_err) {
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int kM = kTokens * 8;
  __shared__ float s_part[2][kRound][kWarps][kM * 8];    // [round parity][tile][warp][token][row]
  __shared__ float4 s_state[kRound][kM];
  __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages];
  __shared__ int s_last, abort_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  wait_for_predecessor();
  let_successor_start();
  const uint32_t ring = umma::smem_u32(smem), bars = umma::smem_u32(s_bars);
  const uint32_t row_bytes = (uint32_t)d * 2, stage_bytes = kRows * row_bytes;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kMaxStages + s); };
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < stages; ++s) { umma::mbar_init(full_bar(s), 1); umma::mbar_init(empty_bar(s), kWarps); }
    umma::fence_mbar_init();
  }
  __syncthreads();

  const int tiles = (V + kRows - 1) / kRows;
  const int my_tiles = (tiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;    // tiles b, b + grid, ...
  SoftmaxState st[kTokens];                // of a finishing thread's (tile of the round, token, row)
#pragma unroll
  for (int j = 0; j < kTokens; ++j) st[j] = SoftmaxState{kNone, 0.f, 0.f};
  bool ok = true;                          // false once a wait ran out of time
  auto issue = [&](int i) {                // thread 0: brings the CTA's tile i into its stage
    const int tile = (int)blockIdx.x + i * (int)gridDim.x, stage = i % stages;
    const int rows = V - tile * kRows < kRows ? V - tile * kRows : kRows;
    umma::mbar_arrive_expect_tx(full_bar(stage), rows * row_bytes);
    bulk_load(ring + stage * stage_bytes, W + (size_t)tile * stage_bytes, rows * row_bytes, full_bar(stage));
  };
  if (threadIdx.x == 0)
    for (int i = 0; i < stages && i < my_tiles; ++i) issue(i);
  __syncwarp();

  const int n_lines = (d + kLineK - 1) / kLineK;
  const int line0 = n_lines * warp / kWarps, lines = n_lines * (warp + 1) / kWarps - line0;   // this warp's part of k
  // what of a line's 32 bytes of this lane lies in the row: all but in the last line
  auto halves_in = [&](int line) { return (d - line * kLineK - t * 16) / 8; };              // >= 2: both
  // ---- this warp's part of the hidden states: tokens g and g + 8
  uint32_t h[kTokens][kLines][8];
#pragma unroll
  for (int j = 0; j < kTokens; ++j)
#pragma unroll
    for (int l = 0; l < kLines; ++l)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int tok = j * 8 + g;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (tok < T && l < lines && halves_in(line0 + l) > e)
          x = __ldg(H + ((size_t)tok * d + (line0 + l) * kLineK + t * 16) / 8 + e);
        h[j][l][4 * e] = x.x; h[j][l][4 * e + 1] = x.y; h[j][l][4 * e + 2] = x.z; h[j][l][4 * e + 3] = x.w;
      }
  const bool ragged = d % kLineK != 0 && line0 + lines == n_lines;      // the last line of this part is not whole
  int stage = 0;
  uint32_t phase = 0;
  for (int i = 0; i < my_tiles; ++i) {
    // the stage of tile i - 1 is refilled once every warp has left it
    if (threadIdx.x == 0 && ok && i >= 1 && i - 1 + stages < my_tiles) {
      const int before = stage == 0 ? stages - 1 : stage - 1;
      if (umma::mbar_wait(empty_bar(before), stage == 0 ? phase ^ 1u : phase, &abort_flag)) issue(i - 1 + stages);
    }
    __syncwarp();
    ok = __all_sync(0xffffffffu, ok && umma::mbar_wait(full_bar(stage), phase, &abort_flag));
    float acc[2][4] = {};                // rows 2t and 2t + 1 for token g, then for token g + 8; two chains each
    const uint32_t at = ring + stage * stage_bytes + (uint32_t)g * row_bytes + (uint32_t)line0 * 128u + (uint32_t)t * 32u;
    if (ok) {
#pragma unroll
      for (int l = 0; l < kLines; ++l) {
        if (l >= lines) break;
        uint4 x = lds_u128(at + l * 128), y = lds_u128(at + l * 128 + 16);
        if (ragged && l == lines - 1) {  // the next row's values, or none at all
          if (halves_in(line0 + l) < 1) x = make_uint4(0, 0, 0, 0);
          if (halves_in(line0 + l) < 2) y = make_uint4(0, 0, 0, 0);
        }
        uint32_t u[8] = {};
        if constexpr (kTokens == 2) {
#pragma unroll
          for (int e = 0; e < 8; ++e) u[e] = h[kTokens - 1][l][e];
        }
        mma16816(acc[0], h[0][l][0], u[0], h[0][l][1], u[1], x.x, x.y);
        mma16816(acc[1], h[0][l][2], u[2], h[0][l][3], u[3], x.z, x.w);
        mma16816(acc[0], h[0][l][4], u[4], h[0][l][5], u[5], y.x, y.y);
        mma16816(acc[1], h[0][l][6], u[6], h[0][l][7], u[7], y.z, y.w);
      }
    }
    __syncwarp();
    if (lane == 0) umma::mbar_arrive(empty_bar(stage));
    if (++stage == stages) { stage = 0; phase ^= 1u; }
    // this warp's part of the tile; after the round's last tile meet the others and finish the round.  Two copies of
    // the parts, so one meeting per round is enough.
    const int in_round = i % kRound, parity = (i / kRound) & 1;
    float* const p = s_part[parity][in_round][warp] + g * 8 + 2 * t;
    *reinterpret_cast<float2*>(p) = make_float2(acc[0][0] + acc[1][0], acc[0][1] + acc[1][1]);
    if constexpr (kTokens == 2)
      *reinterpret_cast<float2*>(p + 64) = make_float2(acc[0][2] + acc[1][2], acc[0][3] + acc[1][3]);
    if (in_round + 1 < kRound && i + 1 < my_tiles) continue;
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
    const int which = threadIdx.x >> 6, in = threadIdx.x & 63;   // a finishing thread per tile of the round, token and row
    if (which <= in_round) {
      const int v = ((int)blockIdx.x + (i - in_round + which) * (int)gridDim.x) * kRows + (in & 7);
#pragma unroll
      for (int j = 0; j < kTokens; ++j) {
        const int tok = j * 8 + (in >> 3);
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum += s_part[parity][which][w][j * 64 + in];
        if (tok < T && v < V) {
          z[(size_t)tok * V + v] = sum;
          st[j].add(sum);
        }
      }
    }
  }

  static_assert(kThreads / 64 == kRound, "a finishing thread per tile of the round, token and row");

  // ---- states: over the finishing threads of a token, and to memory
#pragma unroll
  for (int j = 0; j < kTokens; ++j) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1)        // the 8 rows
      st[j].join(__shfl_xor_sync(0xffffffffu, st[j].m, o), __shfl_xor_sync(0xffffffffu, st[j].s, o),
                 __shfl_xor_sync(0xffffffffu, st[j].u, o));
    if ((lane & 7) == 0)
      s_state[threadIdx.x >> 6][j * 8 + ((threadIdx.x & 63) >> 3)] = make_float4(st[j].m, st[j].s, st[j].u, 0.f);
  }
  __syncthreads();
  if ((int)threadIdx.x < T) {
    SoftmaxState a{kNone, 0.f, 0.f};
    for (int w = 0; w < kRound; ++w) {
      const float4 v = s_state[w][threadIdx.x];
      a.join(v.x, v.y, v.z);
    }
    partial[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = make_float4(a.m, a.s, a.u, 0.f);
  }
  __threadfence();
  __syncthreads();
  if (abort_flag) {        // a bulk copy did not arrive in time: flag it, let copies in flight land
    if (threadIdx.x == 0) atomicOr(d_err, umma::kWatchdogBit);
    __nanosleep(1000000);
  }
  if (threadIdx.x == 0) s_last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  for (int tok = warp; tok < T; tok += kWarps) {
    SoftmaxState a{kNone, 0.f, 0.f};
    for (int i = lane; i < (int)gridDim.x; i += 32) {
      const float4 v = __ldcg(partial + (size_t)tok * gridDim.x + i);
      a.join(v.x, v.y, v.z);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      a.join(__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o),
             __shfl_xor_sync(0xffffffffu, a.u, o));
    const float log_s = logf(a.s), lse = a.m + log_s;
    if (lane == 0) {
      if (lse_out) lse_out[tok] = lse;
      if (entropy) entropy[tok] = log_s - a.u / (a.s * kLog2e);
    }
    for (int k = lane; k < K; k += 32) {
      const int id = __ldg(cand + (size_t)tok * K + k);
      float lq;
      if (id >= 0 && id < V) {
        lq = __ldcg(z + (size_t)tok * V + id) - lse;
      } else if (id < 0) {
        lq = -INFINITY;
      } else {
        lq = __int_as_float(0x7fc00000);
        atomicOr(d_err, AF_DEVERR_TARGET_RANGE);
      }
      cand_logp[(size_t)tok * K + k] = lq;
    }
  }
  if (threadIdx.x == 0) *ticket = 0;         // ready for the next call on this stream
}

int stream_stages(int d) {
  const int n = (kRingBytes - 128) / (kRows * d * 2);     // 128: a last line that is not whole is read past its end
  return n < kMaxStages ? n : kMaxStages;
}
int stream_lines(int d) { return ((d + kLineK - 1) / kLineK + kWarps - 1) / kWarps; }

template <int kTokens, int kLines>
af_status launch_stream(const StreamCall& c, int blocks, cudaStream_t s) {
  static SmemAttrOnce once;
  if (set_smem_once(once, candidate_stream_kernel<kTokens, kLines>, kRingBytes) != cudaSuccess) return AF_ERR_CUDA;
  const int stages = stream_stages(c.d);
  return launch_overlapped(candidate_stream_kernel<kTokens, kLines>, blocks, kThreads, (size_t)stages * kRows * c.d * 2 + 128, s,
                           static_cast<const uint4*>(c.hidden), static_cast<const char*>(c.W), c.cand, c.T, c.K, c.d, c.V, stages,
                           c.z, c.partial, c.cand_logp, c.entropy, c.lse, c.ticket, c.d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace

// Two stages of the ring at least, and a warp's part of the hidden states in registers: 8 of them per line and group
// of 8 tokens.
bool stream_fits(int64_t T, int32_t d) {
  return T <= kStreamTokens && stream_stages(d) >= 2 && stream_lines(d) <= (T <= 8 ? 12 : 8);
}

af_status launch_candidate_stream(const StreamCall& c, int sm_count, cudaStream_t s) {
  const int tiles = (c.V + kRows - 1) / kRows, blocks = tiles < sm_count ? tiles : sm_count;
  const int lines = stream_lines(c.d);
  if (c.T > 8) return lines <= 4 ? launch_stream<2, 4>(c, blocks, s) : launch_stream<2, 8>(c, blocks, s);
  if (lines <= 4) return launch_stream<1, 4>(c, blocks, s);
  if (lines <= 8) return launch_stream<1, 8>(c, blocks, s);
  return launch_stream<1, 12>(c, blocks, s);
}

}  // namespace af
