// af_quant_logits: one pass over the codes of a 4-bit head for up to 64 tokens, on the tensor cores.
//
//   logits[t, v] = sum_k hidden[t, k] * bf16(scale[v, k / group] * (digit[v, k] - 8))
//
// Few tokens make the head a stream of d / 2 bytes a row (and its scales), 280 MB for the 7B-shaped one, and turning digits
// into operands has to keep up with it: 45 weights per cycle and SM.  The rows of the head are the M of tcgen05.mma, the tokens
// its N, and the dequantised rows go from registers straight into tensor memory as its A operand: a thread has a row, and
// neither stores to shared memory nor sums across threads are needed.
//   (w >> s_i) & 0x00780078 | 0x41804180 is the pair 16 + u of bf16 of digits i and i + 4 of a word, neighbours in k;  times
//   the scale, less 24 scales, it is the pair of weights, in one fused multiply-add: exactly so where the scale has five
//   significant bits, as af_quantize_head's have (24 s then is a bf16).  Rows with other scales take the two steps.
// So a pair costs a shift, a mask-and-or (both on the ALU pipe, at half rate, which is what this kernel is bound by next to
// memory) and a multiply-add.
//
// Warps: 0 loads boxes of 256 weights by 128 rows and the tokens' 256 k into a ring, 1 issues the MMAs, the next four per
// 128 rows read accumulators, the others dequantise in groups of four, 128 weights of 128 rows at a time, into four buffers
// in tensor memory.  Sums are taken in parts of 512 of k, which the readers add in fp32, rounding to nearest (see umma.cuh on
// truncation).
#include "gemm_launch.cuh"
#include "rollout.cuh"

namespace af {
namespace {

using namespace umma;

constexpr int kRowsM = 128;                        // rows of an MMA
constexpr int kStageK = 256;                       // k of a stage: 128 bytes of codes
constexpr int kHalfK = 128;                        // k that a group dequantises at a time
constexpr int kBufs = 4;                           // of dequantised rows in tensor memory
constexpr int kBufCols = kHalfK / 2;               // columns of one: two bf16 each
constexpr int kBufCol0 = 256;
constexpr int kMiscWarps = 4;                      // loads, MMAs, and two that make the readers start at a quarter of TMEM's lanes
constexpr int kCodesBytes = kRowsM * 128;
constexpr int kMaxRing = 10;
constexpr int kSmemLimit = 225 * 1024;

__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// Digits i and i + 4 of a word as 16 + u, a pair of bf16.
template <int i>
__device__ __forceinline__ uint32_t digit_pair(uint32_t w) {
  const uint32_t at = i == 0 ? w << 3 : w >> (4 * i - 3);
  uint32_t u;
  asm("lop3.b32 %0, %1, 0x00780078, 0x41804180, 0xea;" : "=r"(u) : "r"(at));        // a & b | c
  return u;
}
constexpr uint32_t kMinus24 = 0xc1c0c1c0u, kOne2 = 0x3f803f80u, kZero2 = 0x80008000u;     // -24, 1 and -0 as pairs
struct Pair { uint32_t s, c; bool quick; };        // a scale twice, -24 of it, and whether that is exact
__device__ __forceinline__ Pair scale_pair(uint32_t bits) {
  const uint32_t s = bits | bits << 16;
  return {s, bf2_fma(s, kMinus24, kZero2), (bits & 7u) == 0 && (bits & 0x7fffu) < 0x7c00u};
}
template <bool kQuick>
__device__ __forceinline__ uint32_t weight_pair(uint32_t v, const Pair& p) {
  return kQuick ? bf2_fma(v, p.s, p.c) : bf2_fma(bf2_fma(v, kOne2, kMinus24), p.s, kZero2);
}
template <bool kQuick, int kPerHalf>
__device__ __forceinline__ void dequantise(const uint8_t* row, uint32_t swizzle, const Pair (&p)[kPerHalf], uint32_t to) {
#pragma unroll
  for (int piece = 0; piece < kHalfK / 32; ++piece) {
    const uint4 w4 = *reinterpret_cast<const uint4*>(row + (((uint32_t)piece << 4) ^ swizzle));
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    const Pair& s = p[piece * kPerHalf / 4];
    uint32_t r[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r[4 * j] = weight_pair<kQuick>(digit_pair<0>(w[j]), s);
      r[4 * j + 1] = weight_pair<kQuick>(digit_pair<1>(w[j]), s);
      r[4 * j + 2] = weight_pair<kQuick>(digit_pair<2>(w[j]), s);
      r[4 * j + 3] = weight_pair<kQuick>(digit_pair<3>(w[j]), s);
    }
    tmem_st16(to + piece * 16, r);
  }
}

struct UmmaShape {
  int T, V, d, groups;
  int halves, stages;            // pieces of 128 and of 256 of k in a row
  int rows_box;                  // rows of a box, 128 at most
  int boxes;                     // boxes of the head
  int ring;                      // stages of the ring
};

__device__ __forceinline__ void put_logit(void* logits, int type, int64_t at, float v) {
  if (type == AF_F32) static_cast<float*>(logits)[at] = v;
  else static_cast<__nv_bfloat16*>(logits)[at] = __float2bfloat16_rn(v);
}

// kN: tokens, rounded up; kM: boxes that share a stage's tokens; kGroups: of four dequantising warps; kPerHalf: scales in 128 weights.
template <int kM, int kGroups>
constexpr int kUmmaThreads = 32 * (kMiscWarps + 4 * kM + 4 * kGroups);
template <int kN, int kM>
constexpr int kUmmaStageBytes = kM * kCodesBytes + 4 * kN * 128;

template <int kN, int kM, int kGroups, int kPerHalf>
__global__ void __launch_bounds__(kUmmaThreads<kM, kGroups>, 1) quant_umma_kernel(
    const __grid_constant__ CUtensorMap codes, const __grid_constant__ CUtensorMap hidden, const __nv_bfloat16* __restrict__ scale,
    const UmmaShape sh, void* __restrict__ logits, int type, int64_t pitch, unsigned int* d_err) {
  constexpr int kStage = kUmmaStageBytes<kN, kM>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bars[2 * kMaxRing + 2 * kBufs + 4];
  __shared__ uint32_t s_tmem;
  __shared__ int abort_flag;
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t ring_at = smem_u32(smem), bars = smem_u32(s_bars);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kMaxRing + s); };
  auto a_full = [&](int b) { return bars + 8u * (2 * kMaxRing + b); };
  auto a_empty = [&](int b) { return bars + 8u * (2 * kMaxRing + kBufs + b); };
  auto acc_full = [&](int a) { return bars + 8u * (2 * kMaxRing + 2 * kBufs + a); };
  auto acc_empty = [&](int a) { return bars + 8u * (2 * kMaxRing + 2 * kBufs + 2 + a); };
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < sh.ring; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int b = 0; b < kBufs; ++b) { mbar_init(a_full(b), 4); mbar_init(a_empty(b), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), 4 * kM); }
    fence_mbar_init();
    tma_prefetch_desc(&codes);
    tma_prefetch_desc(&hidden);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&s_tmem), kTmemCols);
    tmem_relinquish();
  }
  wait_for_predecessor();
  let_successor_start();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  // boxes b, b + grid, ... are this CTA's; kM of them at a time are a tile
  const int my_boxes = (sh.boxes - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
  const int tiles = (my_boxes + kM - 1) / kM;
  auto boxes_in = [&](int tile) { return kM == 1 ? 1 : min(kM, my_boxes - tile * kM); };
  auto box_row = [&](int tile, int m) { return (int64_t)((int64_t)(tile * kM + m) * gridDim.x + blockIdx.x) * sh.rows_box; };
  auto halves_in = [&](int s) { return min(2, sh.halves - 2 * s); };

  if (warp == 0) {
    if (lane == 0) {                               // ---- loads
      int slot = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = 0; tile < tiles && ok; ++tile) {
        const int boxes = boxes_in(tile);
        for (int s = 0; s < sh.stages; ++s) {
          if (!mbar_wait(empty_bar(slot), phase ^ 1u, &abort_flag)) { ok = false; break; }
          const int blocks = min(4, (sh.d - s * kStageK + 63) / 64);
          const uint32_t at = ring_at + slot * kStage;
          mbar_arrive_expect_tx(full_bar(slot), boxes * sh.rows_box * 128 + blocks * kN * 128);
          for (int m = 0; m < boxes; ++m)
            tma_load_2d(at + m * kCodesBytes, &codes, full_bar(slot), s * (kStageK / 4), (int)box_row(tile, m));
          for (int b = 0; b < blocks; ++b)
            tma_load_2d(at + kM * kCodesBytes + b * kN * 128, &hidden, full_bar(slot), s * kStageK + b * 64, 0);
          if (++slot == sh.ring) { slot = 0; phase ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {                               // ---- products
      const uint32_t idesc = instr_desc_bf16_f32(kRowsM, kN);
      int slot = 0, buf = 0, acc = 0;
      uint32_t phase = 0, buf_phase = 0, acc_phase = 0;
      bool ok = true;
      for (int tile = 0; tile < tiles && ok; ++tile) {
        const int boxes = boxes_in(tile);
        for (int s = 0; s < sh.stages && ok; ++s) {
          if (!mbar_wait(full_bar(slot), phase, &abort_flag)) { ok = false; break; }
          if (s % 2 == 0 && !mbar_wait(acc_empty(acc), acc_phase ^ 1u, &abort_flag)) { ok = false; break; }
          const uint32_t x_at = ring_at + slot * kStage + kM * kCodesBytes;
          for (int h = 0; h < halves_in(s) && ok; ++h) {
            const int steps = min(kHalfK, sh.d - s * kStageK - h * kHalfK) / 16;
            for (int m = 0; m < boxes; ++m) {
              if (!mbar_wait(a_full(buf), buf_phase, &abort_flag)) { ok = false; break; }
              tc_fence_after();
              const uint32_t a_at = tmem + kBufCol0 + buf * kBufCols, d_at = tmem + (acc * kM + m) * kN;
              for (int k = 0; k < steps; ++k) {
                const uint64_t b_desc = smem_desc_k_sw128(x_at + (h * 2 + k / 4) * (kN * 128)) + (uint64_t)(k % 4) * 2;
                mma_bf16_ts(d_at, a_at + k * 8, b_desc, idesc, s % 2 == 0 && h == 0 && k == 0 ? 0u : 1u);
              }
              mma_commit(a_empty(buf));
              if (++buf == kBufs) { buf = 0; buf_phase ^= 1u; }
            }
          }
          if (!ok) break;
          mma_commit(empty_bar(slot));
          if (++slot == sh.ring) { slot = 0; phase ^= 1u; }
          if (s % 2 == 1 || s + 1 == sh.stages) {  // a part ends
            mma_commit(acc_full(acc));
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
          }
        }
      }
    }
    __syncwarp();
  } else if (warp >= kMiscWarps && warp < kMiscWarps + 4 * kM) {
    // ---- sums of the parts, and out
    const int m = (warp - kMiscWarps) / 4, quarter = warp & 3, r = quarter * 32 + lane;
    const int parts = (sh.stages + 1) / 2;
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int tile = 0; tile < tiles && ok; ++tile) {
      float sum[kN];
#pragma unroll
      for (int n = 0; n < kN; ++n) sum[n] = 0.f;
      const bool here = m < boxes_in(tile);
      for (int part = 0; part < parts; ++part) {
        ok = __all_sync(0xffffffffu, mbar_wait(acc_full(acc), acc_phase, &abort_flag));
        if (!ok) break;
        tc_fence_after();
        if (here) {
#pragma unroll
          for (int n0 = 0; n0 < kN; n0 += 16) {
            uint32_t v[16];
            tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + (acc * kM + m) * kN + n0, v);
            tmem_ld_wait();
#pragma unroll
            for (int n = 0; n < 16; ++n) sum[n0 + n] += __uint_as_float(v[n]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_empty(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      const int64_t v = box_row(tile, m) + r;
      if (ok && here && r < sh.rows_box && v < sh.V) {
#pragma unroll
        for (int n = 0; n < kN; ++n)
          if (n < sh.T) put_logit(logits, type, n * pitch + v, sum[n]);
      }
    }
  } else if (warp >= kMiscWarps + 4 * kM) {
    // ---- digits to weights
    const int group = (warp - kMiscWarps - 4 * kM) / 4, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t swizzle_row = (uint32_t)(r & 7) << 4;
    const bool row_in_box = r < sh.rows_box;
    // units in the order of the products: tile, stage, half, box
    int tile = 0, s = 0, h = 0, m = 0, slot = 0, buf = 0;
    uint32_t phase = 0, buf_phase = 0;
    auto next = [&] {
      if (++buf == kBufs) { buf = 0; buf_phase ^= 1u; }
      if (++m < boxes_in(tile)) return;
      m = 0;
      if (++h < halves_in(s)) return;
      h = 0;
      if (++slot == sh.ring) { slot = 0; phase ^= 1u; }
      if (++s < sh.stages) return;
      s = 0;
      ++tile;
    };
    uint32_t bits[kPerHalf];                       // the unit's scales, one unit ahead of its codes
    auto fetch = [&] {
      const int64_t v = tile < tiles ? box_row(tile, m) + r : sh.V;
      const int g0 = (2 * s + h) * kPerHalf;
#pragma unroll
      for (int k = 0; k < kPerHalf; ++k)
        bits[k] = row_in_box && v < sh.V ? __ldg(reinterpret_cast<const uint16_t*>(scale) + v * sh.groups + min(g0 + k, sh.groups - 1)) : 0u;
    };
    for (int k = 0; k < group; ++k) next();
    fetch();
    while (tile < tiles) {
      if (!__all_sync(0xffffffffu, mbar_wait(full_bar(slot), phase, &abort_flag))) break;
      const uint8_t* const row = smem + slot * kStage + m * kCodesBytes + r * 128;
      const uint32_t swizzle = ((uint32_t)h << 6) ^ swizzle_row;
      const int this_buf = buf;
      const uint32_t this_phase = buf_phase;
      Pair p[kPerHalf];
      bool quick = true;
#pragma unroll
      for (int k = 0; k < kPerHalf; ++k) { p[k] = scale_pair(bits[k]); quick = quick && p[k].quick; }
      quick = __all_sync(0xffffffffu, quick);
      for (int k = 0; k < kGroups; ++k) next();
      fetch();
      if (!__all_sync(0xffffffffu, mbar_wait(a_empty(this_buf), this_phase ^ 1u, &abort_flag))) break;
      tc_fence_after();
      const uint32_t to = tmem + ((uint32_t)(quarter * 32) << 16) + kBufCol0 + this_buf * kBufCols;
      if (quick) dequantise<true, kPerHalf>(row, swizzle, p, to);
      else dequantise<false, kPerHalf>(row, swizzle, p, to);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(a_full(this_buf));
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (abort_flag) {                                // a wait ran out of time: flag it, let copies in flight land
    if (threadIdx.x == 0) atomicOr(d_err, kWatchdogBit);
    __nanosleep(1000000);
  }
  if (warp == 1) tmem_dealloc(tmem, kTmemCols);
}

template <int kN, int kM, int kGroups, int kPerHalf>
af_status launch_umma(af_ctx* ctx, const void* hidden, const QuantHead& h, int T, void* logits, int type, int64_t pitch, cudaStream_t s) {
  UmmaShape sh;
  sh.T = T; sh.V = h.V; sh.d = h.d; sh.groups = h.groups();
  sh.halves = (h.d + kHalfK - 1) / kHalfK;
  sh.stages = (h.d + kStageK - 1) / kStageK;
  // boxes of one size, as many to every CTA: 128 rows or a little less
  const int64_t per_cta = ((int64_t)h.V + (int64_t)ctx->sm_count * kRowsM - 1) / ((int64_t)ctx->sm_count * kRowsM);
  const int64_t want = per_cta * ctx->sm_count;
  sh.rows_box = (int)((h.V + want - 1) / want);
  sh.boxes = (h.V + sh.rows_box - 1) / sh.rows_box;
  constexpr int stage = kUmmaStageBytes<kN, kM>, ring = (kSmemLimit - 1024) / stage < kMaxRing ? (kSmemLimit - 1024) / stage : kMaxRing;
  sh.ring = ring;
  constexpr int smem = 1024 + ring * stage;
  CUtensorMap codes, x;                            // the codes as a matrix of d / 4 16-bit elements
  const GemmEnv env = gemm_env(ctx);
  af_status st = encode_operand(env, &codes, Operand{h.codes, (uint64_t)h.V, (uint64_t)h.d / 4, (uint64_t)h.d / 2}, (uint32_t)sh.rows_box);
  if (st == AF_OK) st = encode_operand(env, &x, Operand{hidden, (uint64_t)T, (uint64_t)h.d, (uint64_t)h.d * 2}, kN);
  if (st != AF_OK) return st;
  static SmemAttrOnce once;
  if (set_smem_once(once, quant_umma_kernel<kN, kM, kGroups, kPerHalf>, smem) != cudaSuccess) return AF_ERR_CUDA;
  const int blocks = sh.boxes < ctx->sm_count ? sh.boxes : ctx->sm_count;
  return launch_overlapped(quant_umma_kernel<kN, kM, kGroups, kPerHalf>, blocks, kUmmaThreads<kM, kGroups>, smem, s, codes, x, h.scale, sh,
                           logits, type, pitch, ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}
template <int kN, int kM, int kGroups>
af_status launch_umma_group(af_ctx* ctx, const void* hidden, const QuantHead& h, int T, void* logits, int type, int64_t pitch, cudaStream_t s) {
  if (h.group == 32) return launch_umma<kN, kM, kGroups, 4>(ctx, hidden, h, T, logits, type, pitch, s);
  if (h.group == 64) return launch_umma<kN, kM, kGroups, 2>(ctx, hidden, h, T, logits, type, pitch, s);
  return launch_umma<kN, kM, kGroups, 1>(ctx, hidden, h, T, logits, type, pitch, s);
}

}  // namespace

af_status launch_quant_umma(af_ctx* ctx, const void* hidden, const QuantHead& h, int T, void* logits, int32_t type, int64_t pitch,
                            cudaStream_t s) {
  if (T <= 16) return launch_umma_group<16, 1, 2>(ctx, hidden, h, T, logits, type, pitch, s);
  if (T <= 32) return launch_umma_group<32, 1, 2>(ctx, hidden, h, T, logits, type, pitch, s);
  return launch_umma_group<64, 1, 2>(ctx, hidden, h, T, logits, type, pitch, s);
}

}  // namespace af
