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
// So a pair costs a shift, a mask-and-or (both on the ALU pipe, at half rate) and a multiply-add.
//
// 152064 x 3584, groups of 128: one token 62-72 us, 3.9-4.5 TB/s of codes and scales, 64 tokens 100-120 us; 151643 x 5120, groups of
// 32, 16 tokens: 105-125 us.  One token keeps the ALU pipe busy 64 % of the time, issue slots 69 %, memory 50 %: what is left
// are the hand-overs from stage to buffer to product (shifts as multiplications on the idler pipe: no faster, or 10 % slower).
//
// Warps: 0 loads stages of 256 of k into a ring (the codes of a box of 128 rows, or of two, and the tokens'), 1 and 2 issue the
// MMAs, each for an accumulator of its own, the next four (or eight) read accumulators, the others dequantise, in groups of four
// warps with two buffers of 128 of k in tensor memory each, so that a group writes one while the other is multiplied.  Sums are
// taken in parts of 512 of k, which the readers add in fp32, rounding to nearest (see umma.cuh on truncation).
// Up to 32 tokens: one box a stage, three groups taking stages in turn, the accumulators taking parts in turn.  More: the
// tokens' share of a stage, fetched from L2 by every CTA, outweighs the codes', so two boxes share it, each with its group,
// accumulator and readers.
#include "gemm_launch.cuh"
#include "rollout.cuh"

namespace af {
namespace {

using namespace umma;

constexpr int kRowsM = 128;                        // rows of an MMA
constexpr int kStageK = 256;                       // k of a stage: 128 bytes of codes
constexpr int kHalfK = 128;                        // k of a buffer of dequantised rows
constexpr int kBufCols = kHalfK / 2;               // its columns: two bf16 each
constexpr int kBufCol0 = 128;                      // behind two accumulators of up to 64 columns
constexpr int kReaders = 4;                        // the first of the warps that read accumulators: a multiple of 4, as TMEM's lanes go
constexpr int kCodesBytes = kRowsM * 128;
constexpr int kMaxRing = 9, kMaxBufs = 6;
constexpr int kSmemLimit = 225 * 1024;
// kM: boxes that share a stage.
template <int kM>
struct Roles {
  static constexpr int kGroups = kM == 1 ? 3 : 2;  // of four dequantising warps
  static constexpr int kFirstGroup = kReaders + 4 * kM;
  static constexpr int kThreads = 32 * (kFirstGroup + 4 * kGroups);
};
template <int kN, int kM>
struct Stage {
  static constexpr int kTokensAt = kM * kCodesBytes;
  static constexpr int kBytes = kTokensAt + 4 * kN * 128;
  // with one box a slot belongs to one group, which so has seen each of its phases: a parity cannot be mistaken for that of the
  // phase before the last
  static constexpr int kFit = (kSmemLimit - 1024) / kBytes, kMost = kFit < kMaxRing ? kFit : kMaxRing;
  static constexpr int kRing = kM == 1 ? kMost / Roles<1>::kGroups * Roles<1>::kGroups : kMost;
  static_assert(kRing >= 3, "loads ahead of the products");
};

// The dequantising warps sleep while they wait (mbar_sleep_wait): the scheduler's issue slots belong to those that have work.  A warp
// that others wait for keeps asking for a while first.
__device__ __forceinline__ bool ready_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
#pragma unroll 1
  for (int i = 0; i < 64; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return mbar_sleep_wait(bar, parity, abort_flag);
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst_smem, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst_smem), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
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
// 128 of k of a row, with scales p[first], ...; piece0: 16-byte piece of the line that they start at.
template <bool kQuick, int kScales, int kPiece0>
__device__ __forceinline__ void dequantise(const uint8_t* row, uint32_t swizzle, const Pair (&p)[kScales], uint32_t to) {
#pragma unroll
  for (int piece = kPiece0; piece < kPiece0 + kHalfK / 32; ++piece) {
    const uint4 w4 = *reinterpret_cast<const uint4*>(row + (((uint32_t)piece << 4) ^ swizzle));
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    const Pair& s = p[piece * kScales / (kStageK / 32)];
    uint32_t r[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r[4 * j] = weight_pair<kQuick>(digit_pair<0>(w[j]), s);
      r[4 * j + 1] = weight_pair<kQuick>(digit_pair<1>(w[j]), s);
      r[4 * j + 2] = weight_pair<kQuick>(digit_pair<2>(w[j]), s);
      r[4 * j + 3] = weight_pair<kQuick>(digit_pair<3>(w[j]), s);
    }
    tmem_st16(to + (piece - kPiece0) * 16, r);
  }
}

struct UmmaShape {
  int T, V, d, groups;
  int stages;                    // pieces of 256 of k in a row
  int rows_box;                  // rows of a box, 128 at most
  int boxes;                     // boxes of the head
  int whole_blocks;              // d is a multiple of 64: the tokens' map has a third dimension, the blocks of 64 of k
};

__device__ __forceinline__ void put_logit(void* logits, int type, int64_t at, float v) {
  if (type == AF_F32) static_cast<float*>(logits)[at] = v;
  else static_cast<__nv_bfloat16*>(logits)[at] = __float2bfloat16_rn(v);
}

// kN: tokens, rounded up; kM: boxes that share a stage; kScales: scales in 256 weights.
template <int kN, int kM, int kScales>
__global__ void __launch_bounds__(Roles<kM>::kThreads, 1) quant_umma_kernel(
    const __grid_constant__ CUtensorMap codes, const __grid_constant__ CUtensorMap hidden, const __nv_bfloat16* __restrict__ scale,
    const UmmaShape sh, void* __restrict__ logits, int type, int64_t pitch, unsigned int* d_err) {
  using St = Stage<kN, kM>;
  constexpr int kStage = St::kBytes, kRing = St::kRing, kGroups = Roles<kM>::kGroups;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bars[2 * kRing + 3 * kMaxBufs + 4];
  __shared__ uint32_t s_tmem;
  __shared__ int abort_flag;
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t ring_at = smem_u32(smem), bars = smem_u32(s_bars);
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kRing + s); };
  // a buffer is full for one of the accumulators: each issuing warp follows its own barriers, phase by phase
  auto a_full = [&](int a, int group, int half) { return bars + 8u * (2 * kRing + kMaxBufs * a + 2 * group + half); };
  auto a_empty = [&](int group, int half) { return bars + 8u * (2 * kRing + 2 * kMaxBufs + 2 * group + half); };
  auto acc_full = [&](int a) { return bars + 8u * (2 * kRing + 3 * kMaxBufs + a); };
  auto acc_empty = [&](int a) { return bars + 8u * (2 * kRing + 3 * kMaxBufs + 2 + a); };
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < kRing; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), kM); }
    for (int b = 0; b < 2 * kGroups; ++b) { mbar_init(a_full(0, 0, b), 4); mbar_init(a_full(1, 0, b), 4); mbar_init(a_empty(0, b), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), 4); }
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
  const int boxes = (sh.boxes - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x, tiles = (boxes + kM - 1) / kM;
  const int64_t row0 = (int64_t)blockIdx.x * sh.rows_box, row_step = (int64_t)gridDim.x * sh.rows_box;
  const int parts = (sh.stages + 1) / 2;

  if (warp == 0) {
    // ---- loads
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = 0; tile < tiles && ok; ++tile) {
      const int here = min(kM, boxes - tile * kM);
      const int row = (int)(row0 + tile * kM * row_step);
      for (int s = 0; s < sh.stages; ++s) {
        ok = __all_sync(0xffffffffu, ready_wait(empty_bar(slot), phase ^ 1u, &abort_flag));
        if (!ok) break;
        const int blocks = min(4, (sh.d - s * kStageK + 63) / 64);
        const uint32_t at = ring_at + slot * kStage;
        if (elect_one()) {
          mbar_arrive_expect_tx(full_bar(slot), here * sh.rows_box * 128 + (sh.whole_blocks ? 4 : blocks) * kN * 128);
          tma_load_2d(at, &codes, full_bar(slot), s * (kStageK / 4), row);
          if (kM == 2 && here == 2) tma_load_2d(at + kCodesBytes, &codes, full_bar(slot), s * (kStageK / 4), row + (int)row_step);
          if (sh.whole_blocks) {                   // all blocks of 64 of k at once; those past the row arrive as zeros
            tma_load_3d(at + St::kTokensAt, &hidden, full_bar(slot), 0, 0, s * 4);
          } else {
            for (int b = 0; b < blocks; ++b)
              tma_load_2d(at + St::kTokensAt + b * kN * 128, &hidden, full_bar(slot), s * kStageK + b * 64, 0);
          }
        }
        __syncwarp();
        if (++slot == kRing) { slot = 0; phase ^= 1u; }
      }
    }
  } else if (warp <= 2) {
    // ---- products: the whole warp keeps step, one lane issues; so that addresses stay in uniform registers
    const int a = warp - 1;                        // its accumulator
    const uint32_t idesc = instr_desc_bf16_f32(kRowsM, kN), d_at = tmem + a * kN;
    const uint64_t desc0 = smem_desc_k_sw128(ring_at + St::kTokensAt);
    int slot = 0, group = kM == 1 ? 0 : a, part = 0;
    uint32_t phase = 0, acc_phase = 0, seen = 0;   // seen: a bit per group, the parity of what it has handed this warp
    bool ok = true;
    for (int tile = 0; tile < tiles && ok; ++tile) {
      const bool absent = kM == 2 && tile * kM + a >= boxes;
      for (int s = 0; s < sh.stages; ++s) {
        const bool part_ends = s % 2 == 1 || s + 1 == sh.stages;
        if (absent) {                              // the last tile has one box: its stages are freed for the other accumulator
          ok = __all_sync(0xffffffffu, ready_wait(full_bar(slot), phase, &abort_flag));
          if (!ok) break;
          if (elect_one()) mbar_arrive(empty_bar(slot));
        } else if (kM == 2 || (part & 1) == a) {
          if (s % 2 == 0) ok = __all_sync(0xffffffffu, ready_wait(acc_empty(a), acc_phase ^ 1u, &abort_flag));
          const uint64_t desc = desc0 + (uint64_t)(uint32_t)(slot * (kStage / 16));
          const uint32_t a_at = tmem + kBufCol0 + group * (2 * kBufCols);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            // a group that hands rows over has seen their stage arrive, the tokens with it
            ok = ok && __all_sync(0xffffffffu, ready_wait(a_full(a, group, half), seen >> group & 1u, &abort_flag));
            if (!ok) break;
            tc_fence_after();
            const int steps = min(kHalfK, sh.d - s * kStageK - half * kHalfK) / 16;       // none: a last half past the row
            if (elect_one()) {
              auto product = [&](int k) {
                mma_bf16_ts(d_at, a_at + half * kBufCols + k * 8, desc + (uint64_t)((2 * half + k / 4) * (kN * 128 / 16) + (k % 4) * 2), idesc,
                            half + k != 0 ? 1u : (uint32_t)(s % 2));
              };
              if (steps == kHalfK / 16) {
#pragma unroll
                for (int k = 0; k < kHalfK / 16; ++k) product(k);
              } else {
                for (int k = 0; k < steps; ++k) product(k);
              }
              mma_commit(a_empty(group, half));
              if (half == 1) mma_commit(empty_bar(slot));
              if (half == 1 && part_ends) mma_commit(acc_full(a));
            }
            __syncwarp();
          }
          if (!ok) break;
          seen ^= 1u << group;
          if (part_ends) acc_phase ^= 1u;
        }
        if (part_ends) ++part;
        if (kM == 1 && ++group == kGroups) group = 0;
        if (++slot == kRing) { slot = 0; phase ^= 1u; }
      }
    }
  } else if (warp >= kReaders && warp < Roles<kM>::kFirstGroup) {
    // ---- sums of the parts, and out
    const int m = (warp - kReaders) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    int a = m;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int box = m; box < boxes && ok; box += kM) {
      float sum[kN];
#pragma unroll
      for (int n = 0; n < kN; ++n) sum[n] = 0.f;
      for (int part = 0; part < parts; ++part) {
        ok = __all_sync(0xffffffffu, mbar_sleep_wait(acc_full(a), acc_phase, &abort_flag));
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int n0 = 0; n0 < kN; n0 += 16) {
          uint32_t v[16];
          tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + a * kN + n0, v);
          tmem_ld_wait();
#pragma unroll
          for (int n = 0; n < 16; ++n) sum[n0 + n] += __uint_as_float(v[n]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_empty(a));
        if (kM == 2 || (a ^= 1) == 0) acc_phase ^= 1u;
      }
      const int64_t v = row0 + box * row_step + r;
      if (ok && r < sh.rows_box && v < sh.V) {
#pragma unroll
        for (int n = 0; n < kN; ++n)
          if (n < sh.T) put_logit(logits, type, n * pitch + v, sum[n]);
      }
    }
  } else if (warp >= Roles<kM>::kFirstGroup) {
    // ---- digits to weights: one box a stage: every third stage; two: every stage of one of them
    const int group = (warp - Roles<kM>::kFirstGroup) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    constexpr int kTurn = kM == 1 ? kGroups : 1;   // stages from turn to turn
    const uint32_t swizzle = (uint32_t)(r & 7) << 4;
    const uint32_t to = tmem + ((uint32_t)(quarter * 32) << 16) + kBufCol0 + group * (2 * kBufCols);
    const uint8_t* const rows = smem + (kM == 1 ? 0 : group * kCodesBytes) + r * 128;
    int box = kM == 1 ? 0 : group, s = kM == 1 ? group : 0, slot = s;
    auto owner = [&] { return kM == 1 ? (box * parts + (s >> 1)) & 1 : group; };   // accumulator of the stage's part
    uint32_t phase = 0, buf_phase = 0;
    while (s >= sh.stages) { s -= sh.stages; box += kM; }
    int64_t v = row0 + box * row_step + r;
    // the stage's scales, one turn ahead of its codes
    const uint16_t* const scales = reinterpret_cast<const uint16_t*>(scale);
    uint32_t bits[kScales];
    auto fetch = [&] {
      const bool in = box < boxes && r < sh.rows_box && v < sh.V;
#pragma unroll
      for (int k = 0; k < kScales; ++k) bits[k] = in ? __ldg(scales + v * sh.groups + min(s * kScales + k, sh.groups - 1)) : 0u;
    };
    fetch();
    while (box < boxes) {
      Pair p[kScales];
      bool quick = true;
#pragma unroll
      for (int k = 0; k < kScales; ++k) { p[k] = scale_pair(bits[k]); quick = quick && p[k].quick; }
      quick = __all_sync(0xffffffffu, quick);
      const uint8_t* const row = rows + slot * kStage;
      const int a = owner();
      if (!__all_sync(0xffffffffu, mbar_sleep_wait(full_bar(slot), phase, &abort_flag) && mbar_sleep_wait(a_empty(group, 0), buf_phase ^ 1u, &abort_flag))) break;
      slot += kTurn;
      if (slot >= kRing) { slot -= kRing; phase ^= 1u; }
      s += kTurn;
      while (s >= sh.stages) { s -= sh.stages; box += kM; v += kM * row_step; }
      fetch();
      auto hand_over = [&](int half) {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(a_full(a, group, half));
      };
      tc_fence_after();
      if (quick) dequantise<true, kScales, 0>(row, swizzle, p, to);
      else dequantise<false, kScales, 0>(row, swizzle, p, to);
      hand_over(0);
      if (!__all_sync(0xffffffffu, mbar_sleep_wait(a_empty(group, 1), buf_phase ^ 1u, &abort_flag))) break;
      tc_fence_after();
      if (quick) dequantise<true, kScales, 4>(row, swizzle, p, to + kBufCols);
      else dequantise<false, kScales, 4>(row, swizzle, p, to + kBufCols);
      hand_over(1);
      buf_phase ^= 1u;
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

// hidden [T, d] as [d / 64][T][64], boxes of four blocks of n tokens.
af_status encode_tokens(af_ctx* ctx, CUtensorMap* map, const void* hidden, int T, int d, uint32_t n) {
  const cuuint64_t dims[3] = {64, (cuuint64_t)T, (cuuint64_t)d / 64}, strides[2] = {(cuuint64_t)d * 2, 128};
  const cuuint32_t box[3] = {64, n, 4}, step[3] = {1, 1, 1};
  return ctx->encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(hidden), dims, strides, box, step,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? AF_OK : AF_ERR_CUDA;
}

template <int kN, int kM, int kScales>
af_status launch_umma(af_ctx* ctx, const void* hidden, const QuantHead& h, int T, void* logits, int type, int64_t pitch, cudaStream_t s) {
  UmmaShape sh;
  sh.T = T; sh.V = h.V; sh.d = h.d; sh.groups = h.groups();
  sh.stages = (h.d + kStageK - 1) / kStageK;
  // boxes of one size, as many to every CTA: 128 rows or a little less
  const int64_t per_cta = ((int64_t)h.V + (int64_t)ctx->sm_count * kRowsM - 1) / ((int64_t)ctx->sm_count * kRowsM);
  const int64_t want = per_cta * ctx->sm_count;
  sh.rows_box = (int)((h.V + want - 1) / want);
  sh.boxes = (h.V + sh.rows_box - 1) / sh.rows_box;
  constexpr int smem = 1024 + Stage<kN, kM>::kRing * Stage<kN, kM>::kBytes;
  CUtensorMap codes, x;                            // the codes as a matrix of d / 4 16-bit elements
  const GemmEnv env = gemm_env(ctx);
  af_status st = encode_operand(env, &codes, Operand{h.codes, (uint64_t)h.V, (uint64_t)h.d / 4, (uint64_t)h.d / 2}, (uint32_t)sh.rows_box);
  sh.whole_blocks = h.d % 64 == 0;
  if (st == AF_OK && !sh.whole_blocks) st = encode_operand(env, &x, Operand{hidden, (uint64_t)T, (uint64_t)h.d, (uint64_t)h.d * 2}, kN);
  if (st == AF_OK && sh.whole_blocks) st = encode_tokens(ctx, &x, hidden, T, h.d, kN);
  if (st != AF_OK) return st;
  static SmemAttrOnce once;
  if (set_smem_once(once, quant_umma_kernel<kN, kM, kScales>, smem) != cudaSuccess) return AF_ERR_CUDA;
  const int blocks = sh.boxes < ctx->sm_count ? sh.boxes : ctx->sm_count;
  return launch_overlapped(quant_umma_kernel<kN, kM, kScales>, blocks, Roles<kM>::kThreads, smem, s, codes, x, h.scale, sh, logits, type, pitch,
                           ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}
template <int kN, int kM>
af_status launch_umma_group(af_ctx* ctx, const void* hidden, const QuantHead& h, int T, void* logits, int type, int64_t pitch, cudaStream_t s) {
  if (h.group == 32) return launch_umma<kN, kM, 8>(ctx, hidden, h, T, logits, type, pitch, s);
  if (h.group == 64) return launch_umma<kN, kM, 4>(ctx, hidden, h, T, logits, type, pitch, s);
  return launch_umma<kN, kM, 2>(ctx, hidden, h, T, logits, type, pitch, s);
}

}  // namespace

af_status launch_quant_umma(af_ctx* ctx, const void* hidden, const QuantHead& h, int T, void* logits, int32_t type, int64_t pitch,
                            cudaStream_t s) {
  // more tokens than the batch has are products for nothing; from 33 on two boxes share a stage's tokens.  For 16 / 32 / 64, on the
  // 152064 x 3584 head with scales of any kind: 1 token 73 / 83 / 105 us, 16 tokens 74 / 77 / 103, 17 - / 77 / 101, 32 - / 82 / 100
  if (T <= 16) return launch_umma_group<16, 1>(ctx, hidden, h, T, logits, type, pitch, s);
  if (T <= 32) return launch_umma_group<32, 1>(ctx, hidden, h, T, logits, type, pitch, s);
  return launch_umma_group<64, 2>(ctx, hidden, h, T, logits, type, pitch, s);
}

}  // namespace af
