// af_distill_loss: divergence between a teacher's and the student's log-probs of K listed ids per token,
// and its gradient in the student's log-probs, in one pass (8 bytes read and 4 written per slot: HBM-bound).
//
// kG lanes of a warp share a row and hold kE of its slots each, so a row's sums and maxima are a few
// shuffles inside the group and every value is read once.  At full bandwidth an SM takes about two slots
// per clock, which leaves some 60 thread instructions for each: sixteen slots per lane keep the shuffles of up
// to five row reductions and the row's bookkeeping at a few instructions per slot (with eight, the
// renormalised divergences took 1.15 times as long), and the slots that take no part are turned into
// values whose every term is 0 once, at the load.  The rows of a step are contiguous in memory: one
// thread feeds a ring of two shared-memory stages with bulk copies of both columns, one step while the other is
// worked on, so the bytes in flight do not depend on registers, and a warp's gradients leave the same way, as
// one bulk store of its rows from the stage they came in.
// Measured: 1106674 rows of 50 slots, student to teacher with a tail, 113-122 us (5.9-5.5 TB/s, several B200s); of 64 slots
// 148 us (5.8 TB/s); 2000000 rows of 16, 67 us (5.9 TB/s); 32768 rows of 64, renormalised, 12 us in a graph (13-14 called one
// by one), half of it launch, first loads and the last block's sum.
// Row sums are taken in fp32 over at most 256 terms in a fixed tree, a lane's over up to 256 rows (K = 1; 128 or fewer
// from there on) in fp32, the batch's in fp64, all in a fixed order: results are bit-reproducible.  The exponentials are
// ex2.approx (2^-22): a token's loss is within 2e-7 of 64 bits renormalised and 6e-7 with a tail, in root mean square.
#pragma once

#include "common.cuh"
#include "device_util.cuh"
#include "umma.cuh"

namespace af {
namespace distill {

constexpr int kThreads = 128;
constexpr int kBlocksPerSm = 4;
constexpr int kNumSums = 3;                // weighted loss, teacher mass, student mass
constexpr float kTailFloor = 1.f / 65536.f;
constexpr int kStageSlots = kThreads * 16; // slots of one column in a ring stage, at most
constexpr int kStageBytes = 2 * kStageSlots * 4;
constexpr int kStages = 2;                // three kept more in flight and were slower (K = 50: 127 us against 111)
constexpr int kFlush = 16;                 // steps whose sums a lane keeps in fp32 (at most 256 rows) before fp64
constexpr int kSmemBytes = kStages * kStageBytes + 128 /*alignment*/ + 64 /*barriers*/ + 1024 /*reads past a row*/;

struct DistillWs {                         // the header and blocks of the policy loss's reduction workspace
  unsigned int ticket;
  unsigned int pad[15];
};
__device__ __forceinline__ double* ws_partial(DistillWs* ws, int block) {
  return reinterpret_cast<double*>(ws + 1) + (size_t)block * 4;
}

__device__ __forceinline__ void bulk_load(uint32_t dst_smem, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               :: "r"(dst_smem), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

__device__ __forceinline__ void bulk_store(void* dst, uint32_t src_smem, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" :: "l"(dst), "r"(src_smem), "r"(bytes) : "memory");
}

// min(v, 1e30), so that times 0 is 0; a NaN stays one (fminf would drop it).
__device__ __forceinline__ float finite_above(float v) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(1.0e30f));
  return r;
}

// a log(a / b) + b - a with d = log(a / b): the terms of a divergence between two distributions, each of them
// non-negative.  The b - a sum to nothing, but with them an error of the sums that normalise a and b, which
// shifts every d alike, no longer moves the result to first order.
__device__ __forceinline__ float divergence_term(float a, float b, float d) {
  // (e^-d - 1 + d) / d^2 by its series (at 0.5 the first term left out is 8e-7 of it)
  float f = fmaf(d, -1.f / 5040.f, 1.f / 720.f);
  f = fmaf(d, -f, 1.f / 120.f);
  f = fmaf(d, -f, 1.f / 24.f);
  f = fmaf(d, -f, 1.f / 6.f);
  f = fmaf(d, -f, 0.5f);
  const float series = (a * d) * (d * f);
  const float direct = a == 0.f ? b : fmaf(a, d, b - a);      // d is infinite where b is 0; a NaN stays one
  return fabsf(d) < 0.5f ? series : direct;
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
__device__ __forceinline__ void load_slots(uint32_t addr, float* v) {
  if constexpr (kVec == 4)
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr));
  else if constexpr (kVec == 2)
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(addr));
  else
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[0]) : "r"(addr));
}
template <int kVec>
__device__ __forceinline__ void store_slots_shared(uint32_t addr, const float* v) {
  if constexpr (kVec == 4)
    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
  else if constexpr (kVec == 2)
    asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(addr), "f"(v[0]), "f"(v[1]) : "memory");
  else
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v[0]) : "memory");
}
template <int kVec>
__device__ __forceinline__ void store_slots(float* p, const float* v) {
  if constexpr (kVec == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  else if constexpr (kVec == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  else *p = v[0];
}

// What a distribution's listed probabilities leave of 1: a small difference, so they are added up in 64 bits, from
// sums of four (one conversion for every slot would cost as much as the rest of the row).
template <int kG, int kE>
__device__ __forceinline__ float group_rest(const float (&v)[kE]) {
  double x = 0.0;
#pragma unroll
  for (int i = 0; i < kE; i += 4) {
    float four = v[i];
#pragma unroll
    for (int j = i + 1; j < kE && j < i + 4; ++j) four += v[j];
    x += (double)four;
  }
#pragma unroll
  for (int o = kG / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return (float)(1.0 - x);
}

constexpr float kAbsentLogp = -1.0e30f;      // its exponential is 0; finite, so that a row's maximum of these is a number

// The divergence of one row and its gradient: lane `lane` of the group holds the slots lt / lq, absent ones
// (and those past K) with kAbsentLogp and -inf, which makes every term of theirs 0 (the student's is -inf so that a
// student with nothing on the present slots does not find its maximum among the absent ones).  Returns the row's loss
// (all lanes); g receives dloss/dlq; tm and sm gain the lane's share of the teacher's and the student's mass.
template <int kSupport, bool kForward, int kG, int kE>
__device__ __forceinline__ float row_divergence(const float (&lt)[kE], const float (&lq)[kE], float tau, float inv_tau,
                                                float (&g)[kE], float& tm, float& sm) {
  if constexpr (kSupport == 1) {
    // a = softmax(lt / tau), b = softmax(lq / tau) over the present slots; d = log a - log b
    float ma = lt[0], mb = lq[0];
#pragma unroll
    for (int i = 1; i < kE; ++i) {
      ma = fmaxf(ma, lt[i]);
      mb = fmaxf(mb, lq[i]);
    }
    ma = group_max<kG>(ma);
    mb = group_max<kG>(mb);
    // a row without any slot: shifted by nothing, all of its exponentials are 0
    if (ma <= kAbsentLogp) { ma = 0.f; mb = 0.f; }
    const float c = kLog2e * inv_tau, ca = -ma * c, cb = -mb * c;
    float za = 0.f, zb = 0.f;
    float a[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      a[i] = ex2f(fmaf(lt[i], c, ca));
      g[i] = ex2f(fmaf(lq[i], c, cb));
      za += a[i];
      zb += g[i];
    }
    if (tau != 1.f) {
#pragma unroll
      for (int i = 0; i < kE; ++i) { tm += ex2f(lt[i] * kLog2e); sm += ex2f(lq[i] * kLog2e); }
    } else {
      tm = fmaf(ex2f(ma * kLog2e), za, tm);
      // a student with nothing on the present slots has no distribution over them (zb is NaN, as the loss is), but a mass
      if (mb != -INFINITY) sm = fmaf(ex2f(mb * kLog2e), zb, sm);
    }
    za = group_sum<kG>(za);
    zb = group_sum<kG>(zb);
    const float ia = za != 0.f ? 1.f / za : 0.f, ib = zb != 0.f ? 1.f / zb : 0.f;
    const float shift = za != 0.f ? fmaf(mb - ma, inv_tau, logf(zb * ia)) : 0.f;   // log of the ratio of the sums
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const float d = fmaf(lt[i] - lq[i], inv_tau, shift);
      const float p = a[i] * ia, b = g[i] * ib;
      if constexpr (kForward) {
        loss += divergence_term(p, b, d);
        g[i] = tau * (b - p);
      } else {
        loss += divergence_term(b, p, -d);
        a[i] = finite_above(d);                 // kept for the gradient: b = 0 gives 0
        g[i] = tau * b;
      }
    }
    loss = group_sum<kG>(loss);
    if constexpr (!kForward) {
#pragma unroll
      for (int i = 0; i < kE; ++i) g[i] *= -a[i] - loss;
    }
    return tau * tau * loss;
  } else {
    float loss = 0.f, ps = 0.f, qs = 0.f;
    float q[kE], listed[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      const float p = ex2f(lt[i] * kLog2e);
      listed[i] = p;
      q[i] = ex2f(lq[i] * kLog2e);
      float gap = lt[i] - lq[i];
      ps += p;
      qs += q[i];
      if constexpr (kForward) {
        loss = fmaf(p, p == 0.f ? finite_above(gap) : gap, loss);      // an infinite gap counts where p > 0
        g[i] = -p;
      } else {
        gap = finite_above(gap);                // a q of 0 gives 0
        loss -= q[i] * gap;
        g[i] = fmaf(-q[i], gap, q[i]);
      }
    }
    tm += ps;
    sm += qs;
    if constexpr (kSupport == 2) {
      // one more outcome holds what the listed ones leave of either distribution
      const float p_left = group_rest<kG>(listed), q_left = group_rest<kG>(q);
      const float pr = p_left < kTailFloor ? kTailFloor : p_left, qr = q_left < kTailFloor ? kTailFloor : q_left;
      // approximate: off by 2^-22 of a ratio near 1, and weighted with the tail's mass
      const float quot = pr / qr, ratio = logf(quot);
      const float slope = q_left <= kTailFloor ? 0.f : kForward ? quot : ratio - 1.f;
#pragma unroll
      for (int i = 0; i < kE; ++i) g[i] = fmaf(q[i], slope, g[i]);
      return group_sum<kG>(loss) + (kForward ? pr * ratio : -qr * ratio);
    }
    return group_sum<kG>(loss);
  }
}

template <int kSupport, bool kForward, int kG, int kE, int kVec>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) distill_loss_kernel(
    const float* __restrict__ cand_logp, const float* __restrict__ teacher_logp, const int32_t* __restrict__ cu, int B,
    int T, int t0, int rows, int K, int batches, int bulk, af_distill_params prm, af_distill_out* __restrict__ out,
    float* __restrict__ token_loss, float* __restrict__ dcand, DistillWs* ws, unsigned int* d_err) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_flag;
  wait_for_predecessor();
  let_successor_start();
  constexpr int kRows = kThreads / kG;              // rows the CTA works on at a time
  const int step_rows = kRows * batches;            // rows of a step, one ring stage
  constexpr int kWarpRows = 32 / kG;                // rows a warp works on at a time
  const int wlane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = wlane / kG, lane = wlane % kG;    // row among the warp's, place in it
  const uint32_t ring_base = (umma::smem_u32(smem_raw) + 127u) & ~127u;
  const uint32_t bars = ring_base + kStages * kStageBytes;
  auto full_bar = [&](int st) { return bars + 8u * st; };
  auto empty_bar = [&](int st) { return bars + 8u * (kStages + st); };
  const float tau = prm.temperature, inv_tau = 1.f / prm.temperature;
  const float w_all = prm.agg_mode == 0 ? (B > 0 ? prm.loss_scale / (float)B : 0.f)
                                        : (T > 0 ? prm.loss_scale / (float)T : 0.f);

  const int steps = (rows + step_rows - 1) / step_rows;
  const int begin = (int)(((int64_t)steps * blockIdx.x) / gridDim.x);
  const int n_mine = (int)(((int64_t)steps * (blockIdx.x + 1)) / gridDim.x) - begin;
  // steps that go through the ring: all but a last one that is not full (its bytes may not be a multiple of 16)
  const int n_ring = !(bulk & 1) ? 0 : (begin + n_mine) * (int64_t)step_rows <= rows ? n_mine : n_mine - 1;
  const bool bulk_out = (bulk & 2) && dcand != nullptr;
  auto issue = [&](int i) {
    const size_t at = (size_t)(begin + i) * step_rows * K;
    const uint32_t bytes = (uint32_t)(step_rows * K) * 4u;
    const uint32_t bar = full_bar(i % kStages), dst = ring_base + (i % kStages) * kStageBytes;
    umma::mbar_arrive_expect_tx(bar, 2 * bytes);
    bulk_load(dst, teacher_logp + at, bytes, bar);
    bulk_load(dst + kStageSlots * 4, cand_logp + at, bytes, bar);
  };
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < kStages; ++s) { umma::mbar_init(full_bar(s), 1); umma::mbar_init(empty_bar(s), kThreads / 32); }
    umma::fence_mbar_init();
    for (int i = 0; i < kStages && i < n_ring; ++i) issue(i);
  }
  if (out)      // as in the policy loss: entries out of order raise the flag, nothing is indexed by them
    for (int q = blockIdx.x * kThreads + threadIdx.x; q < B; q += gridDim.x * kThreads)
      if (__ldg(cu + q) > __ldg(cu + q + 1)) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
  __syncthreads();

  double sum_loss = 0.0, sum_t = 0.0, sum_s = 0.0;
  float part_loss = 0.f, part_t = 0.f, part_s = 0.f;     // of up to kFlush steps
  float w = w_all;
  int seq = -1, seq_beg = 0, seq_end = 0;                // the sequence of the lane's previous row
  bool ok = true;      // false once a wait ran out of time: the warp touches no more data
  const int n_valid = (K - lane * kVec + kG * kVec - 1) / (kG * kVec);    // groups of this lane that lie in the row
  const int warp_row = warp * kWarpRows * batches;       // the warp's first row of a step; its rows are contiguous
  const uint32_t my_slots = ring_base + (uint32_t)((warp_row + sub) * K + lane * kVec) * 4u;
  for (int i = 0; i < n_mine; ++i) {
    const uint32_t stage = (uint32_t)(i % kStages);
    const bool staged = i < n_ring;
    if (bulk_out && i > 0 && i <= n_ring && ok && wlane == 0) {   // what step i - 1 left has gone out
      asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      umma::mbar_arrive(empty_bar((i - 1) % kStages));
    }
    __syncwarp();
    if (!staged) {            // not a whole step, or columns a bulk copy cannot read: the threads bring it over
      __syncthreads();
      const size_t at = (size_t)(begin + i) * step_rows * K;
      const int left = rows - (begin + i) * step_rows, n = (left < step_rows ? left : step_rows) * K;
      float* const to = reinterpret_cast<float*>(smem_raw + (ring_base - umma::smem_u32(smem_raw)) + stage * kStageBytes);
      for (int q = threadIdx.x; q < n; q += kThreads) {
        to[q] = __ldg(teacher_logp + at + q);
        to[kStageSlots + q] = __ldg(cand_logp + at + q);
      }
      __syncthreads();
    } else if (ok) {
      // the stage of step i - 1 is refilled with step i + kStages - 1 once every warp has left it
      if (threadIdx.x == 0 && i >= 1 && i + kStages - 1 < n_ring &&
          umma::mbar_wait(empty_bar((i - 1) % kStages), (uint32_t)((i - 1) / kStages) & 1u, &abort_flag))
        issue(i + kStages - 1);
      ok = __all_sync(0xffffffffu, umma::mbar_wait(full_bar(stage), (uint32_t)(i / kStages) & 1u, &abort_flag));
    }
    if (!ok) continue;
    int row = (begin + i) * step_rows + warp_row + sub;
    float* dst = dcand ? dcand + (size_t)row * K + lane * kVec : nullptr;
    uint32_t at = my_slots + stage * kStageBytes;
    for (int b = 0; b < batches; ++b, row += kWarpRows, at += kWarpRows * K * 4) {
      const bool live = row < rows;                 // a group's lanes agree; all stay for the shuffles
      if (prm.agg_mode == 0 && live) {
        const int t = t0 + row;
        if (t >= seq_end || t < seq_beg) {          // rows come in order: a few sequences on, else a search
          for (int hops = 0; hops < 4 && seq >= 0 && t >= seq_end && seq + 1 < B; ++hops) {
            ++seq;
            seq_beg = seq_end;
            seq_end = __ldg(cu + seq + 1);
          }
          if (seq < 0 || t >= seq_end || t < seq_beg) {
            seq = find_seq(cu, B, t);
            seq_beg = __ldg(cu + seq);
            seq_end = __ldg(cu + seq + 1);
          }
          w = w_all * __frcp_rn((float)(seq_end - seq_beg));
        }
      }
      // slots past the row's end are read too (the stage has room for them) and count as absent
      const int valid = live ? n_valid : 0;
      float lt[kE], lq[kE], g[kE];
#pragma unroll
      for (int e = 0; e < kE / kVec; ++e) {
        load_slots<kVec>(at + e * kG * kVec * 4, lt + e * kVec);
        load_slots<kVec>(at + kStageSlots * 4 + e * kG * kVec * 4, lq + e * kVec);
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const bool present = e / kVec < valid && !(lt[e] <= kAbsentLogp);      // a NaN is present
        lt[e] = present ? lt[e] : kAbsentLogp;
        lq[e] = present ? lq[e] : -INFINITY;
      }
      if (staged && !bulk_out && b == batches - 1) {    // the values are in registers: this warp is done with the stage
        __syncwarp();
        if (wlane == 0) umma::mbar_arrive(empty_bar(stage));
      }
      const float loss = row_divergence<kSupport, kForward, kG, kE>(lt, lq, tau, inv_tau, g, part_t, part_s);
      if (live && lane == 0) {
        part_loss = fmaf(w, loss, part_loss);
        if (token_loss) token_loss[row] = loss;
      }
      if (dst) {
        const float scale = loss == loss ? w : loss;     // a NaN of one slot is in all of the token's gradients
#pragma unroll
        for (int e = 0; e < kE; ++e) g[e] *= scale;
        if (staged && bulk_out) {                   // over the row's own slots, to go out in one piece
#pragma unroll
          for (int e = 0; e < kE / kVec; ++e)
            if (e < valid) store_slots_shared<kVec>(at + e * kG * kVec * 4, g + e * kVec);
        } else {
#pragma unroll
          for (int e = 0; e < kE / kVec; ++e)
            if (e < valid) store_slots<kVec>(dst + e * kG * kVec, g + e * kVec);
          dst += kWarpRows * K;
        }
      }
    }
    if (staged && bulk_out) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (wlane == 0) {
        bulk_store(dcand + ((size_t)(begin + i) * step_rows + warp_row) * K,
                   ring_base + stage * kStageBytes + (uint32_t)(warp_row * K) * 4u, (uint32_t)(kWarpRows * batches * K) * 4u);
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
    }
    if ((i & (kFlush - 1)) == kFlush - 1 || i + 1 == n_mine) {
      sum_loss += (double)part_loss; sum_t += (double)part_t; sum_s += (double)part_s;
      part_loss = 0.f; part_t = 0.f; part_s = 0.f;
    }
  }
  if (bulk_out && wlane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  __syncthreads();
  if (abort_flag) {   // a bulk copy did not arrive in time: flag it, let copies in flight land
    if (threadIdx.x == 0) atomicOr(d_err, umma::kWatchdogBit);
    __nanosleep(1000000);
  }
  if (!out) return;

  __shared__ double s_part[kThreads / 32][kNumSums];
  __shared__ int s_last;
  double v[kNumSums] = {sum_loss, sum_t, sum_s};
  auto block_sum = [&]() {        // thread 0 gets the block's sums, added in a fixed order
#pragma unroll
    for (int q = 0; q < kNumSums; ++q)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v[q] += __shfl_xor_sync(0xffffffffu, v[q], o);
    if (wlane == 0)
      for (int q = 0; q < kNumSums; ++q) s_part[warp][q] = v[q];
    __syncthreads();
    if (threadIdx.x == 0)
      for (int q = 0; q < kNumSums; ++q) {
        v[q] = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) v[q] += s_part[i][q];
      }
  };
  block_sum();
  if (threadIdx.x == 0) {
    for (int q = 0; q < kNumSums; ++q) ws_partial(ws, blockIdx.x)[q] = v[q];
    __threadfence();
    s_last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  for (int q = 0; q < kNumSums; ++q) v[q] = 0.0;
  for (int b = threadIdx.x; b < (int)gridDim.x; b += kThreads)
    for (int q = 0; q < kNumSums; ++q) v[q] += __ldcg(ws_partial(ws, b) + q);
  block_sum();
  if (threadIdx.x == 0) {
    af_distill_out r;
    r.loss = (float)v[0];
    r.teacher_mass = T > 0 ? (float)(v[1] / (double)T) : 0.f;
    r.student_mass = T > 0 ? (float)(v[2] / (double)T) : 0.f;
    r.reserved = 0;
    r.n_tokens = T;
    *out = r;
    if (__ldg(cu) != 0 || __ldg(cu + B) != T) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
    ws->ticket = 0;        // ready for the next call on this stream
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
  int bulk;          // 1: both columns start on 16 bytes, so that whole steps may be copied in bulk; 2: so does dcand
};

template <int kSupport, bool kForward, int kG, int kE, int kVec>
cudaError_t launch_rows(const DistillCall& c, cudaStream_t s) {
  static SmemAttrOnce once;
  const cudaError_t e = set_smem_once(once, distill_loss_kernel<kSupport, kForward, kG, kE, kVec>, kSmemBytes);
  if (e != cudaSuccess) return e;
  constexpr int kRows = kThreads / kG;
  const int64_t most = (int64_t)c.sm_count * kBlocksPerSm;
  // short rows: several batches of rows per step, as many as fill a stage and leave every CTA a step
  int batches = kStageSlots / (kRows * c.K);
  const int64_t share = c.rows / (kRows * most);
  if (batches > share) batches = (int)share;
  if (batches < 1) batches = 1;
  const int64_t steps = ((int64_t)c.rows + kRows * batches - 1) / (kRows * batches);
  const int blocks = (int)(steps < 1 ? 1 : steps < most ? steps : most);
  return launch_overlapped(
      distill_loss_kernel<kSupport, kForward, kG, kE, kVec>, blocks, kThreads, kSmemBytes, s, c.cand_logp, c.teacher_logp, c.cu,
      c.B, c.T, c.t0, c.rows, c.K, batches, c.bulk & (32 / kG * c.K % 4 == 0 ? 3 : 1), c.prm, c.out, c.token_loss, c.dcand, c.ws,
      c.d_err);
}
// Rows that start on 16 bytes (K a multiple of 4) are read four slots at a time, even ones two.
// The fewest slots per lane that hold the row: what a lane has beyond that is computed for nothing.
template <int kSupport, bool kForward, int kG>
cudaError_t launch_group(const DistillCall& c, int vec, cudaStream_t s) {
  if (vec == 4) return c.K <= kG * 12 ? launch_rows<kSupport, kForward, kG, 12, 4>(c, s)
                                      : launch_rows<kSupport, kForward, kG, 16, 4>(c, s);
  if (vec == 2) {
    if (c.K <= kG * 10) return launch_rows<kSupport, kForward, kG, 10, 2>(c, s);
    if (c.K <= kG * 12) return launch_rows<kSupport, kForward, kG, 12, 2>(c, s);
    if (c.K <= kG * 14) return launch_rows<kSupport, kForward, kG, 14, 2>(c, s);
    return launch_rows<kSupport, kForward, kG, 16, 2>(c, s);
  }
  return launch_rows<kSupport, kForward, kG, 16, 1>(c, s);
}
// The smallest group whose lanes hold the row with sixteen slots each; fewer slots for rows shorter than that.
template <int kSupport, bool kForward>
cudaError_t launch_support(const DistillCall& c, int vec, cudaStream_t s) {
  if (c.K == 1) return launch_rows<kSupport, kForward, 1, 1, 1>(c, s);
  if (c.K == 2) return vec >= 2 ? launch_rows<kSupport, kForward, 1, 2, 2>(c, s) : launch_rows<kSupport, kForward, 1, 2, 1>(c, s);
  if (c.K <= 4) return vec == 4 ? launch_rows<kSupport, kForward, 1, 4, 4>(c, s) : launch_rows<kSupport, kForward, 1, 4, 1>(c, s);
  if (c.K <= 8) return vec == 4   ? launch_rows<kSupport, kForward, 1, 8, 4>(c, s)
                       : vec == 2 ? launch_rows<kSupport, kForward, 1, 8, 2>(c, s)
                                  : launch_rows<kSupport, kForward, 1, 8, 1>(c, s);
  if (c.K <= 16) return launch_group<kSupport, kForward, 1>(c, vec, s);
  if (c.K <= 32) return launch_group<kSupport, kForward, 2>(c, vec, s);
  if (c.K <= 64) return launch_group<kSupport, kForward, 4>(c, vec, s);
  if (c.K <= 128) return launch_group<kSupport, kForward, 8>(c, vec, s);
  return launch_group<kSupport, kForward, 16>(c, vec, s);
}

// One translation unit per support (they take a while to compile).
cudaError_t launch_listed(const DistillCall& c, int vec, cudaStream_t s);
cudaError_t launch_renormalised(const DistillCall& c, int vec, cudaStream_t s);
cudaError_t launch_tail(const DistillCall& c, int vec, cudaStream_t s);

}  // namespace distill
}  // namespace af
