// af_preference_loss: paired sequence log ratios -> preference loss and its gradient per token.
//
//   S_j = sum over the tokens of sequence j of (logp - ref);  x_p = beta (n_c S_c - n_r S_r) - margin;
//   l_p = f(x_p) + nll_coef * mean(-logp over the chosen);    dlogp is constant over a sequence.
//
// 8 (or 4, without reference) bytes read and 4 written per token: HBM-bound, in two passes with the pairs in
// between, since a token's gradient needs its pair's sums.  One cooperative launch does all three, with a
// grid barrier after the first and the second phase:
//   1. sums    a warp walks a range in steps of 512 tokens, eight per lane at a time, each lane adding up its tokens of the
//              current sequence and the warp joining them when the sequence or the range ends.  The next steps come
//              by bulk copies into a ring of the warp's own, so nothing waits on another warp.  A sequence inside one
//              range is done; one that crosses ranges leaves a piece in each, at most one coming in (head) and one
//              going out (tail), so pieces need no counters and no atomics.  Where
//              several sequences end inside a slice, running sums that start anew at every border are taken over it, and a
//              lane per sequence reads the one at its end: the cost is that of a few reductions however many end.
//   2. pairs   a few lanes per pair add the pieces, evaluate the loss and write the two sequences' coefficients.
//   3. fill    the same ranges again: the coefficient of each token's sequence.
// Measured: 24576 pairs of 1024 tokens on average without a reference 94-96 us (403 MB: 4.3 TB/s, of which the read pass 4.5,
// held by the conversions to fp64, the fill 6, half of which L2 takes, and about 3 us for each barrier); 64 pairs of 2161 tokens
// 14 us in a graph, 16 called one by one; 49152 sequences of 64 tokens 33-37 us (106 with one warp reduction per sequence).
// Three launches in place of one took 173 and 24 us.
// All sums are fp64 (thousands of near-cancelling terms, and the card has the rate: two additions per token)
// and taken in a fixed order, so results are bit-reproducible.
#include "common.cuh"
#include "device_util.cuh"
#include "umma.cuh"

#include <climits>

namespace af {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBlocksPerSm = 3;
constexpr int kSlice = 256;                 // tokens a warp works on at a time: two groups of 4 per lane, 128 apart
constexpr int kStep = 2 * kSlice;           // tokens of a stage of its ring
constexpr int kStages = 2;
constexpr int kStageBytes = 2 * kStep * 4;  // logp | ref
constexpr int kSmemBytes = kWarps * kStages * kStageBytes + 128 /*alignment*/ + kWarps * kStages * 8 /*barriers*/;
constexpr int kNumSums = 6;                 // loss, pair loss, nll, accuracy, chosen score, rejected score
constexpr int kMaxBlocks = 1024;

struct PrefHeader {                         // in the context's device block; zero between calls
  unsigned int arrived;                     // blocks at the grid barriers (counts up through both)
  unsigned int left;                        // blocks that are done
  unsigned int failed;                      // a barrier's wait ran out
  unsigned int pad[13];
};
struct PrefWs {                             // device views into the workspace, and the header
  PrefHeader* header;
  double2* seq;                             // [B] sums of the sequences that lie inside one range: S, sum of logp
  double2* head;                            // [workers] piece of the sequence that comes into the range
  double2* tail;                            // [workers] piece of the sequence that starts in it and goes on
  double* partial;                          // [blocks][kNumSums]
  float* coef;                              // [B] dloss/dlogp of a sequence's tokens
};

int64_t steps_of(int64_t T) { return (T + kStep - 1) / kStep; }

PrefWs carve(void* ws, void* header, int32_t B) {
  PrefWs w;
  w.header = static_cast<PrefHeader*>(header);
  w.head = static_cast<double2*>(ws);
  w.tail = w.head + kMaxBlocks * kWarps;
  w.seq = w.tail + kMaxBlocks * kWarps;
  w.partial = reinterpret_cast<double*>(w.seq + B);
  w.coef = reinterpret_cast<float*>(w.partial + (size_t)kMaxBlocks * kNumSums);
  return w;
}

// Token of slot i (0..7) of a lane: group i / 4 starts 128 tokens after the first.
__device__ __forceinline__ int slot_token(int base, int lane, int i) { return base + (i >> 2) * 128 + lane * 4 + (i & 3); }

__device__ __forceinline__ void bulk_load(uint32_t dst_smem, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               :: "r"(dst_smem), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float4 lds128(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

// The lane's eight values of a column of a slice staged at `stage`; zeros past the end.  A group of four that no bulk
// copy brought (the last, not full one, or any of a column that does not start on 16 bytes) is read directly.
__device__ __forceinline__ void load_slice(const float* __restrict__ p, uint32_t stage, int base, int lane, int T,
                                           bool staged, float (&v)[8]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int t = slot_token(base, lane, 4 * q);
    if (staged && t + 4 <= T) {
      const float4 x = lds128(stage + (uint32_t)(q * 128 + lane * 4) * 4u);
      v[4 * q] = x.x; v[4 * q + 1] = x.y; v[4 * q + 2] = x.z; v[4 * q + 3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * q + i] = t + i < T ? __ldg(p + t + i) : 0.f;
    }
  }
}

// A warp's place in the list of sequences, with the border (and coefficient) of the one after already on its way.
// Uniform over the warp.
struct Place {
  const int32_t* __restrict__ cu;
  const float* coef;                // null in the first phase
  int B;
  int j, beg, end, next_end;
  float c, next_c;
  __device__ __forceinline__ void ahead() {
    next_end = j + 2 <= B ? __ldg(cu + j + 2) : INT_MAX;
    if (coef) next_c = j + 1 < B ? __ldcg(coef + j + 1) : 0.f;
  }
  __device__ __forceinline__ void set(int i) {                       // i in [0, B)
    j = i;
    beg = __ldg(cu + j);
    end = __ldg(cu + j + 1);
    if (coef) c = __ldcg(coef + j);
    ahead();
  }
  // Whether one sequence ends in (base, last], this one.
  __device__ __forceinline__ bool one_border(int base, int last) const { return end > base && end <= last && next_end > last; }
  __device__ __forceinline__ void advance() {
    if (j + 1 >= B) return;
    ++j;
    beg = end;
    end = next_end;
    if (coef) c = next_c;
    ahead();
  }
};

// Marks in bits (8 words of the warp's) where sequences start in (base, last), from the one after j on; start(i, p) is
// called by one lane for each such sequence that is not empty, p its place in the slice.  Returns how many sequences
// from j on end at or before last.
template <class Start>
__device__ __forceinline__ int mark_starts(const int32_t* __restrict__ cu, int B, int j, int base, int last,
                                           uint32_t* bits, int lane, Start start) {
  if (lane < kSlice / 32) bits[lane] = 0u;
  __syncwarp();
  int ended = 0;
  for (;;) {
    const int i = j + ended + lane + 1;
    const int beg = i <= B ? __ldg(cu + i) : INT_MAX;
    if (beg > base && beg < last) {
      const int end = i < B ? __ldg(cu + i + 1) : beg;
      atomicOr(bits + ((beg - base) >> 5), 1u << ((beg - base) & 31));
      if (end > beg) start(i, beg - base);
    }
    const unsigned on = __ballot_sync(0xffffffffu, beg > last);
    ended += on ? __ffs(on) - 1 : 32;
    if (on) break;                                 // at the latest behind cu[B]
  }
  __syncwarp();
  return ended;
}
// The lane's four marks of group q.
__device__ __forceinline__ unsigned marks_of(const uint32_t* bits, int q, int lane) {
  return (bits[q * 4 + (lane >> 3)] >> ((lane & 7) * 4)) & 15u;
}

// Running sums of a slice's values in token order, each from the last mark on; `sum` is what came in and what goes on.
// A sum takes its own sequence's values only, so that an infinity or a NaN stays with its sequence.
__device__ __forceinline__ void running_sums(const double (&v)[8], const unsigned (&marks)[2], int lane, double& sum,
                                             double (&at)[8]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    double own = lane == 0 ? sum : 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      own = marks[q] >> i & 1u ? v[4 * q + i] : own + v[4 * q + i];
      at[4 * q + i] = own;
    }
    const unsigned before = __ballot_sync(0xffffffffu, marks[q] != 0u) & (0xffffffffu >> (31 - lane));
    const int back = before ? lane - (31 - __clz(before)) : lane;       // lanes since the last one with a mark
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double x = __shfl_up_sync(0xffffffffu, own, o);
      if (o <= back) own += x;
    }
    const double in = __shfl_up_sync(0xffffffffu, own, 1);
    const int stop = marks[q] ? __ffs(marks[q]) - 1 : 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (lane > 0 && i < stop) at[4 * q + i] += in;
    sum = __shfl_sync(0xffffffffu, own, 31);
  }
}

__device__ __forceinline__ void warp_sums(double& s, double& l, bool both) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    l += __shfl_xor_sync(0xffffffffu, l, o);
    if (both) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
}

// Phase 1 over the steps [s0, s1) of worker `me`.  ring: the warp's stages, bars: their barriers.
__device__ __forceinline__ void sum_steps(const float* __restrict__ logp, const float* __restrict__ ref,
                                          const int32_t* __restrict__ cu, int B, int T, const PrefWs& ws, bool bulk,
                                          int me, int s0, int s1, uint32_t ring, uint32_t bars, uint32_t* bits,
                                          int lane, volatile int* abort_flag) {
  if (s0 >= s1) return;
  const bool both = ref != nullptr;
  auto issue = [&](int it) {                       // lane 0; a step is copied up to its last whole group of 4 tokens
    const int base = (s0 + it) * kStep, left = T - base < kStep ? T - base : kStep;
    const uint32_t bytes = bulk ? (uint32_t)(left & ~3) * 4u : 0u;
    const uint32_t bar = bars + 8u * (it % kStages), dst = ring + (uint32_t)(it % kStages) * kStageBytes;
    umma::mbar_arrive_expect_tx(bar, both ? 2 * bytes : bytes);
    if (bytes > 0) {
      bulk_load(dst, logp + base, bytes, bar);
      if (both) bulk_load(dst + kStep * 4, ref + base, bytes, bar);
    }
  };
  if (lane == 0)
    for (int it = 0; it < kStages && s0 + it < s1; ++it) issue(it);
  const int range_beg = s0 * kStep;
  Place at{cu, nullptr, B};
  at.set(find_seq_warp(cu, B, range_beg, lane));
  double s = 0.0, l = 0.0;                         // the lane's share of the current sequence
  int last = range_beg;
  for (int step = s0; step < s1; ++step) {
    const int it = step - s0;
    const uint32_t stage = ring + (uint32_t)(it % kStages) * kStageBytes;
    if (!__all_sync(0xffffffffu, umma::mbar_wait(bars + 8u * (it % kStages), (uint32_t)(it / kStages) & 1u, abort_flag)))
      return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int base = step * kStep + half * kSlice;
      if (half > 0 && base >= T) break;
      float lp[8], rf[8];
      if (bulk && base + kSlice <= T) {            // as the others, without a question per lane
        const uint32_t from = stage + (uint32_t)(half * kSlice + lane * 4) * 4u;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float4 x = lds128(from + q * 512);
          lp[4 * q] = x.x; lp[4 * q + 1] = x.y; lp[4 * q + 2] = x.z; lp[4 * q + 3] = x.w;
          if (both) {
            const float4 y = lds128(from + kStep * 4 + q * 512);
            rf[4 * q] = y.x; rf[4 * q + 1] = y.y; rf[4 * q + 2] = y.z; rf[4 * q + 3] = y.w;
          }
        }
        last = base + kSlice;
      } else {
        const uint32_t from = stage + (uint32_t)(half * kSlice) * 4u;
        load_slice(logp, from, base, lane, T, bulk, lp);
        if (both) load_slice(ref, from + kStep * 4, base, lane, T, bulk, rf);
        last = T - base < kSlice ? T : base + kSlice;
      }
      if (half == 1 || last == T) {
        __syncwarp();                              // every lane has its values: the stage may be filled again
        if (lane == 0 && step + kStages < s1) issue(it + kStages);
      }
      auto add_all = [&]() {                       // the whole slice (past the end the values are zero)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          l += (double)lp[i];
          if (both) s += (double)lp[i] - (double)rf[i];
        }
      };
      if (at.beg <= base && at.end > last) {       // most often: one sequence from before this slice to behind it
        add_all();
        continue;
      }
      if (at.one_border(base, last)) {             // long sequences: one ends in here
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (slot_token(base, lane, i) < at.end) {
            l += (double)lp[i];
            if (both) s += (double)lp[i] - (double)rf[i];
            lp[i] = 0.f;
            if (both) rf[i] = 0.f;
          }
        }
        warp_sums(s, l, both);
        if (lane == 0) *(at.beg >= range_beg ? ws.seq + at.j : ws.head + me) = make_double2(both ? s : l, l);
        s = 0.0;
        l = 0.0;
        at.advance();
        add_all();                                 // the rest belongs to the next one
        continue;
      }
      // several: running sums over the slice, and a lane per sequence reads the one at its end
      const int ended = mark_starts(cu, B, at.j, base, last, bits, lane, [](int, int) {});
      const unsigned marks[2] = {marks_of(bits, 0, lane), marks_of(bits, 1, lane)};
      warp_sums(s, l, both);                       // of the first one, from earlier slices
#pragma unroll 1
      for (int column = both ? 0 : 1; column < 2; ++column) {
        double v[8], run[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = column == 0 ? (double)lp[i] - (double)rf[i] : (double)lp[i];
        double sum = column == 0 ? s : l;
        running_sums(v, marks, lane, sum, run);
        for (int done = 0; done < ended; done += 32) {
          const int i = at.j + done + lane;        // below B where it counts
          const bool mine = done + lane < ended;
          const int beg = mine ? __ldg(cu + i) : 0, end = mine ? __ldg(cu + i + 1) : 0;
          const int x = (end - 1 - base) & (kSlice - 1), slot = (x >> 7) * 4 + (x & 3);
          double r = 0.0;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const double y = __shfl_sync(0xffffffffu, run[k], (x & 127) >> 2);
            if (slot == k) r = y;
          }
          if (mine && end > beg) {
            double2* const to = beg < range_beg ? ws.head + me : ws.seq + i;
            if (column == 0) to->x = r; else to->y = r;
            if (!both) to->x = r;
          }
        }
        if (column == 0) s = sum; else l = sum;
      }
      at.set(at.j + ended < B ? at.j + ended : B - 1);
      if (lane > 0 || at.beg >= last) { s = 0.0; l = 0.0; }             // else the sum so far of what goes on
    }
  }
  if (at.beg < last && at.end > last) {
    warp_sums(s, l, both);
    if (lane == 0) (at.beg >= range_beg ? ws.tail : ws.head)[me] = make_double2(both ? s : l, l);
  }
}

// Phase 3 over the steps [s0, s1).
__device__ __forceinline__ void fill_steps(const int32_t* __restrict__ cu, int B, int T, const PrefWs& ws, float* dlogp,
                                           bool vec, int s0, int s1, uint32_t* bits, float* coefs, int lane) {
  if (s0 >= s1) return;
  Place at{cu, ws.coef, B};
  at.set(find_seq_warp(cu, B, s0 * kStep, lane));
  const int end = s1 * (int64_t)kStep < T ? s1 * kStep : T;
  for (int base = s0 * kStep; base < end; base += kSlice) {
    const int last = T - base < kSlice ? T : base + kSlice;
    float* const out = dlogp + slot_token(base, lane, 0);
    if (vec && at.beg <= base && at.end > last && base + kSlice <= T) {
      const float4 v = make_float4(at.c, at.c, at.c, at.c);
      __stcs(reinterpret_cast<float4*>(out), v);
      __stcs(reinterpret_cast<float4*>(out + 128), v);
      continue;
    }
    if (at.one_border(base, last)) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int t = slot_token(base, lane, 4 * q);
        float g[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = t + i < at.end ? at.c : at.next_c;
        if (vec && t + 4 <= T) {
          __stcs(reinterpret_cast<float4*>(out + q * 128), make_float4(g[0], g[1], g[2], g[3]));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) if (t + i < T) dlogp[t + i] = g[i];
        }
      }
      at.advance();
      continue;
    }
    // coefficients at the places where sequences start; a token's is the one at the last start before it
    const int ended = mark_starts(cu, B, at.j, base, last, bits, lane,
                                  [&](int i, int p) { coefs[p] = __ldcg(ws.coef + i); });
    int came_in = -1;                              // the last start in earlier groups
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int t = slot_token(base, lane, 4 * q);
      const unsigned marks = marks_of(bits, q, lane);
      const unsigned with = __ballot_sync(0xffffffffu, marks != 0u), before = with & ((1u << lane) - 1u);
      const int newest = t - base + 31 - __clz(marks | 1u);             // counts where marks is not 0
      const int left = __shfl_sync(0xffffffffu, newest, before ? 31 - __clz(before) : lane);
      const int from = before ? left : came_in;
      const int final = __shfl_sync(0xffffffffu, newest, with ? 31 - __clz(with) : 0);
      float c = from >= 0 ? coefs[from] : at.c, g[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (marks >> i & 1u) c = coefs[t - base + i];
        g[i] = c;
      }
      if (with) came_in = final;
      if (vec && t + 4 <= T) {
        __stcs(reinterpret_cast<float4*>(out + q * 128), make_float4(g[0], g[1], g[2], g[3]));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (t + i < T) dlogp[t + i] = g[i];
      }
    }
    __syncwarp();                                  // coefs and bits are read
    at.set(at.j + ended < B ? at.j + ended : B - 1);
  }
}

// Sums of one sequence, by kLanes lanes together (all get the result; every lane of the warp takes part).
// beg and end lie in [0, T]; a range is `per` steps.
template <int kLanes>
__device__ __forceinline__ double2 sequence_sum(const PrefWs& ws, int j, int beg, int end, int per, int lane) {
  double s = 0.0, l = 0.0;
  if (end > beg) {
    const int first = beg / kStep / per, final = (end - 1) / kStep / per;
    if (first == final) {
      if (lane == 0) { const double2 v = __ldcg(ws.seq + j); s = v.x; l = v.y; }
    } else {
      for (int i = first + lane; i <= final; i += kLanes) {
        const double2 v = __ldcg((i == first ? ws.tail : ws.head) + i);
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

// Phase 2: pairs p0, p0 + step, ... of this block; `sum` gains the block's share of the record.
template <int kLanes>
__device__ __forceinline__ void pair_terms(const int32_t* __restrict__ cu, int B, int T, const af_preference_params& prm,
                                           const PrefWs& ws, int per, float* __restrict__ pair_loss,
                                           float* __restrict__ seq_score, double (&sum)[kNumSums]) {
  constexpr int kPairs = kThreads / kLanes;
  const int P = B / 2;
  const int lane = threadIdx.x % kLanes;
  const double beta = (double)prm.beta, w = P > 0 ? (double)prm.loss_scale / (double)P : 0.0;
  for (int p0 = blockIdx.x * kPairs; p0 < P; p0 += gridDim.x * kPairs) {
    const int p = p0 + threadIdx.x / kLanes;
    const bool live = p < P;
    const int c = !live ? 0 : prm.pair_layout ? p : 2 * p, r = !live ? 0 : prm.pair_layout ? P + p : 2 * p + 1;
    // clamped: a cu_seqlens out of order is flagged, but must not index anything
    const int cb = min(max(__ldg(cu + c), 0), T), ce = min(max(__ldg(cu + c + 1), 0), T);
    const int rb = min(max(__ldg(cu + r), 0), T), re = min(max(__ldg(cu + r + 1), 0), T);
    const double2 sc = sequence_sum<kLanes>(ws, c, cb, live ? ce : cb, per, lane);
    const double2 sr = sequence_sum<kLanes>(ws, r, rb, live ? re : rb, per, lane);
    if (!live || lane != 0) continue;
    const double per_c = 1.0 / (double)(ce > cb ? ce - cb : 1), per_r = 1.0 / (double)(re > rb ? re - rb : 1);
    const double n_c = prm.length_norm ? per_c : 1.0, n_r = prm.length_norm ? per_r : 1.0;
    const double score_c = beta * sc.x * n_c, score_r = beta * sr.x * n_r;
    const double x = score_c - score_r - (double)prm.margin;
    double l, slope;
    if (prm.kind == 0) {
      const double eps = (double)prm.label_smoothing;
      l = log1p(exp(-fabs(x))) + (x < 0.0 ? (eps - 1.0) * x : eps > 0.0 ? eps * x : 0.0);     // no two infinities meet
      slope = eps - 1.0 / (1.0 + exp(x));
    } else if (prm.kind == 1) {
      const double y = (x - 0.5) / beta;
      l = y * y;
      slope = 2.0 * y / beta;
    } else {
      l = x < 1.0 ? 1.0 - x : x >= 1.0 ? 0.0 : x;        // a NaN stays one, here and in the gradient
      slope = x < 1.0 ? -1.0 : x >= 1.0 ? 0.0 : x;
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
}

// All blocks of the launch meet (a cooperative launch: they are all resident).  `target`: blocks times barriers so
// far.  False if the wait ran out of time here or elsewhere: the caller goes on to its end, touching nothing more.
__device__ __forceinline__ bool grid_barrier(PrefHeader* h, unsigned int target) {
  __shared__ int s_ok;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    atomicAdd(&h->arrived, 1u);
    const unsigned long long t0 = umma::globaltimer_ns();
    int ok = 1;
    for (unsigned int spins = 0;; ++spins) {
      unsigned int seen;
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&h->arrived) : "memory");
      if (seen >= target) break;
      if ((spins & 63u) == 63u) {
        unsigned int failed;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(failed) : "l"(&h->failed) : "memory");
        if (failed || umma::globaltimer_ns() - t0 > umma::kWaitLimitNs) { atomicExch(&h->failed, 1u); ok = 0; break; }
      }
    }
    __threadfence();
    s_ok = ok;
  }
  __syncthreads();
  return s_ok != 0;
}

__global__ void __launch_bounds__(kThreads, kBlocksPerSm) preference_kernel(
    const float* __restrict__ logp, const float* __restrict__ ref, const int32_t* __restrict__ cu, int B, int T,
    const af_preference_params prm, const PrefWs ws, af_preference_out* __restrict__ out, float* __restrict__ pair_loss,
    float* __restrict__ seq_score, float* __restrict__ dlogp, int vec, int wide_pairs, unsigned int* d_err) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_flag;
  __shared__ uint32_t bits[kWarps][kSlice / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int P = B / 2;
  const uint32_t smem = (umma::smem_u32(smem_raw) + 127u) & ~127u;
  const uint32_t ring = smem + (uint32_t)(warp * kStages) * kStageBytes;
  const uint32_t bars = smem + kWarps * kStages * kStageBytes + (uint32_t)(warp * kStages) * 8u;
  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) {
    for (int q = 0; q < kStages; ++q) umma::mbar_init(bars + 8u * q, 1);
    umma::fence_mbar_init();
  }
  __syncthreads();
  const int steps = (int)(((int64_t)T + kStep - 1) / kStep);
  const int workers = gridDim.x * kWarps, me = blockIdx.x * kWarps + warp;
  const int per = steps > workers ? (steps + workers - 1) / workers : 1;       // steps of a range
  const int s0 = (int64_t)me * per < steps ? me * per : steps, s1 = steps - s0 < per ? steps : s0 + per;

  sum_steps(logp, ref, cu, B, T, ws, vec & 1, me, s0, s1, ring, bars, bits[warp], lane, &abort_flag);
  for (int q = blockIdx.x * kThreads + threadIdx.x; q < B; q += gridDim.x * kThreads)
    if (__ldg(cu + q) > __ldg(cu + q + 1)) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
  bool ok = grid_barrier(ws.header, gridDim.x);
  double sum[kNumSums] = {};
  if (ok) {
    if (wide_pairs) pair_terms<32>(cu, B, T, prm, ws, per, pair_loss, seq_score, sum);
    else pair_terms<4>(cu, B, T, prm, ws, per, pair_loss, seq_score, sum);
  }
  __shared__ double s_part[kWarps][kNumSums];
  __syncwarp();
#pragma unroll
  for (int q = 0; q < kNumSums; ++q)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], o);
  if (lane == 0)
    for (int q = 0; q < kNumSums; ++q) s_part[warp][q] = sum[q];
  __syncthreads();
  if (threadIdx.x < kNumSums) {
    double t = 0.0;
    for (int i = 0; i < kWarps; ++i) t += s_part[i][threadIdx.x];
    ws.partial[(size_t)blockIdx.x * kNumSums + threadIdx.x] = t;
  }
  ok = grid_barrier(ws.header, 2 * gridDim.x) && ok;
  if (ok && dlogp) fill_steps(cu, B, T, ws, dlogp, (vec & 2) != 0, s0, s1, bits[warp],
                               reinterpret_cast<float*>(smem_raw + (ring - umma::smem_u32(smem_raw))), lane);
  if (ok && blockIdx.x == 0 && warp < kNumSums) {      // the record: a warp per sum, the blocks in a fixed order
    double t = 0.0;
    for (int b = lane; b < (int)gridDim.x; b += 32) t += __ldcg(ws.partial + (size_t)b * kNumSums + warp);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (lane == 0) {
      const double inv = P > 0 ? 1.0 / (double)P : 0.0;
      reinterpret_cast<float*>(out)[warp] = (float)(warp == 0 ? inv * (double)prm.loss_scale * t : inv * t);
      if (warp == 0) {
        out->n_pairs = P;
        if (__ldg(cu) != 0 || __ldg(cu + B) != T) atomicOr(d_err, AF_DEVERR_CU_SEQLENS);
      }
    }
  }
  __syncthreads();
  if (abort_flag) {          // a bulk copy did not arrive in time: let copies in flight land
    if (threadIdx.x == 0) atomicExch(&ws.header->failed, 1u);
    __nanosleep(1000000);
  }
  if (threadIdx.x == 0 && atomicAdd(&ws.header->left, 1u) == gridDim.x - 1) {   // every block is past both barriers
    if (ws.header->failed) atomicOr(d_err, umma::kWatchdogBit);
    ws.header->arrived = 0; ws.header->failed = 0; ws.header->left = 0;
    __threadfence();
  }
}

}  // namespace

size_t preference_workspace_bytes(int32_t B) {
  return (size_t)kMaxBlocks * (kNumSums * sizeof(double) + 2 * kWarps * sizeof(double2)) +
         (size_t)B * (sizeof(double2) + sizeof(float));
}
static_assert(sizeof(PrefHeader) == 64 && kPrefHeaderByte % 128 == 0 && kPrefHeaderByte + 128 <= kDieTableByte,
              "the header has a line of the device block to itself");

cudaError_t launch_preference_loss(const float* logp, const float* ref_logp, const int32_t* cu, int32_t B, int64_t T,
                                   const af_preference_params& p, af_preference_out* out, float* pair_loss,
                                   float* seq_score, float* dlogp, void* ws_mem, void* header, unsigned int* d_err,
                                   int sm_count, cudaStream_t s) {
  auto al = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  PrefWs ws = carve(ws_mem, header, B);
  static SmemAttrOnce once;
  const cudaError_t e = set_smem_once(once, preference_kernel, kSmemBytes);
  if (e != cudaSuccess) return e;
  // four lanes per pair while sequences have few pieces, a warp for long ones (a range is 512 tokens at least)
  int wide = B > 0 && T / B > 2048 ? 1 : 0;
  const int64_t by_steps = (steps_of(T) + kWarps - 1) / kWarps;
  const int64_t by_pairs = ((int64_t)B / 2 * (wide ? 32 : 4) + kThreads - 1) / kThreads;
  const int64_t want = by_steps > by_pairs ? by_steps : by_pairs;
  const int64_t most = (int64_t)sm_count * kBlocksPerSm < kMaxBlocks ? (int64_t)sm_count * kBlocksPerSm : kMaxBlocks;
  const int blocks = (int)(want < 1 ? 1 : want < most ? want : most);
  int vec = (al(logp) && al(ref_logp) ? 1 : 0) | (al(dlogp) ? 2 : 0);
  int Bi = B, Ti = (int)T;
  af_preference_params prm = p;
  void* args[] = {&logp, &ref_logp, &cu, &Bi, &Ti, &prm, &ws, &out, &pair_loss, &seq_score, &dlogp, &vec, &wide, &d_err};
  return cudaLaunchCooperativeKernel(reinterpret_cast<const void*>(preference_kernel), dim3(blocks), dim3(kThreads), args,
                                     kSmemBytes, s);
}

}  // namespace af
