// af_draft_verify: drafted tokens against the target's distribution, from given uniforms.
//
// Two launches.  The first reads rows of logits once, in slices, for their maxima and sums of exponentials (fp32: a stream at
// the memory's rate, next to which the exponentials fit).  It goes through the batch by positions, first drafts first, and a
// row of a request that has already been seen to stop is not read.  Whoever finishes a row decides whether its draft passes.
// The second, a cluster per request, finds the first that does not and draws the token after those before it.
//
// What has to be exact is whole numbers: a comparison u q < p, and the place of u C among running sums C_v of up to
// 10^5 terms, where fp32 would be off by as much as many terms are large.  So a comparison whose sides are within 1e-5 is
// made again from sums in 64 bits, and a draw's sums are in 64 bits throughout: per logit ten 64-bit operations, 2^x from a table
// of 64 powers and a polynomial of degree 4 (2^-44 relative), which are what the second launch is bound by.
#include <cooperative_groups.h>

#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowBlocks = 4;                      // rows, or slices, on an SM at a time: few, so that positions end in order
constexpr int kDrawThreads = 512;
constexpr int kDrawWarps = kDrawThreads / 32;
constexpr int kMostCluster = 16;                   // CTAs that draw for one request
constexpr float kNoMax = -INFINITY;
constexpr double kResidualFloor = 0x1p-30;         // a residual with less mass than this is drawn from the target itself
constexpr int kGoesOn = 0x7fffffff;

struct RowPart {                                   // a slice of a row: max z, sum exp((z - m) / tau), place of the maximum
  float m, s;
  int32_t at, pad;
};
struct Row {                                       // of a whole row: maximum, its place, sum about the maximum in 64 bits
  float m;
  int32_t at;
  double s;
};
enum Verdict : int32_t { kPasses, kFails, kTooNear, kNoRow };       // too near to tell in 32 bits; target or draft is no distribution
// Places are by unit, position * R + request: each request has its own, whatever cu_draft says.
struct Workspace {
  RowPart* target;                                 // [units][slices]
  RowPart* draft;                                  // [units][slices]
  Row* target_row;                                 // [units]
  Row* draft_row;                                  // [units]
  int32_t* verdict;                                // [units]
  unsigned int* ticket;                            // [units] slices done, zero between calls
  int* stop;                                       // [R] first draft that is known not to pass, kGoesOn between calls
};
struct Shape {
  int slices, positions;                           // slices of a row; max_draft + 1
};

__device__ __forceinline__ float load(const LogitRows& x, int64_t row, int v) {
  const int64_t i = row * x.pitch + v;
  return x.type == AF_F32 ? __ldg(static_cast<const float*>(x.p) + i)
                          : __bfloat162float(static_cast<const __nv_bfloat16*>(x.p)[i]);
}

// Drafts of request r: rows [first, first + n) of the drafts, [first + r, first + r + n] of the target.
struct Span { int first, n; bool ok; };
__device__ __forceinline__ Span span_of(const VerifyCall& c, int r) {
  const int a = __ldg(c.cu + r), b = __ldg(c.cu + r + 1);
  const bool ok = a >= 0 && a <= b && b <= c.D && b - a <= c.max_draft;
  return {ok ? a : 0, ok ? b - a : 0, ok};
}

// ------------------------------------------------------------------------------------ rows, in fp32
__device__ __forceinline__ RowPart join(const RowPart& a, const RowPart& b, float scale) {
  RowPart o;
  const bool first = a.m > b.m || (a.m == b.m && a.at < b.at);
  o.m = first ? a.m : b.m;
  o.at = first ? a.at : b.at;
  // a part without mass adds nothing (its maximum may be -inf); a NaN stays
  o.s = (a.s == 0.f ? 0.f : a.s * ex2f((a.m - o.m) * scale)) + (b.s == 0.f ? 0.f : b.s * ex2f((b.m - o.m) * scale));
  o.pad = 0;
  return o;
}

template <int n>
struct Values { float v[n]; };
__device__ __forceinline__ Values<4> widen(const float*, uint4 x) {
  return {{__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w)}};
}
__device__ __forceinline__ Values<8> widen(const __nv_bfloat16*, uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  Values<8> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) { o.v[2 * i] = __uint_as_float(w[i] << 16); o.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  return o;
}
__device__ __forceinline__ Values<1> widen1(const float* p) { return {{__ldg(p)}}; }
__device__ __forceinline__ Values<1> widen1(const __nv_bfloat16* p) { return {{__bfloat162float(*p)}}; }

// Adds n neighbours, the first at place `at`, to a thread's part.
template <bool kPlace, int n>
__device__ __forceinline__ void add(RowPart& a, const Values<n>& x, int at, float scale) {
  float top = x.v[0];
#pragma unroll
  for (int i = 1; i < n; ++i) top = fmaxf(top, x.v[i]);
  if (top > a.m) {                                 // rare after the first few
    a.s *= ex2f((a.m - top) * scale);              // 0 times 0 at first
    a.m = top;
    if constexpr (kPlace) {
#pragma unroll
      for (int i = n - 1; i >= 0; --i)
        if (x.v[i] == top) a.at = at + i;
    }
  }
  if (a.m == kNoMax) {                             // nothing but -inf so far, or a NaN
#pragma unroll
    for (int i = 0; i < n; ++i)
      if (x.v[i] != x.v[i]) a.s = x.v[i];
    return;
  }
  // a NaN, and infinity less itself, make the sum NaN
  if constexpr (n == 1) {
    a.s += ex2f((x.v[0] - a.m) * scale);
  } else {
    const float2 less = make_float2(-a.m, -a.m), by = make_float2(scale, scale);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < n; i += 2) {
      const float2 e = __fmul2_rn(__fadd2_rn(make_float2(x.v[i], x.v[i + 1]), less), by);
      sum = __fadd2_rn(sum, make_float2(ex2f(e.x), ex2f(e.y)));
    }
    a.s += sum.x + sum.y;
  }
}

template <bool kPlace, class T>
__device__ RowPart row_part(const T* row, int lo, int hi, float scale) {
  constexpr int kVec = 16 / sizeof(T), kLoads = 4;
  RowPart a{kNoMax, 0.f, kGoesOn, 0};
  // single elements up to a multiple of 16 bytes, and behind the last one
  const int to_line = (int)((16u - ((uint32_t)reinterpret_cast<uintptr_t>(row + lo) & 15u)) & 15u) / (int)sizeof(T);
  const int body = min(hi, lo + to_line), vecs = (hi - body) / kVec, tail = body + vecs * kVec;
  if (lo + (int)threadIdx.x < body) add<kPlace>(a, widen1(row + lo + threadIdx.x), lo + threadIdx.x, scale);
  const uint4* const at = reinterpret_cast<const uint4*>(row + body);
  // the next loads are under way while the last ones' exponentials are taken
  constexpr int kStep = kLoads * kRowThreads;
  uint4 w[kLoads], ahead[kLoads];
  auto fetch = [&](uint4 (&to)[kLoads], int i) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) to[k] = __ldg(at + i + k * kRowThreads);
  };
  int i = threadIdx.x;
  const int whole = vecs / kStep * kStep;          // the same number of whole steps for every thread
  if (whole > 0) fetch(w, i);
  for (; i < whole; i += kStep) {
    if (i + kStep < whole) fetch(ahead, i + kStep);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) add<kPlace>(a, widen(row, w[k]), body + (i + k * kRowThreads) * kVec, scale);
#pragma unroll
    for (int k = 0; k < kLoads; ++k) w[k] = ahead[k];
  }
  for (; i < vecs; i += kRowThreads) add<kPlace>(a, widen(row, __ldg(at + i)), body + i * kVec, scale);
  if (tail + (int)threadIdx.x < hi) add<kPlace>(a, widen1(row + tail + threadIdx.x), tail + threadIdx.x, scale);
  return a;
}

template <bool kPlace>
__device__ RowPart thread_part(const LogitRows& x, int64_t row, int lo, int hi, float scale) {
  return x.type == AF_F32 ? row_part<kPlace>(static_cast<const float*>(x.p) + row * x.pitch, lo, hi, scale)
                          : row_part<kPlace>(static_cast<const __nv_bfloat16*>(x.p) + row * x.pitch, lo, hi, scale);
}
__device__ __forceinline__ void join_warp(RowPart& a, float scale) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    RowPart b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
    b.at = __shfl_xor_sync(0xffffffffu, a.at, o);
    a = join(a, b, scale);
  }
}

__device__ __forceinline__ bool good(const Row& x) { return fabsf(x.m) < INFINITY && x.s > 0.0 && x.s < 1e300; }
// Called by a whole warp.
__device__ Row warp_row(const RowPart* parts, int slices, double inv_tau) {
  const int lane = threadIdx.x & 31;
  Row x{kNoMax, kGoesOn, 0.0};
  for (int i = lane; i < slices; i += 32) {
    const float m = __ldcg(&parts[i].m);
    const int32_t at = __ldcg(&parts[i].at);
    if (m > x.m || (m == x.m && at < x.at)) { x.m = m; x.at = at; }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m = __shfl_xor_sync(0xffffffffu, x.m, o);
    const int32_t at = __shfl_xor_sync(0xffffffffu, x.at, o);
    if (m > x.m || (m == x.m && at < x.at)) { x.m = m; x.at = at; }
  }
  for (int i = lane; i < slices; i += 32) {
    const float m = __ldcg(&parts[i].m), s = __ldcg(&parts[i].s);
    if (s != 0.f) x.s += m == x.m ? (double)s : (double)s * exp(((double)m - (double)x.m) * inv_tau);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
  return x;
}

// u q(x) and p(x), both times both sums: x passes iff left < right.
struct Sides { double left, right; };
__device__ __forceinline__ Sides sides_of(const VerifyCall& c, const Row& t, const Row& q, int64_t row, int draft_row, int x, double inv_tau) {
  const double u = (double)__ldg(c.u_accept + draft_row);
  const double pw = exp(((double)load(c.target, row, x) - (double)t.m) * inv_tau);
  const double qw = c.draft.p ? exp(((double)load(c.draft, draft_row, x) - (double)q.m) * inv_tau) : 1.0;
  return {u * qw * t.s, pw * (c.draft.p ? q.s : 1.0)};
}
__device__ __forceinline__ bool too_near(const Sides& e) { return fabs(e.left - e.right) <= 1e-5 * fabs(e.right); }

__global__ void __launch_bounds__(kRowThreads, kRowBlocks) verify_rows_kernel(const VerifyCall c, const Shape shape, float scale, const Workspace ws) {
  __shared__ RowPart warp_parts[2][kRowThreads / 32];
  __shared__ int s_skip;
  wait_for_predecessor();
  let_successor_start();
  const int slice = (int)(blockIdx.x % shape.slices), unit = (int)(blockIdx.x / shape.slices);
  const int r = unit % c.R, i = unit / c.R;        // first positions first
  const Span sp = span_of(c, r);
  if (!sp.ok || i > sp.n) return;
  if (threadIdx.x == 0) s_skip = *reinterpret_cast<volatile int*>(ws.stop + r) < i;
  __syncthreads();
  if (s_skip) {                                    // the request ends before this row, whatever is in it
    // A skipped slice is counted too: the ticket has to come back to 0.  Whoever is last then finds the request stopped before
    // i already, and what the skipped slice's part holds changes nothing.
    if (shape.slices > 1 && threadIdx.x == 0) atomicInc(ws.ticket + unit, shape.slices - 1);
    return;
  }
  const int lo = (int)((int64_t)c.V * slice / shape.slices), hi = (int)((int64_t)c.V * (slice + 1) / shape.slices);
  const int64_t row = sp.first + r + i;
  const int k = sp.first + i;                      // the draft's row
  const bool greedy = c.temperature == 0.f, dense = c.draft.p && i < sp.n;
  RowPart t = greedy ? thread_part<true>(c.target, row, lo, hi, scale) : thread_part<false>(c.target, row, lo, hi, scale);
  RowPart d{kNoMax, 0.f, kGoesOn, 0};
  if (dense) d = thread_part<false>(c.draft, k, lo, hi, scale);
  join_warp(t, scale);
  if (dense) join_warp(d, scale);
  if ((threadIdx.x & 31) == 0) { warp_parts[0][threadIdx.x >> 5] = t; warp_parts[1][threadIdx.x >> 5] = d; }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const bool in = threadIdx.x < kRowThreads / 32;
  t = in ? warp_parts[0][threadIdx.x] : RowPart{kNoMax, 0.f, kGoesOn, 0};
  d = in ? warp_parts[1][threadIdx.x] : t;
  join_warp(t, scale);
  if (dense) join_warp(d, scale);
  // whoever has the last slice puts the row together
  const double inv_tau = greedy ? 1.0 : 1.0 / (double)c.temperature;
  Row tr{t.m, t.at, (double)t.s}, dr{d.m, d.at, (double)d.s};
  if (shape.slices > 1) {
    RowPart* const t_at = ws.target + (int64_t)unit * shape.slices;
    RowPart* const d_at = ws.draft + (int64_t)unit * shape.slices;
    int last = 0;
    if (threadIdx.x == 0) {
      t_at[slice] = t;
      if (dense) d_at[slice] = d;
      __threadfence();
      last = atomicInc(ws.ticket + unit, shape.slices - 1) == shape.slices - 1u;       // back to 0 with the last
    }
    last = __shfl_sync(0xffffffffu, last, 0);
    if (!last) return;
    __threadfence();
    tr = warp_row(t_at, shape.slices, inv_tau);
    if (dense) dr = warp_row(d_at, shape.slices, inv_tau);
  }
  if (threadIdx.x != 0) return;
  ws.target_row[unit] = tr;
  if (i == sp.n) return;
  if (dense) ws.draft_row[unit] = dr;
  // if the draft surely does not pass, later rows of the request need not be read
  const int x = __ldg(c.draft_ids + k);
  Verdict v = kFails;                              // an id outside the vocabulary does
  if (!good(tr) || (dense && !good(dr))) v = kNoRow;
  else if (x >= 0 && x < c.V) {
    if (greedy) v = x == tr.at ? kPasses : kFails;
    else {
      const Sides e = sides_of(c, tr, dr, row, k, x, inv_tau);
      v = too_near(e) ? kTooNear : e.left < e.right ? kPasses : kFails;
    }
  }
  ws.verdict[unit] = v;
  if (v == kFails || v == kNoRow) atomicMin(ws.stop + r, i);
}

// --------------------------------------------------------------------------------- draws, in 64 bits
constexpr int kPowers = 64;
// 2^((z - m) / tau log2 e), relative to within 2^-44, and 2^-1000 from there down: what is no more than kNothing is no mass.
constexpr double kNothing = 0x1p-900;
struct Exp64 {
  const double* power;                             // 2^(j / 64)
  double c, b;                                     // log2 e / tau, -m times it
  __device__ __forceinline__ double operator()(float z) const {
    const double far = fma((double)z, c, b);
    // no less than -1000 or so, -inf too: among high words as unsigned numbers, -1000's is below those of all lesser numbers
    const double t = __hiloint2double((int)min((uint32_t)__double2hiint(far), 0xc08f4000u), __double2loint(far));
    constexpr double kShift = 0x1.8p52 / kPowers;  // adding it rounds to a multiple of 1/64, a whole number in the low bits
    const double shifted = t + kShift;
    const int n = __double2loint(shifted);
    const double r = t - (shifted - kShift);       // |r| <= 1/128
    // 2^r - 1 = r (ln 2 + r (ln^2 2 / 2 + r (ln^3 2 / 6 + r ln^4 2 / 24))); the next term is below 2^-44
    double p = fma(r, 9.6181291076284772e-3, 5.5504108664821580e-2);
    p = fma(r, p, 2.4022650695910071e-1);
    p = fma(r, p, 6.9314718055994531e-1);
    const double y = power[n & (kPowers - 1)];
    const double w = fma(y, r * p, y);
    return __hiloint2double(__double2hiint(w) + ((n & -kPowers) << (20 - 6)), __double2loint(w));       // times 2^(n / 64)
  }
};
__device__ __forceinline__ Exp64 exp_about(const double* power, float m, double inv_tau) {
  const double c = inv_tau * 1.4426950408889634074;
  return {power, c, -(double)m * c};
}

// Sum over the block, in a fixed order; every thread gets it.
__device__ double block_sum(double a, double* warp_sums) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = a;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < kDrawWarps; ++w) all += warp_sums[w];
  return all;
}
__device__ __forceinline__ float value(const float* p) { return __ldg(p); }
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
template <class T>
__device__ __forceinline__ const T* row_of(const LogitRows& x, int64_t row) { return static_cast<const T*>(x.p) + row * x.pitch; }

constexpr int kAhead = 8;                          // loads under way per thread
// Calls use(v, row[v]) for v = first, first + step, ... below hi.
template <class T, class Use>
__device__ __forceinline__ void each(const T* row, int first, int hi, int step, Use use) {
  int v = first;
  for (; v + (kAhead - 1) * step < hi; v += kAhead * step) {
    float z[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) z[k] = value(row + v + k * step);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) use(v + k * step, z[k]);
  }
  for (; v < hi; v += step) use(v, value(row + v));
}
// The same for two rows at a time.
template <class T, class Q, class Use>
__device__ __forceinline__ void each_pair(const T* row, const Q* other, int first, int hi, int step, Use use) {
  int v = first;
  for (; v + (kAhead / 2 - 1) * step < hi; v += kAhead / 2 * step) {
    float z[kAhead / 2], q[kAhead / 2];
#pragma unroll
    for (int k = 0; k < kAhead / 2; ++k) { z[k] = value(row + v + k * step); q[k] = value(other + v + k * step); }
#pragma unroll
    for (int k = 0; k < kAhead / 2; ++k) use(v + k * step, z[k], q[k]);
  }
  for (; v < hi; v += step) use(v, value(row + v), value(other + v));
}
template <class T>
__device__ double exact_sum(const T* row, int lo, int hi, const Exp64& e, double* warp_sums) {
  double a = 0.0, b = 0.0;
  each(row, lo + (int)threadIdx.x, hi, kDrawThreads, [&](int, float z) {
    const double w = a;                            // two chains
    a = b;
    b = w + e(z);
  });
  return block_sum(a + b, warp_sums);
}

__device__ __forceinline__ Row dense_of(const Workspace& ws, const VerifyCall& c, int unit) { return c.draft.p ? ws.draft_row[unit] : Row{}; }

// A cluster per request.  T, Q: types of the target's and the drafts' logits.
template <class T, class Q>
__global__ void __launch_bounds__(kDrawThreads, 2) verify_draw_kernel(const VerifyCall c, const Shape shape, const Workspace ws, unsigned int* d_err) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  __shared__ double s_power[kPowers], s_warp[kDrawWarps], s_sum[4];       // s_sum: this CTA's shares, read by the cluster
  __shared__ double s_segment[kDrawWarps];
  __shared__ int s_first;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x < kPowers) s_power[threadIdx.x] = exp2((double)threadIdx.x / kPowers);
  wait_for_predecessor();
  let_successor_start();
  const int r = (int)blockIdx.x / ctas;
  const Span sp = span_of(c, r);
  const bool leader = rank == 0 && threadIdx.x == 0;
  if (leader) {
    unsigned int bad = sp.ok ? 0 : AF_DEVERR_CU_SEQLENS;
    if (r == 0 && __ldg(c.cu) != 0) bad |= AF_DEVERR_CU_SEQLENS;
    if (r == c.R - 1 && __ldg(c.cu + c.R) != c.D) bad |= AF_DEVERR_CU_SEQLENS;
    if (bad) atomicOr(d_err, bad);
    if (!sp.ok) c.n_emitted[r] = 0;
    ws.stop[r] = kGoesOn;                                     // for the next call
  }
  if (!sp.ok) return;                                         // the whole cluster
  const bool greedy = c.temperature == 0.f;
  const double inv_tau = greedy ? 1.0 : 1.0 / (double)c.temperature;
  const int64_t base = sp.first + r;
  const int lo = (int)((int64_t)c.V * rank / ctas), hi = (int)((int64_t)c.V * (rank + 1) / ctas);

  // ---- the first draft that does not pass: every CTA of the cluster finds it by itself
  auto unit = [&](int j) { return j * c.R + r; };
  auto log_prob = [&](const Row& x, int64_t row, int v) {
    return (float)(((double)load(c.target, row, v) - (double)x.m) * inv_tau - log(x.s));
  };
  int i = 0;
  for (;;) {
    if (warp == 0) {                                          // the next one that does not pass in 32 bits
      int j = i;
      for (; j < sp.n; j += 32) {
        const bool stops = j + lane < sp.n && __ldcg(ws.verdict + unit(j + lane)) != kPasses;
        const unsigned any = __ballot_sync(0xffffffffu, stops);
        if (any) { j += __ffs(any) - 1; break; }
      }
      if (lane == 0) s_first = min(j, sp.n);
    }
    __syncthreads();
    i = s_first;
    if (i == sp.n || __ldcg(ws.verdict + unit(i)) != kTooNear) break;
    Row t = ws.target_row[unit(i)], q = dense_of(ws, c, unit(i));        // the same in all threads of the cluster
    t.s = exact_sum(row_of<T>(c.target, base + i), 0, c.V, exp_about(s_power, t.m, inv_tau), s_warp);
    if (c.draft.p) q.s = exact_sum(row_of<Q>(c.draft, sp.first + i), 0, c.V, exp_about(s_power, q.m, inv_tau), s_warp);
    const Sides e = sides_of(c, t, q, base + i, sp.first + i, __ldg(c.draft_ids + sp.first + i), inv_tau);
    if (!(e.left < e.right)) break;
    ++i;                                                      // it passes; go on behind it
    __syncthreads();                                          // s_first has been read
  }
  const Row t = ws.target_row[unit(i)];
  const Row q = i < sp.n ? dense_of(ws, c, unit(i)) : Row{};
  const bool has_row = good(t) && (i == sp.n || !c.draft.p || good(q));
  if (rank == 0 && warp == 0) {
    for (int j = lane; j <= sp.n; j += 32) {
      const int x = j < i ? __ldg(c.draft_ids + sp.first + j) : j > i ? -1 : greedy && has_row ? t.at : -1;
      if (j != i || greedy || !has_row) c.token[base + j] = x;        // the others draw it
      if (!c.logp) continue;
      if (j < i) c.logp[base + j] = log_prob(ws.target_row[unit(j)], base + j, x);
      else if (j > i) c.logp[base + j] = 0.f;
      else if (!has_row) c.logp[base + j] = __int_as_float(0x7fc00000);
      else if (greedy) c.logp[base + j] = (float)-log(t.s);
    }
    if (lane == 0) {
      c.n_emitted[r] = has_row ? i + 1 : i;
      unsigned int bad = has_row ? 0 : AF_DEVERR_DISTRIBUTION;
      if (good(t) && i < sp.n) {
        const int x = __ldg(c.draft_ids + sp.first + i);
        if (x < 0 || x >= c.V) bad |= AF_DEVERR_TARGET_RANGE;
      }
      if (bad) atomicOr(d_err, bad);
    }
  }
  if (!has_row || greedy) return;                             // the whole cluster

  // ---- the token after them, from row base + i
  const bool rejected = i < sp.n, dense = rejected && c.draft.p != nullptr;
  const int cut = rejected && !dense ? __ldg(c.draft_ids + sp.first + i) : -1;
  const T* const p_row = row_of<T>(c.target, base + i);
  const Q* const q_row = dense ? row_of<Q>(c.draft, sp.first + i) : nullptr;
  const Exp64 pe = exp_about(s_power, t.m, inv_tau), qe = exp_about(s_power, q.m, inv_tau);
  double p_unit = 1.0, q_unit = 1.0;                          // dense: 1 / sums
  double row_sum = 0.0;                                       // of the target's weights
  if (dense) {
    double a = 0.0, b = 0.0;
    each_pair(p_row, q_row, lo + (int)threadIdx.x, hi, kDrawThreads, [&](int, float z, float zq) { a += pe(z); b += qe(zq); });
    a = block_sum(a, s_warp);
    b = block_sum(b, s_warp);
    if (threadIdx.x == 0) { s_sum[0] = a; s_sum[1] = b; }
    cluster.sync();
    double sum_q = 0.0;
    for (int k = 0; k < ctas; ++k) {
      row_sum += *cluster.map_shared_rank(&s_sum[0], k);
      sum_q += *cluster.map_shared_rank(&s_sum[1], k);
    }
    p_unit = 1.0 / row_sum;
    q_unit = 1.0 / sum_q;
  }
  // a warp's segment of the CTA's share
  const int seg_lo = lo + (int)((int64_t)(hi - lo) * warp / kDrawWarps), seg_hi = lo + (int)((int64_t)(hi - lo) * (warp + 1) / kDrawWarps);
  bool plain = !rejected;                                     // drawn from the target itself
  auto left = [&](float z, float zq) { return fmax(pe(z) * p_unit - qe(zq) * q_unit, 0.0); };      // of p less q
  double before, total;
  for (;;) {
    double a = 0.0, whole = 0.0;
    if (dense && !plain) each_pair(p_row, q_row, seg_lo + lane, seg_hi, 32, [&](int, float z, float zq) { a += left(z, zq); });
    else {
      const auto take = [&](int, float z) { a += pe(z); };
      const bool cuts = !plain && cut >= seg_lo && cut < seg_hi;
      each(p_row, seg_lo + lane, cuts ? cut : seg_hi, 32, take);
      if (cuts) each(p_row, cut + 1 + lane, seg_hi, 32, take);
      whole = a + (cuts && lane == 0 ? pe(value(p_row + cut)) : 0.0);
    }
    if (dense && plain) a *= p_unit;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      whole += __shfl_xor_sync(0xffffffffu, whole, o);
    }
    __syncthreads();
    if (lane == 0) { s_segment[warp] = a; s_warp[warp] = whole; }
    __syncthreads();
    if (threadIdx.x == 0) {
      double run = 0.0, all = 0.0;
      for (int k = 0; k < kDrawWarps; ++k) {
        const double x = s_segment[k];
        s_segment[k] = run;
        run += x;
        all += s_warp[k];
      }
      s_sum[2] = run;
      s_sum[3] = all;
    }
    cluster.sync();
    before = total = 0.0;
    double all = 0.0;
    for (int k = 0; k < ctas; ++k) {
      if (k == rank) before = total;
      total += *cluster.map_shared_rank(&s_sum[2], k);
      all += *cluster.map_shared_rank(&s_sum[3], k);
    }
    cluster.sync();                                           // s_sum is read by all before it is written again, or its CTA ends
    if (!dense) row_sum = all;
    if (plain || (dense ? total : total / row_sum) > kResidualFloor) break;
    plain = true;                                             // next to nothing is left: the target itself
  }
  // the CTA whose share holds the first v with C_v > u C, and the segment of it that does
  const double u = (double)fminf(fmaxf(__ldg(c.u_sample + r), 0.f), 1.f - 0x1p-24f), goal = u * total;
  if (!(before <= goal && goal < before + s_sum[2])) return;  // the whole CTA
  int found = 0;
  for (int k = 1; k < kDrawWarps; ++k)
    if (before + s_segment[k] <= goal) found = k;
  const double at_segment = before + s_segment[found];
  const int f_lo = lo + (int)((int64_t)(hi - lo) * found / kDrawWarps), f_hi = lo + (int)((int64_t)(hi - lo) * (found + 1) / kDrawWarps);
  auto mass = [&](int v) {
    if (!plain && v == cut) return 0.0;
    if (!dense) return pe(value(p_row + v));
    return plain ? pe(value(p_row + v)) * p_unit : left(value(p_row + v), value(q_row + v));
  };
  // all warps share that segment out once more
  const int part_lo = f_lo + (int)((int64_t)(f_hi - f_lo) * warp / kDrawWarps), part_hi = f_lo + (int)((int64_t)(f_hi - f_lo) * (warp + 1) / kDrawWarps);
  double a = 0.0;
#pragma unroll 4
  for (int v = part_lo + lane; v < part_hi; v += 32) a += mass(v);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  if (lane == 0) s_warp[warp] = a;
  __syncthreads();
  double run = at_segment, start = at_segment;
  int mine = 0;                                               // the last part with mass that starts at or before the goal
  for (int k = 0; k < kDrawWarps; ++k) {
    if (run <= goal && s_warp[k] > kNothing) { mine = k; start = run; }
    run += s_warp[k];
  }
  if (warp != mine) return;
  run = start;
  int y = part_lo;                                            // the last with mass, if rounding leaves the goal beyond the part
  for (int v0 = part_lo; v0 < part_hi; v0 += 32) {
    const int v = v0 + lane;
    const double w = v < part_hi ? mass(v) : 0.0;
    double upto = w;                                          // sum over the lanes up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    const unsigned some = __ballot_sync(0xffffffffu, w > kNothing), beyond = __ballot_sync(0xffffffffu, w > kNothing && run + upto > goal);
    if (beyond) { y = v0 + __ffs(beyond) - 1; break; }
    if (some) y = v0 + 31 - __clz(some);
    run += __shfl_sync(0xffffffffu, upto, 31);
  }
  if (lane == 0) {
    c.token[base + i] = y;
    if (c.logp) c.logp[base + i] = (float)(((double)load(c.target, base + i, y) - (double)t.m) * inv_tau - log(row_sum));
  }
}

// Slices of a row.  A batch of rows that fills the device several times over goes row by row, so that positions end in order;
// fewer are cut until every SM has about four slices, of 2048 logits at least.
Shape shape_of(int32_t R, int32_t V, int32_t max_draft, int sm_count) {
  const int64_t units = (int64_t)R * (max_draft + 1), want = ((int64_t)sm_count * 4 + units - 1) / units, most = V / 2048;
  const int64_t slices = want < most ? want : most;
  return {(int)(slices < 1 ? 1 : slices), max_draft + 1};
}
// CTAs to a request: as many as a full device has room for.
int cluster_of(int32_t R, int32_t V, int sm_count) {
  int ctas = kMostCluster;
  while (ctas > 1 && ((int64_t)R * ctas > (int64_t)sm_count * (ctas == kMostCluster ? 1 : 8) || V / ctas < 512)) ctas /= 2;
  return ctas;
}

template <class T, class Q>
af_status launch_draws(const cudaLaunchConfig_t& cfg, const VerifyCall& c, const Shape& shape, const Workspace& ws, unsigned int* d_err) {
  static SmemAttrOnce once;                                   // per device: clusters of more CTAs than every part has to take
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return AF_ERR_CUDA;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
  if (!bit || !(once.done.load(std::memory_order_acquire) & bit)) {
    if (cudaFuncSetAttribute(verify_draw_kernel<T, Q>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return AF_ERR_CUDA;
    once.done.fetch_or(bit, std::memory_order_release);
  }
  return cudaLaunchKernelEx(&cfg, verify_draw_kernel<T, Q>, c, shape, ws, d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }
struct Sizes { size_t parts, rows, verdicts, tickets, stops; };
// Rows in several slices are few: fewer than 8 parts per SM in all, and as many of the drafts; and parts and tickets are used
// only there.  So smaller calls of any kind fit in what a larger one needs.
Sizes sizes_of(int32_t R, int32_t max_draft, int sm_count) {
  const size_t units = (size_t)R * ((size_t)max_draft + 1);
  return {(size_t)sm_count * 16 * sizeof(RowPart), units * 2 * sizeof(Row), units * sizeof(int32_t),
          round16((size_t)sm_count * 4 * sizeof(unsigned int)), (size_t)R * sizeof(int)};
}

}  // namespace

// Sizes the workspace; what a call leaves as it found it, the tickets and the stops, is set where the memory is new.
af_status reserve_draft_verify(af_ctx* ctx, int32_t R, int32_t max_draft, cudaStream_t s) {
  const Sizes z = sizes_of(R, max_draft, ctx->sm_count);
  af_status st = ws_grow(ctx->verify_ws, z.parts + z.rows + z.verdicts);
  if (st != AF_OK) return st;
  const size_t had = ctx->verify_state.cap;
  st = ws_grow(ctx->verify_state, z.tickets + z.stops);
  if (st != AF_OK) return st;
  if (ctx->verify_state.cap != had) {
    char* const p = static_cast<char*>(ctx->verify_state.p);
    const size_t stops = ctx->verify_state.cap - z.tickets;
    if (cudaMemsetAsync(p, 0, z.tickets, s) != cudaSuccess || cudaMemsetAsync(p + z.tickets, 0x7f, stops, s) != cudaSuccess)
      return AF_ERR_CUDA;
  }
  return AF_OK;
}

af_status launch_draft_verify(af_ctx* ctx, const VerifyCall& c, cudaStream_t s) {
  const af_status st = reserve_draft_verify(ctx, c.R, c.max_draft, s);
  if (st != AF_OK) return st;
  const Shape shape = shape_of(c.R, c.V, c.max_draft, ctx->sm_count);
  Workspace ws;
  const Sizes z = sizes_of(c.R, c.max_draft, ctx->sm_count);
  char* const at = static_cast<char*>(ctx->verify_ws.p);
  ws.target = reinterpret_cast<RowPart*>(at);
  ws.draft = ws.target + (size_t)c.R * shape.positions * shape.slices;
  ws.target_row = reinterpret_cast<Row*>(at + z.parts);
  ws.draft_row = ws.target_row + (size_t)c.R * shape.positions;
  ws.verdict = reinterpret_cast<int32_t*>(at + z.parts + z.rows);
  ws.ticket = static_cast<unsigned int*>(ctx->verify_state.p);
  ws.stop = reinterpret_cast<int*>(static_cast<char*>(ctx->verify_state.p) + z.tickets);
  const float scale = c.temperature == 0.f ? kLog2e : kLog2e / c.temperature;
  const int64_t blocks = (int64_t)c.R * shape.positions * shape.slices;
  if (launch_overlapped(verify_rows_kernel, (unsigned)blocks, kRowThreads, 0, s, c, shape, scale, ws) != cudaSuccess) return AF_ERR_CUDA;
  const int ctas = c.temperature == 0.f ? 1 : cluster_of(c.R, c.V, ctx->sm_count);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = (unsigned)c.R * ctas;
  cfg.blockDim = kDrawThreads;
  cfg.stream = s;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const bool wide_draft = !c.draft.p || c.draft.type == AF_F32;
  using bf16 = __nv_bfloat16;
  if (c.target.type == AF_F32)
    return wide_draft ? launch_draws<float, float>(cfg, c, shape, ws, ctx->d_err) : launch_draws<float, bf16>(cfg, c, shape, ws, ctx->d_err);
  return wide_draft ? launch_draws<bf16, float>(cfg, c, shape, ws, ctx->d_err) : launch_draws<bf16, bf16>(cfg, c, shape, ws, ctx->d_err);
}

}  // namespace af
