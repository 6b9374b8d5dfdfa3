// af_draft_verify: drafted tokens against the target's distribution, from given uniforms.
//
// The first launch reads rows of logits once, in slices, for their maxima and sums of exponentials (fp32: a stream at the
// memory's rate, next to which the exponentials fit).  It goes through the batch by positions, first drafts first, and a
// row of a request that has already been seen to stop is not read.  Whoever finishes a row decides whether its draft passes.
// Then, per request: the first draft that does not pass and, for a draw from what the draft leaves of the target, both rows' exact
// sums; the mass of a few hundred segments; the segment, and in it the token, that the uniform points at.  Three launches of
// slices that know nothing of one another: a cluster per request, with the sums in its shared memory, spent most of
// its time waiting for its slowest CTA (64 requests: 75 us for 15 us of 64-bit operations).
//
// What has to be exact is whole numbers: a comparison u q < p, and the place of u C among running sums C_v of up to
// 10^5 terms, where fp32 would be off by as much as many terms are large.  So a comparison whose sides are within 2e-5 is
// made again from sums in 64 bits, and a draw's sums are in 64 bits throughout: per logit nine 64-bit operations, 2^x from a table
// of 256 powers and a polynomial of degree 3 (2^-42 relative).
//
// 64 requests of up to 4 drafts, bf16 and fp32 logits of 152064: 103-105 us.  Each alone and cold the rows take 51 (253 MB at 5 TB/s,
// of which 208 had to be read; their exponentials keep the special unit busy half of the time), sums 22, mass 33, find 10: a call
// overlaps their beginnings and ends.  One request 24-28 us, four launches.
#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowBlocks = 4;                      // rows, or slices, on an SM at a time: few, so that positions end in order
constexpr int kDrawThreads = 256;                  // a slice of a request's vocabulary
constexpr int kDrawWarps = kDrawThreads / 32;      // each with a segment of the slice
constexpr int kMostSlices = 64;
constexpr int kFindThreads = kMostSlices * kDrawWarps;       // one per segment
constexpr int kFindWarps = kFindThreads / 32;
constexpr float kNoMax = -INFINITY;
constexpr double kResidualFloor = 0x1p-30;         // a residual with less mass than this is drawn from the target itself
constexpr int kGoesOn = 0x7fffffff;

// A row's sum exp((z - m) / tau) is about its maximum, or about a logit up to four halvings of the exponential less (greedy: the
// maximum, and its place).
struct RowPart {                                   // of a slice
  float m, s;
  int32_t at, pad;
};
struct Row {                                       // of the whole, in 64 bits
  float m;
  int32_t at;
  double s;
};
enum Verdict : int32_t { kPasses, kFails, kTooNear, kNoRow };       // too near to tell in 32 bits; target or draft is no distribution
// Places are by unit, position * R + request: each request has its own, whatever cu_draft says.
struct Draw;
struct Workspace {
  RowPart* target;                                 // [units][slices]
  RowPart* draft;                                  // [units][slices]
  Row* target_row;                                 // [units]
  Row* draft_row;                                  // [units]
  int32_t* verdict;                                // [units]
  unsigned int* ticket;                            // [units] slices done, zero between calls
  int* stop;                                       // [R] first draft that is known not to pass, kGoesOn between calls
  Draw* draw;                               // [R]
  double2* sums;                                   // [R][draw slices] exact sums of the target's and the draft's row
  double2* mass;                                   // [R][segments] mass, and the target's whole weight
};
enum Kind : int32_t { kNoDraw, kPlain, kCut, kDense };       // from the target; without the draft; from max(target - draft, 0)
struct Draw {                                      // how a request's last token is drawn
  int64_t row;                                     // the target's row
  int32_t kind, draft_row, cut;                    // cut: the draft that is left out
  float m, m_draft;                                // what the rows' sums are about
};
struct Shape {
  int slices, positions;                           // slices of a row; max_draft + 1
  int draw_slices;                                 // slices of a vocabulary in a draw
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
// A thread's part on the way.  `sum` takes eight additions at most before it is folded into `whole`, whose roundings `rest` keeps: in a
// long row of equal terms those of one plain sum would all go the same way (4 million flat logits: 1.5e-5 off).  m moves only to a
// logit of two halvings more, so that the sums are scaled once or twice, not with every step of a rising row.
struct RowSum {
  float m, sum, whole, rest;
  float limit;                                     // above it m moves; kPlace: the maximum, and its place
  int32_t at;
  __device__ __forceinline__ void fold() {
    const float t = __fadd_rn(whole, sum);
    rest += __fsub_rn(sum, __fsub_rn(t, whole));             // what t lacks, exactly but where m has just moved and `whole` is the less
    whole = t;
    sum = 0.f;
  }
};

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
__device__ __forceinline__ void add(RowSum& a, const Values<n>& x, int at, float scale, float slack) {
  float top = x.v[0];
#pragma unroll
  for (int i = 1; i < n; ++i) top = fmaxf(top, x.v[i]);
  if (top > a.limit) {                             // rare after the first few
    if constexpr (kPlace) {
      a.limit = top;
#pragma unroll
      for (int i = n - 1; i >= 0; --i)
        if (x.v[i] == top) a.at = at + i;
    }
    if (!kPlace || top > a.m + slack) {
      const float less = ex2f((a.m - top) * scale);          // 0 times 0 at first
      a.sum *= less;
      a.whole *= less;
      a.rest *= less;
      a.m = top;
      if (!kPlace) a.limit = top + slack;
    }
  }
  if (a.m == kNoMax) {                             // nothing but -inf so far, or a NaN
#pragma unroll
    for (int i = 0; i < n; ++i)
      if (x.v[i] != x.v[i]) a.sum = x.v[i];
    return;
  }
  // a NaN, and infinity less itself, make the sum NaN
  if constexpr (n == 1) {
    a.sum += ex2f((x.v[0] - a.m) * scale);
  } else {
    const float2 less = make_float2(-a.m, -a.m), by = make_float2(scale, scale);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < n; i += 2) {
      const float2 e = __fmul2_rn(__fadd2_rn(make_float2(x.v[i], x.v[i + 1]), less), by);
      sum = __fadd2_rn(sum, make_float2(ex2f(e.x), ex2f(e.y)));
    }
    a.sum += sum.x + sum.y;
  }
}

template <bool kPlace, class T>
__device__ RowPart row_part(const T* row, int lo, int hi, float scale, float slack) {
  constexpr int kVec = 16 / sizeof(T), kLoads = 4;
  RowSum a{kNoMax, 0.f, 0.f, 0.f, kNoMax, kGoesOn};
  // single elements up to a multiple of 16 bytes, and behind the last one
  const int to_line = (int)((16u - ((uint32_t)reinterpret_cast<uintptr_t>(row + lo) & 15u)) & 15u) / (int)sizeof(T);
  const int body = min(hi, lo + to_line), vecs = (hi - body) / kVec, tail = body + vecs * kVec;
  if (lo + (int)threadIdx.x < body) add<kPlace>(a, widen1(row + lo + threadIdx.x), lo + threadIdx.x, scale, slack);
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
    for (int k = 0; k < kLoads; ++k) add<kPlace>(a, widen(row, w[k]), body + (i + k * kRowThreads) * kVec, scale, slack);
    a.fold();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) w[k] = ahead[k];
  }
  for (; i < vecs; i += kRowThreads) add<kPlace>(a, widen(row, __ldg(at + i)), body + i * kVec, scale, slack);
  if (tail + (int)threadIdx.x < hi) add<kPlace>(a, widen1(row + tail + threadIdx.x), tail + threadIdx.x, scale, slack);
  a.fold();
  const float s = a.whole + a.rest;
  if (kPlace && a.limit > a.m) return {a.limit, s * ex2f((a.m - a.limit) * scale), a.at, 0};
  return {a.m, s, a.at, 0};
}

template <bool kPlace>
__device__ RowPart thread_part(const LogitRows& x, int64_t row, int lo, int hi, float scale, float slack) {
  return x.type == AF_F32 ? row_part<kPlace>(static_cast<const float*>(x.p) + row * x.pitch, lo, hi, scale, slack)
                          : row_part<kPlace>(static_cast<const __nv_bfloat16*>(x.p) + row * x.pitch, lo, hi, scale, slack);
}
__device__ __forceinline__ RowPart no_part() { return {kNoMax, 0.f, kGoesOn, 0}; }
// Parts are joined about the largest m of all, each scaled once.  Floats that are no NaN order as whole numbers do once the bits below the
// sign of negative ones are turned over.
__device__ __forceinline__ int32_t ordered(int32_t bits) { return bits ^ ((bits >> 31) & 0x7fffffff); }
__device__ __forceinline__ float warp_max(float m) {
  return __int_as_float(ordered(__reduce_max_sync(0xffffffffu, ordered(__float_as_int(m)))));
}
// A part without mass adds nothing (its m may be -inf); a NaN stays.
__device__ __forceinline__ float sum_about(const RowPart& a, float m, float scale) { return a.s == 0.f ? 0.f : a.s * ex2f((a.m - m) * scale); }
// s, at: of a lane, about the warp's m.
__device__ __forceinline__ RowPart join_lanes(float m, float s, int at) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return {m, s, __reduce_min_sync(0xffffffffu, at), 0};
}
__device__ __forceinline__ void join_warp(RowPart& a, float scale) {
  const float m = warp_max(a.m);
  a = join_lanes(m, sum_about(a, m, scale), a.m == m ? a.at : kGoesOn);
}

__device__ __forceinline__ bool good(const Row& x) { return fabsf(x.m) < INFINITY && x.s > 0.0 && x.s < 1e300; }
__device__ __forceinline__ RowPart fetch_part(const RowPart* p) {
  const uint4 x = __ldcg(reinterpret_cast<const uint4*>(p));
  return {__uint_as_float(x.x), __uint_as_float(x.y), (int32_t)x.z, 0};
}
// A row's slices, by a whole warp.
__device__ __forceinline__ RowPart join_slices(const RowPart* parts, int slices, float scale) {
  const int lane = threadIdx.x & 31;
  const RowPart first = lane < slices ? fetch_part(parts + lane) : no_part();
  float m = first.m;
  for (int i = lane + 32; i < slices; i += 32) m = fmaxf(m, fetch_part(parts + i).m);
  m = warp_max(m);
  float s = sum_about(first, m, scale);
  int at = first.m == m ? first.at : kGoesOn;
  for (int i = lane + 32; i < slices; i += 32) {
    const RowPart a = fetch_part(parts + i);
    s += sum_about(a, m, scale);
    if (a.m == m) at = min(at, a.at);
  }
  return join_lanes(m, s, at);
}

// u q(x) and p(x), both times both sums: x passes iff left < right.
struct Sides { double left, right; };
__device__ __forceinline__ Sides sides_of(const Row& t, const Row& q, float u, float z, float zq, bool dense, double inv_tau) {
  const double pw = exp(((double)z - (double)t.m) * inv_tau), qw = dense ? exp(((double)zq - (double)q.m) * inv_tau) : 1.0;
  return {(double)u * qw * t.s, pw * (dense ? q.s : 1.0)};
}
// A row's sum is off by 8e-6 at most: an argument of e halvings is rounded three times (difference, 1 / tau, product), 3 u e ln 2 with
// u = 2^-24, and e is log2 V on the weighted average of the terms at most, 4 more for what m is short of;  ex2.approx is good to 4 u,
// for the term, at most twice where m moves, and three times where parts are joined;  40 additions, eight of a thread's and those that join parts.  Both sides together stay within this:
constexpr double kNear = 2e-5;
__device__ __forceinline__ bool too_near(const Sides& e) { return fabs(e.left - e.right) <= kNear * fabs(e.right); }

__global__ void __launch_bounds__(kRowThreads, kRowBlocks) verify_rows_kernel(const VerifyCall c, const Shape shape, float scale, float slack, const Workspace ws) {
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
  RowPart t = greedy ? thread_part<true>(c.target, row, lo, hi, scale, slack) : thread_part<false>(c.target, row, lo, hi, scale, slack);
  RowPart d = no_part();
  if (dense) d = thread_part<false>(c.draft, k, lo, hi, scale, slack);
  join_warp(t, scale);
  if (dense) join_warp(d, scale);
  if ((threadIdx.x & 31) == 0) { warp_parts[0][threadIdx.x >> 5] = t; warp_parts[1][threadIdx.x >> 5] = d; }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const bool in = threadIdx.x < kRowThreads / 32;
  t = in ? warp_parts[0][threadIdx.x] : no_part();
  d = in ? warp_parts[1][threadIdx.x] : t;
  join_warp(t, scale);
  if (dense) join_warp(d, scale);
  // whoever has the last slice puts the row together
  const double inv_tau = greedy ? 1.0 : 1.0 / (double)c.temperature;
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
    t = join_slices(t_at, shape.slices, scale);
    if (dense) d = join_slices(d_at, shape.slices, scale);
  }
  const Row tr{t.m, t.at, (double)t.s}, dr{d.m, d.at, (double)d.s};
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
      const Sides e = sides_of(tr, dr, __ldg(c.u_accept + k), load(c.target, row, x), dense ? load(c.draft, k, x) : 0.f, dense, inv_tau);
      v = too_near(e) ? kTooNear : e.left < e.right ? kPasses : kFails;
    }
  }
  ws.verdict[unit] = v;
  if (v == kFails || v == kNoRow) atomicMin(ws.stop + r, i);
}

// --------------------------------------------------------------------------------- draws, in 64 bits
constexpr int kPowers = 256;
// 2^((z - m) / tau log2 e), relative to within 2^-42, and 2^-1000 from there down: what is no more than kNothing is no mass,
// and sums of it count as 0 (a uniform of 0 takes the first token with mass, which a sum above 0 before it would hide).
constexpr double kNothing = 0x1p-900;
__device__ __forceinline__ double some_mass(double sum) { return sum > kNothing ? sum : 0.0; }
struct Exp64 {
  const double* power;                             // 2^(j / 256)
  double c, m;                                     // log2 e / tau, and what is subtracted before it multiplies:
  // z c - m c in one operation would be off by the rounding of m c, which for the lowest logits of a type is far beyond the range of
  // any exponential, at z = m too
  __device__ __forceinline__ double operator()(float z) const {
    const double far = ((double)z - m) * c;
    // no less than -1000 or so, -inf too: among high words as unsigned numbers, -1000's is below those of all lesser numbers
    const double t = __hiloint2double((int)min((uint32_t)__double2hiint(far), 0xc08f4000u), __double2loint(far));
    constexpr double kShift = 0x1.8p52 / kPowers;  // adding it rounds to a multiple of 1/256, a whole number in the low bits
    const double shifted = t + kShift;
    const int n = __double2loint(shifted);
    const double r = t - (shifted - kShift);       // |r| <= 1/512
    // 2^r = 1 + r (ln 2 + r (ln^2 2 / 2 + r ln^3 2 / 6)); the next term is below 2^-42
    double p = fma(r, 5.5504108664821580e-2, 2.4022650695910071e-1);
    p = fma(r, p, 6.9314718055994531e-1);
    p = fma(r, p, 1.0);
    const double y = power[n & (kPowers - 1)];
    // times 2^(n / 256); where it is added to a sum, so is the product
    return __hiloint2double(__double2hiint(y) + ((n & -kPowers) << (20 - 8)), __double2loint(y)) * p;
  }
};
__device__ __forceinline__ Exp64 exp_about(const double* power, float m, double inv_tau) {
  return {power, inv_tau * 1.4426950408889634074, (double)m};
}

// Sum over the block of kWarps warps, in a fixed order; every thread gets it.
template <int kWarps>
__device__ double block_sum(double a, double* warp_sums) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = a;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) all += warp_sums[w];
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
  return block_sum<kDrawWarps>(a + b, warp_sums);
}

__device__ __forceinline__ Row dense_of(const Workspace& ws, const VerifyCall& c, int unit) { return c.draft.p ? ws.draft_row[unit] : Row{}; }

// Segment k of a vocabulary cut into n.
__device__ __forceinline__ int segment_at(int V, int k, int n) { return (int)((int64_t)V * k / n); }
__device__ __forceinline__ double inverse_temperature(const VerifyCall& c) { return c.temperature == 0.f ? 1.0 : 1.0 / (double)c.temperature; }
__device__ __forceinline__ void set_powers(double* power) {
  if (threadIdx.x < kPowers) power[threadIdx.x] = exp2((double)threadIdx.x / kPowers);
}

// What passes, and how the token after it is drawn.  Every CTA of a request finds out by itself; the first writes it down.
// T, Q: types of the target's and the drafts' logits.
template <class T, class Q>
__global__ void __launch_bounds__(kDrawThreads) verify_sums_kernel(const VerifyCall c, const Shape shape, const Workspace ws, unsigned int* d_err) {
  __shared__ double s_power[kPowers], s_warp[kDrawWarps];
  __shared__ int s_first;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  set_powers(s_power);
  wait_for_predecessor();
  let_successor_start();
  const int r = (int)blockIdx.x / shape.draw_slices, slice = (int)blockIdx.x % shape.draw_slices;
  const Span sp = span_of(c, r);
  if (slice == 0 && threadIdx.x == 0) {
    unsigned int bad = sp.ok ? 0 : AF_DEVERR_CU_SEQLENS;
    if (r == 0 && __ldg(c.cu) != 0) bad |= AF_DEVERR_CU_SEQLENS;
    if (r == c.R - 1 && __ldg(c.cu + c.R) != c.D) bad |= AF_DEVERR_CU_SEQLENS;
    if (bad) atomicOr(d_err, bad);
    ws.stop[r] = kGoesOn;                                     // for the next call
    if (!sp.ok) {
      c.n_emitted[r] = 0;
      ws.draw[r] = Draw{0, kNoDraw, 0, 0, 0.f, 0.f};
    }
  }
  if (!sp.ok) return;
  const bool greedy = c.temperature == 0.f;
  const double inv_tau = inverse_temperature(c);
  const int64_t base = sp.first + r;
  auto unit = [&](int j) { return j * c.R + r; };
  int i = 0;
  for (;;) {
    if (warp == 0) {                                          // the next draft that does not pass in 32 bits
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
    Row t = ws.target_row[unit(i)], q = dense_of(ws, c, unit(i));        // the same in all threads of the request
    t.s = exact_sum(row_of<T>(c.target, base + i), 0, c.V, exp_about(s_power, t.m, inv_tau), s_warp);
    if (c.draft.p) q.s = exact_sum(row_of<Q>(c.draft, sp.first + i), 0, c.V, exp_about(s_power, q.m, inv_tau), s_warp);
    const int x = __ldg(c.draft_ids + sp.first + i);
    const Sides e = sides_of(t, q, __ldg(c.u_accept + sp.first + i), load(c.target, base + i, x),
                             c.draft.p ? load(c.draft, sp.first + i, x) : 0.f, c.draft.p != nullptr, inv_tau);
    if (!(e.left < e.right)) break;
    ++i;                                                      // it passes; go on behind it
    __syncthreads();                                          // s_first has been read
  }
  const Row t = ws.target_row[unit(i)];
  const Row q = i < sp.n ? dense_of(ws, c, unit(i)) : Row{};
  const bool has_row = good(t) && (i == sp.n || !c.draft.p || good(q));
  const int kind = !has_row || greedy ? kNoDraw : i == sp.n ? kPlain : c.draft.p ? kDense : kCut;
  if (slice == 0 && warp == 0) {
    for (int j = lane; j <= sp.n; j += 32) {
      const int x = j < i ? __ldg(c.draft_ids + sp.first + j) : j > i ? -1 : greedy && has_row ? t.at : -1;
      if (j != i || kind == kNoDraw) c.token[base + j] = x;   // else it is drawn
      if (!c.logp) continue;
      if (j < i) {
        const Row p = ws.target_row[unit(j)];
        c.logp[base + j] = (float)(((double)load(c.target, base + j, x) - (double)p.m) * inv_tau - log(p.s));
      } else if (j > i) c.logp[base + j] = 0.f;
      else if (!has_row) c.logp[base + j] = __int_as_float(0x7fc00000);
      else if (greedy) c.logp[base + j] = (float)-log(t.s);
    }
    if (lane == 0) {
      const int x = i < sp.n ? __ldg(c.draft_ids + sp.first + i) : 0;
      c.n_emitted[r] = has_row ? i + 1 : i;
      unsigned int bad = has_row ? 0 : AF_DEVERR_DISTRIBUTION;
      if (good(t) && (x < 0 || x >= c.V)) bad |= AF_DEVERR_TARGET_RANGE;
      if (bad) atomicOr(d_err, bad);
      ws.draw[r] = Draw{base + i, kind, sp.first + i, x, t.m, q.m};
    }
  }
  if (kind != kDense) return;
  const int segments = shape.draw_slices * kDrawWarps;
  const int lo = segment_at(c.V, slice * kDrawWarps, segments), hi = segment_at(c.V, (slice + 1) * kDrawWarps, segments);
  const Exp64 pe = exp_about(s_power, t.m, inv_tau), qe = exp_about(s_power, q.m, inv_tau);
  double a = 0.0, b = 0.0;
  each_pair(row_of<T>(c.target, base + i), row_of<Q>(c.draft, sp.first + i), lo + (int)threadIdx.x, hi, kDrawThreads,
            [&](int, float z, float zq) { a += pe(z); b += qe(zq); });
  a = block_sum<kDrawWarps>(a, s_warp);
  b = block_sum<kDrawWarps>(b, s_warp);
  if (threadIdx.x == 0) ws.sums[(int64_t)r * shape.draw_slices + slice] = make_double2(a, b);
}

// Sums of a request's slices, by a warp, in a fixed order.
__device__ double2 slices_sum(const Workspace& ws, const Shape& shape, int r) {
  double2 a = make_double2(0.0, 0.0);
  for (int k = threadIdx.x & 31; k < shape.draw_slices; k += 32) {
    const double2 x = ws.sums[(int64_t)r * shape.draw_slices + k];
    a.x += x.x;
    a.y += x.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.x += __shfl_xor_sync(0xffffffffu, a.x, o);
    a.y += __shfl_xor_sync(0xffffffffu, a.y, o);
  }
  return a;
}
// The mass of a token in a draw.
template <class T, class Q>
struct Mass {
  const T* p;
  const Q* q;
  Exp64 pe, qe;
  double p_unit, q_unit;                                      // kDense: 1 / sums
  __device__ __forceinline__ Mass(const VerifyCall& c, const Draw& d, const double2& sums, const double* power, double inv_tau)
      : p(row_of<T>(c.target, d.row)), q(d.kind == kDense ? row_of<Q>(c.draft, d.draft_row) : nullptr), pe(exp_about(power, d.m, inv_tau)),
        qe(exp_about(power, d.m_draft, inv_tau)), p_unit(1.0 / sums.x), q_unit(1.0 / sums.y) {}
  __device__ __forceinline__ double left(float z, float zq) const { return fmax(pe(z) * p_unit - qe(zq) * q_unit, 0.0); }
};

// A warp per segment: its mass, and what the target has there.
template <class T, class Q>
__global__ void __launch_bounds__(kDrawThreads) verify_mass_kernel(const VerifyCall c, const Shape shape, const Workspace ws) {
  __shared__ double s_power[kPowers];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  set_powers(s_power);
  __syncthreads();
  wait_for_predecessor();
  let_successor_start();
  const int r = (int)blockIdx.x / shape.draw_slices, k = (int)blockIdx.x % shape.draw_slices * kDrawWarps + warp;
  const Draw d = ws.draw[r];
  if (d.kind == kNoDraw) return;
  const Mass<T, Q> mass(c, d, d.kind == kDense ? slices_sum(ws, shape, r) : make_double2(1.0, 1.0), s_power, inverse_temperature(c));
  const int segments = shape.draw_slices * kDrawWarps, lo = segment_at(c.V, k, segments), hi = segment_at(c.V, k + 1, segments);
  double a = 0.0, whole = 0.0;
  if (d.kind == kDense) {
    each_pair(mass.p, mass.q, lo + lane, hi, 32, [&](int, float z, float zq) { a += mass.left(z, zq); });
  } else {
    const auto take = [&](int, float z) { a += mass.pe(z); };
    const bool cuts = d.kind == kCut && d.cut >= lo && d.cut < hi;
    each(mass.p, lo + lane, cuts ? d.cut : hi, 32, take);
    if (cuts) each(mass.p, d.cut + 1 + lane, hi, 32, take);
    whole = a + (cuts && lane == 0 ? mass.pe(value(mass.p + d.cut)) : 0.0);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    whole += __shfl_xor_sync(0xffffffffu, whole, o);
  }
  if (lane == 0) ws.mass[(int64_t)r * segments + k] = make_double2(some_mass(a), whole);
}

// The token: the segment that holds the first v with C_v > u C, a part of it, and the place in that.
template <class T, class Q>
__global__ void __launch_bounds__(kFindThreads) verify_find_kernel(const VerifyCall c, const Shape shape, const Workspace ws) {
  __shared__ double s_power[kPowers], s_warp[kFindWarps], s_upto[kFindThreads];
  __shared__ double2 s_sums;
  __shared__ int s_found;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  set_powers(s_power);
  if (threadIdx.x == 0) s_found = 0;
  wait_for_predecessor();
  let_successor_start();
  const int r = (int)blockIdx.x;
  const Draw d = ws.draw[r];
  if (d.kind == kNoDraw) return;
  if (warp == 0) {
    const double2 x = d.kind == kDense ? slices_sum(ws, shape, r) : make_double2(1.0, 1.0);
    if (lane == 0) s_sums = x;
  }
  // running sums over the segments
  const int segments = shape.draw_slices * kDrawWarps, k = threadIdx.x;
  const double2 mine = k < segments ? ws.mass[(int64_t)r * segments + k] : make_double2(0.0, 0.0);
  double upto = mine.x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; ++w) upto += s_warp[w];
  s_upto[k] = upto;
  const double whole = block_sum<kFindWarps>(mine.y, s_warp);           // meets all threads
  double total = s_upto[kFindThreads - 1];
  const double row_sum = d.kind == kDense ? s_sums.x : whole;
  const Mass<T, Q> m(c, d, s_sums, s_power, inverse_temperature(c));
  // next to nothing is left of a residual: the target itself
  const bool plain = d.kind == kPlain || !((d.kind == kDense ? total : total / row_sum) > kResidualFloor);
  auto mass = [&](int v) {
    if (plain) return m.pe(value(m.p + v));
    if (d.kind == kDense) return m.left(value(m.p + v), value(m.q + v));
    return v == d.cut ? 0.0 : m.pe(value(m.p + v));
  };
  const double u = (double)fminf(fmaxf(__ldg(c.u_sample + r), 0.f), 1.f - 0x1p-24f);
  int lo = 0, hi = c.V;
  double start = 0.0, goal = 0.0;
  const bool afresh = plain && d.kind != kPlain;              // the segments' mass is of the residual
  if (!afresh) {
    goal = u * total;
    // the last segment with mass that starts at or before the goal
    if (mine.x > 0.0 && (k == 0 ? 0.0 : s_upto[k - 1]) <= goal) atomicMax(&s_found, k);
    __syncthreads();
    const int f = s_found;
    start = f == 0 ? 0.0 : s_upto[f - 1];
    lo = segment_at(c.V, f, segments);
    hi = segment_at(c.V, f + 1, segments);
  }
  // all warps share the stretch out, and one's part is the next stretch
  for (bool first = true;; first = false) {
    const int n = hi - lo;
    auto part = [&](int w) { return lo + (int)((int64_t)n * w / kFindWarps); };
    double a = 0.0;
    const int end = part(warp + 1);
#pragma unroll 4
    for (int v = part(warp) + lane; v < end; v += 32) a += mass(v);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    __syncthreads();
    if (lane == 0) s_warp[warp] = some_mass(a);
    __syncthreads();
    if (afresh && first) {
      double all = 0.0;
      for (int w = 0; w < kFindWarps; ++w) all += s_warp[w];
      goal = u * all;
    }
    double run = start;
    int found = 0;                                            // the last part with mass that starts at or before the goal
    for (int w = 0; w < kFindWarps; ++w) {
      if (run <= goal && s_warp[w] > 0.0) { found = w; start = run; }
      run += s_warp[w];
    }
    const int next_lo = part(found);
    hi = part(found + 1);
    lo = next_lo;
    if (hi - lo <= 128) break;
  }
  if (warp != 0) return;
  int y = lo;                                                 // the last with mass, if rounding leaves the goal beyond the part
  for (int v0 = lo; v0 < hi; v0 += 32) {
    const int v = v0 + lane;
    const double w = v < hi ? mass(v) : 0.0;
    double upto_lane = w;                                     // sum over the lanes up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double x = __shfl_up_sync(0xffffffffu, upto_lane, o);
      if (lane >= o) upto_lane += x;
    }
    const unsigned some = __ballot_sync(0xffffffffu, w > kNothing), beyond = __ballot_sync(0xffffffffu, w > kNothing && start + upto_lane > goal);
    if (beyond) { y = v0 + __ffs(beyond) - 1; break; }
    if (some) y = v0 + 31 - __clz(some);
    start += __shfl_sync(0xffffffffu, upto_lane, 31);
  }
  if (lane == 0) {
    // in the tokens' row of the request's: rows of the target and of the tokens are the same
    c.token[d.row] = y;
    if (c.logp) c.logp[d.row] = (float)(((double)value(m.p + y) - (double)d.m) * inverse_temperature(c) - log(row_sum));
  }
}

// Slices of a row.  A batch of rows that fills the device several times over goes row by row, so that positions end in order;
// fewer are cut until every SM has about four slices, of 2048 logits at least.
Shape shape_of(int32_t R, int32_t V, int32_t max_draft, int sm_count) {
  const int64_t units = (int64_t)R * (max_draft + 1), want = ((int64_t)sm_count * 4 + units - 1) / units, most = V / 2048;
  const int64_t slices = want < most ? want : most;
  // a draw's slices: a few to an SM, of 1024 logits at least
  int64_t draw = ((int64_t)sm_count * 8 + R - 1) / R;
  if (draw > V / 1024) draw = V / 1024;
  if (draw > kMostSlices) draw = kMostSlices;
  return {(int)(slices < 1 ? 1 : slices), max_draft + 1, (int)(draw < 1 ? 1 : draw)};
}
template <class T, class Q>
af_status launch_draws(const VerifyCall& c, Shape shape, const Workspace& ws, unsigned int* d_err, cudaStream_t s) {
  const bool greedy = c.temperature == 0.f;
  if (greedy) shape.draw_slices = 1;
  const unsigned slices = (unsigned)c.R * shape.draw_slices;
  if (launch_overlapped(verify_sums_kernel<T, Q>, slices, kDrawThreads, 0, s, c, shape, ws, d_err) != cudaSuccess) return AF_ERR_CUDA;
  if (greedy) return AF_OK;
  if (launch_overlapped(verify_mass_kernel<T, Q>, slices, kDrawThreads, 0, s, c, shape, ws) != cudaSuccess) return AF_ERR_CUDA;
  return launch_overlapped(verify_find_kernel<T, Q>, (unsigned)c.R, kFindThreads, 0, s, c, shape, ws) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }
struct Sizes { size_t parts, rows, draws, sums, mass, verdicts, tickets, stops; };
// Rows in several slices are few: fewer than 8 parts per SM in all, and as many of the drafts; and parts and tickets are used
// only there.  A draw's slices are 8 per SM and one per request at most.  So smaller calls of any kind fit in what a larger one
// needs.
Sizes sizes_of(int32_t R, int32_t max_draft, int sm_count) {
  const size_t units = (size_t)R * ((size_t)max_draft + 1), slices = (size_t)sm_count * 8 + R;
  return {(size_t)sm_count * 16 * sizeof(RowPart), units * 2 * sizeof(Row), (size_t)R * sizeof(Draw), slices * sizeof(double2),
          slices * kDrawWarps * sizeof(double2), units * sizeof(int32_t), round16((size_t)sm_count * 4 * sizeof(unsigned int)),
          (size_t)R * sizeof(int)};
}
static_assert(sizeof(Draw) % 16 == 0 && sizeof(Row) % 16 == 0, "what lies behind them is aligned");

}  // namespace

// Sizes the workspace; what a call leaves as it found it, the tickets and the stops, is set where the memory is new.
af_status reserve_draft_verify(af_ctx* ctx, int32_t R, int32_t max_draft, cudaStream_t s) {
  const Sizes z = sizes_of(R, max_draft, ctx->sm_count);
  af_status st = ws_grow(ctx->verify_ws, z.parts + z.rows + z.draws + z.sums + z.mass + z.verdicts);
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
  char* at = static_cast<char*>(ctx->verify_ws.p);
  auto take = [&](size_t bytes) { char* const p = at; at += bytes; return p; };
  ws.target = reinterpret_cast<RowPart*>(take(z.parts));
  ws.draft = ws.target + (size_t)c.R * shape.positions * shape.slices;
  ws.target_row = reinterpret_cast<Row*>(take(z.rows));
  ws.draft_row = ws.target_row + (size_t)c.R * shape.positions;
  ws.draw = reinterpret_cast<Draw*>(take(z.draws));
  ws.sums = reinterpret_cast<double2*>(take(z.sums));
  ws.mass = reinterpret_cast<double2*>(take(z.mass));
  ws.verdict = reinterpret_cast<int32_t*>(take(z.verdicts));
  ws.ticket = static_cast<unsigned int*>(ctx->verify_state.p);
  ws.stop = reinterpret_cast<int*>(static_cast<char*>(ctx->verify_state.p) + z.tickets);
  const float scale = c.temperature == 0.f ? kLog2e : kLog2e / c.temperature;
  const int64_t blocks = (int64_t)c.R * shape.positions * shape.slices;
  if (launch_overlapped(verify_rows_kernel, (unsigned)blocks, kRowThreads, 0, s, c, shape, scale, 2.f / scale, ws) != cudaSuccess) return AF_ERR_CUDA;
  const bool wide_draft = !c.draft.p || c.draft.type == AF_F32;
  using bf16 = __nv_bfloat16;
  if (c.target.type == AF_F32)
    return wide_draft ? launch_draws<float, float>(c, shape, ws, ctx->d_err, s) : launch_draws<float, bf16>(c, shape, ws, ctx->d_err, s);
  return wide_draft ? launch_draws<bf16, float>(c, shape, ws, ctx->d_err, s) : launch_draws<bf16, bf16>(c, shape, ws, ctx->d_err, s);
}

}  // namespace af
