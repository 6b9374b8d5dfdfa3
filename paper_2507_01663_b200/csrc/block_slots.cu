// af_block_slots: block tables and the rows of new tokens of a paged store, from the requests' lengths.
//
// A plan first (one CTA): what every request gives back and wants, as running sums over the requests, and who gets it.
// Then everything that the sums determine, item by item and in any order: rows of tokens, table entries of new
// blocks, free-list entries of blocks given back.  Blocks given back in a call serve the same call: the k-th wanted one
// comes from place available - 1 - k of the stack, and a place that this call would have pushed is looked up in the
// table it comes from, so nothing that is written here is read here.  Whole numbers only: the answer is unique.
//
// A decoding step (1024 requests at most) is one launch of one CTA, all latency: loads, one scan, searches in shared memory.
// A larger batch takes two; in the second a CTA takes 2048 neighbouring tokens, whose requests are few, and a thread
// eight of them, which lie in one or two blocks, so that most of the work is to write 12 bytes for each.  4096 requests of 1.1
// million tokens: 20.5 us, the plan 11 and the rest 18 when each runs alone and cold; 64 requests of 5 tokens: 4-6 us.
#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

// One request's share of the plan.  wanted_at: blocks wanted by the requests before it; kMost stands for all from there up, which
// no place of a stack of less than 2^31 blocks reaches.
struct alignas(16) Request {
  int32_t held, need;            // blocks of its table before, and with the new tokens
  int32_t length;                // tokens kept, -1: the request is refused
  int32_t wanted_at;
};
struct Totals {
  int64_t available, count, given, taken, tokens;   // taken: blocks that leave the stack
};
struct Plan {
  Totals* totals;
  Request* request;              // [R]
  int32_t* given_at;             // [R] blocks given back by the requests before it
  int32_t* wanted_at;            // [R] once more, close together for the searches
};
constexpr int kPlanThreads = 1024, kPlanEach = 4;            // of a larger batch: threads, neighbouring requests of each
constexpr int kStepThreads = 1024;                           // of a step, each with one request
constexpr int kFewThreads = 256;                             // of a smaller one
constexpr int kFewTokens = 512, kStepTokens = 8192;          // of a step, at most
constexpr int kTokenThreads = 256, kTokenEach = 8, kTokenTile = kTokenThreads * kTokenEach;
constexpr int kCached = 1024;                                // running token sums that a tile keeps in shared memory
constexpr int kMarks = 4096;                                 // running block sums that it keeps there, evenly apart
constexpr int64_t kMost = 0x7fffffff;

struct Sums { int64_t tokens, given, wanted; };
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return {a.tokens + b.tokens, a.given + b.given, a.wanted + b.wanted};
}
__device__ __forceinline__ Sums shfl_up(const Sums& a, int o) {
  return {__shfl_up_sync(0xffffffffu, a.tokens, o), __shfl_up_sync(0xffffffffu, a.given, o), __shfl_up_sync(0xffffffffu, a.wanted, o)};
}
__device__ __forceinline__ Sums shfl(const Sums& a, int from) {
  return {__shfl_sync(0xffffffffu, a.tokens, from), __shfl_sync(0xffffffffu, a.given, from), __shfl_sync(0xffffffffu, a.wanted, from)};
}
// Sum over the threads before this one (exclusive), and over all of them.  Every thread of the block calls it.
template <int kThreads>
__device__ __forceinline__ Sums scan(Sums mine, Sums* total, Sums* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums up = shfl_up(run, o);
    if (lane >= o) run = run + up;
  }
  __syncthreads();                                           // warp_sums of a scan before
  if (lane == 31) warp_sums[warp] = run;
  __syncthreads();
  constexpr int warps = kThreads / 32;
  Sums upto = lane < warps ? warp_sums[lane] : Sums{0, 0, 0};
#pragma unroll
  for (int o = 1; o < warps; o <<= 1) {
    const Sums up = shfl_up(upto, o);
    if (lane >= o) upto = upto + up;
  }
  *total = shfl(upto, warps - 1);
  const Sums before = shfl(upto, warp == 0 ? 0 : warp - 1);
  const int64_t any = warp == 0 ? 0 : -1;
  return {(before.tokens & any) + run.tokens - mine.tokens, (before.given & any) + run.given - mine.given,
          (before.wanted & any) + run.wanted - mine.wanted};
}

// Block sizes are often powers of two.
struct BlockSize {
  int32_t n, shift;                                          // shift: -1 if n is no power of two
  __device__ __forceinline__ explicit BlockSize(int32_t size) {
    n = size;
    shift = (size & (size - 1)) == 0 ? 31 - __clz(size) : -1;
  }
  __device__ __forceinline__ int32_t of(uint32_t pos) const { return (int32_t)(shift >= 0 ? pos >> shift : pos / (uint32_t)n); }
};
__device__ __forceinline__ int32_t clamped(int64_t x) { return (int32_t)(x < kMost ? x : kMost); }

// x[at .. at + kEach) of n, 0 behind the end; four at a time where the address allows it.
template <int kEach>
__device__ __forceinline__ void get(const int32_t* x, int at, int n, int32_t (&out)[kEach]) {
  if (kEach == 4 && at + 4 <= n && (reinterpret_cast<uintptr_t>(x) & 15) == 0) {
    *reinterpret_cast<int4*>(out) = *reinterpret_cast<const int4*>(x + at);
  } else {
#pragma unroll
    for (int k = 0; k < kEach; ++k) out[k] = at + k < n ? x[at + k] : 0;
  }
}
template <int kEach>
__device__ __forceinline__ void put(int32_t* x, int at, int n, const int32_t (&in)[kEach]) {
  if (kEach == 4 && at + 4 <= n && (reinterpret_cast<uintptr_t>(x) & 15) == 0) {
    *reinterpret_cast<int4*>(x + at) = *reinterpret_cast<const int4*>(in);
  } else {
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (at + k < n) x[at + k] = in[k];
  }
}

struct Wish { int32_t tokens, held, need, length; bool valid; };

// cu (nullable): also receives the running token sums, R + 1 of them.  Every thread of the CTA calls it; what it writes to shared
// memory or to the plan can be read by the CTA after it.
template <int kThreads, int kEach>
__device__ __forceinline__ Totals make_plan(const SlotsCall& c, const Plan& plan, int32_t* cu, unsigned int* d_err) {
  __shared__ Sums warp_sums[32];
  __shared__ unsigned int most;
  const BlockSize size(c.block_size);
  const int64_t room = (int64_t)c.max_blocks * c.block_size;
  if (threadIdx.x == 0) most = 0;
  unsigned int bad = 0;
  Wish w[kEach];
  auto wishes = [&](int r0) {
    alignas(16) int32_t length[kEach], held[kEach], grow[kEach];
    const int r = r0 + (int)threadIdx.x * kEach;
    get(c.length, r, c.R, length);
    get(c.held, r, c.R, held);
    get(c.grow, r, c.R, grow);
    Sums mine{0, 0, 0};
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      w[k].length = length[k];
      w[k].held = held[k];
      const int64_t end = (int64_t)w[k].length + grow[k];
      w[k].tokens = grow[k] > 0 ? grow[k] : 0;
      w[k].valid = w[k].length >= 0 && grow[k] >= 0 && w[k].held >= 0 && w[k].held <= c.max_blocks && end <= kMost && end <= room;
      w[k].need = w[k].valid ? size.of((uint32_t)end + (uint32_t)(c.block_size - 1)) : w[k].held;
      mine.tokens += w[k].tokens;
      const int64_t more = (int64_t)w[k].need - w[k].held;
      if (more < 0) mine.given -= more; else mine.wanted += more;
    }
    return mine;
  };
  int64_t count = *c.free_count;
  int64_t given = 0;
  Sums mine{}, all{}, at{};
  for (int r0 = 0; r0 < c.R; r0 += kThreads * kEach) {       // what comes back, before anything is promised
    mine = wishes(r0);
    at = scan<kThreads>(mine, &all, warp_sums);
    given += all.given;
  }
  if (count < 0 || count > c.n_blocks) { bad |= AF_DEVERR_REQUEST; count = count < 0 ? 0 : c.n_blocks; }
  int64_t available = count + given;
  if (available > c.n_blocks) { bad |= AF_DEVERR_REQUEST; available = c.n_blocks; }
  Sums before{0, 0, 0};
  unsigned int taken = 0;
  for (int r0 = 0; r0 < c.R; r0 += kThreads * kEach) {
    if (c.R > kThreads * kEach) {                            // else all is still at hand
      mine = wishes(r0);
      at = scan<kThreads>(mine, &all, warp_sums);
    }
    Sums here = before + at;
    before = before + all;
    const int r = r0 + (int)threadIdx.x * kEach;
    alignas(16) int32_t given_at[kEach], wanted_at[kEach], held_out[kEach], granted[kEach], first[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t more = (int64_t)w[k].need - w[k].held;
      const bool yes = w[k].valid && (more <= 0 || here.wanted + more <= available);
      if (!w[k].valid) bad |= AF_DEVERR_REQUEST;
      else if (!yes) bad |= AF_DEVERR_BLOCKS;
      given_at[k] = clamped(here.given);
      wanted_at[k] = clamped(here.wanted);
      held_out[k] = yes ? w[k].need : w[k].held;
      granted[k] = yes;
      first[k] = clamped(here.tokens);
      if (r + k < c.R) plan.request[r + k] = Request{w[k].held, w[k].need, yes ? w[k].length : -1, wanted_at[k]};
      // granted requests come first among those that want blocks: what they take is the largest of their ends
      if (yes && more > 0) taken = (unsigned int)(here.wanted + more);
      here = here + Sums{w[k].tokens, more < 0 ? -more : 0, more > 0 ? more : 0};
    }
    put(plan.given_at, r, c.R, given_at);
    put(plan.wanted_at, r, c.R, wanted_at);
    put(c.held_out, r, c.R, held_out);
    if (c.granted) put(c.granted, r, c.R, granted);
    put(c.cu, r, c.R, first);
    if (cu) put(cu, r, c.R, first);
  }
  __syncthreads();                                           // most is 0
  taken = __reduce_max_sync(0xffffffffu, taken);
  if ((threadIdx.x & 31) == 0 && taken > 0) atomicMax(&most, taken);
  if (bad) atomicOr(d_err, bad);
  __syncthreads();
  const Totals t{available, count, given, most, before.tokens};
  if (threadIdx.x == 0) {
    if (t.tokens > c.capacity || t.tokens > kMost) atomicOr(d_err, AF_DEVERR_REQUEST);
    c.cu[c.R] = clamped(t.tokens);
    if (cu) cu[c.R] = clamped(t.tokens);
    *c.free_count_out = (int32_t)(available - t.taken);
  }
  return t;
}

// The largest r in [lo, hi) with key[r] <= x (non-decreasing, key[lo] <= x).
__device__ __forceinline__ int search(const int32_t* key, int lo, int hi, int64_t x) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int64_t)key[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}
// The same by a warp, 32 probes at a time.
__device__ __forceinline__ int search_by_warp(const int32_t* key, int n, int64_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, probe = lo + ((threadIdx.x & 31) + 1) * step;
    lo += step * __popc(__ballot_sync(0xffffffffu, probe < hi && key[probe] <= x));
    hi = min(lo + step, hi);
  }
  return lo;
}
// Running sums over the requests, every 2^shift-th of them in shared memory.
struct Running {
  const int32_t *all, *marks;
  int R, shift;
  __device__ __forceinline__ int find(int64_t x) const {
    const int n = ((R - 1) >> shift) + 1, at = search(marks, 0, n, x) << shift;
    return shift == 0 ? at : search(all, at, min(at + (1 << shift), R), x);
  }
};
struct Taken {                                               // what a thread needs to know of the plan to carry it out
  const SlotsCall& c;
  const Request* request;
  Totals t;
  Running given, wanted;
  // The block at place a >= count of the stack: one that this call gives back.
  __device__ __forceinline__ int32_t given_block(int64_t back) const {
    const int r = given.find(back);
    const int64_t column = request[r].need + back - given.all[r];
    return column < c.max_blocks ? c.table[r * c.table_pitch + column] : -1;
  }
  __device__ __forceinline__ int32_t wanted_block(int64_t k) const {
    const int64_t place = t.available - 1 - k;
    return place < t.count ? c.free_blocks[place] : given_block(place - t.count);
  }
  __device__ __forceinline__ int32_t block_of(const Request& q, int r, int32_t column) const {
    return column < q.held ? c.table[r * c.table_pitch + column] : wanted_block((int64_t)q.wanted_at + column - q.held);
  }
  // Table entries of new blocks, and free-list entries of blocks given back.
  __device__ __forceinline__ void move_blocks(int64_t thread, int64_t threads) const {
    for (int64_t k = thread; k < t.taken; k += threads) {
      const int r = wanted.find(k);
      const Request q = request[r];
      c.table[r * c.table_pitch + q.held + (k - q.wanted_at)] = wanted_block(k);
    }
    const int64_t left = t.available - t.taken;
    for (int64_t p = t.count + thread; p < left; p += threads) c.free_blocks[p] = given_block(p - t.count);
  }
};
__device__ __forceinline__ int64_t tokens_of(const SlotsCall& c, const Totals& t) {
  const int64_t n = t.tokens < kMost ? t.tokens : kMost;
  return n < c.capacity ? n : c.capacity;
}

// All of a batch of at most kThreads requests.
template <int kThreads>
__global__ void __launch_bounds__(kThreads) slots_step_kernel(const SlotsCall c, unsigned int* d_err) {
  __shared__ Request request[kThreads];
  __shared__ int32_t given_at[kThreads], wanted_at[kThreads], cu[kThreads + 1];
  wait_for_predecessor();
  let_successor_start();
  const Totals t = make_plan<kThreads, 1>(c, Plan{nullptr, request, given_at, wanted_at}, cu, d_err);
  __syncthreads();
  const Taken plan{c, request, t, {given_at, given_at, c.R, 0}, {wanted_at, wanted_at, c.R, 0}};
  const BlockSize size(c.block_size);
  const int64_t n = tokens_of(c, t);
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const int r = search(cu, 0, c.R, i);
    const Request q = request[r];
    int64_t row = -1;
    int32_t pos = (int32_t)(i - cu[r]);
    if (q.length >= 0) {
      pos += q.length;
      const int32_t column = size.of(pos);
      row = (int64_t)plan.block_of(q, r, column) * size.n + (pos - column * size.n);
    } else {
      pos = (int32_t)((int64_t)c.length[r] + pos);
    }
    c.slot[i] = row;
    if (c.position) c.position[i] = pos;
  }
  plan.move_blocks(threadIdx.x, kThreads);
}

__global__ void __launch_bounds__(kPlanThreads) slots_plan_kernel(const SlotsCall c, const Plan plan, unsigned int* d_err) {
  wait_for_predecessor();
  let_successor_start();
  const Totals t = make_plan<kPlanThreads, kPlanEach>(c, plan, nullptr, d_err);
  if (threadIdx.x == 0) *plan.totals = t;
}

template <class T>
__device__ __forceinline__ void store_eight(T* to, const T (&x)[kTokenEach], int n) {
  if (n == kTokenEach && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
    uint4 v[sizeof(x) / 16];
    memcpy(v, x, sizeof(x));
#pragma unroll
    for (int k = 0; k < (int)(sizeof(x) / 16); ++k) reinterpret_cast<uint4*>(to)[k] = v[k];
  } else {
#pragma unroll
    for (int k = 0; k < kTokenEach; ++k)
      if (k < n) to[k] = x[k];
  }
}
__global__ void __launch_bounds__(kTokenThreads) slots_carry_out_kernel(const SlotsCall c, const Plan at) {
  __shared__ int32_t s_cu[kCached + 1], s_given[kMarks], s_wanted[kMarks];
  __shared__ int s_ends[2];
  wait_for_predecessor();
  let_successor_start();
  const Totals t = *at.totals;
  const int64_t n = tokens_of(c, t), tiles = (n + kTokenTile - 1) / kTokenTile;
  int shift = 0;
  while (((c.R - 1) >> shift) >= kMarks) ++shift;
  const int marks = ((c.R - 1) >> shift) + 1;
  if (t.taken > 0) {
    for (int k = threadIdx.x; k < marks; k += kTokenThreads) s_wanted[k] = at.wanted_at[k << shift];
    if (t.given > 0)
      for (int k = threadIdx.x; k < marks; k += kTokenThreads) s_given[k] = at.given_at[k << shift];
  } else if (t.given > 0) {
    for (int k = threadIdx.x; k < marks; k += kTokenThreads) s_given[k] = at.given_at[k << shift];
  }
  const Taken plan{c, at.request, t, {at.given_at, s_given, c.R, shift}, {at.wanted_at, s_wanted, c.R, shift}};
  const BlockSize size(c.block_size);
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t i0 = tile * kTokenTile, i1 = min(i0 + kTokenTile, n);
    __syncthreads();                                         // s_cu of the tile before
    if (threadIdx.x < 64) {                                  // the requests of the first and of the last token, a warp each
      const int r = search_by_warp(c.cu, c.R, threadIdx.x < 32 ? i0 : i1 - 1);
      if ((threadIdx.x & 31) == 0) s_ends[threadIdx.x >> 5] = r;
    }
    __syncthreads();
    const int r0 = s_ends[0], m = s_ends[1] - r0 + 1;        // m is large only where most requests have no token
    if (m <= kCached) {
      for (int k = threadIdx.x; k <= m; k += kTokenThreads) s_cu[k] = c.cu[r0 + k];
      __syncthreads();
    }
    const int32_t* const cu = m <= kCached ? s_cu : c.cu + r0;
    const int64_t first = i0 + threadIdx.x * kTokenEach;
    if (first >= i1) continue;
    int r = search(cu, 0, m, first);
    Request q = at.request[r0 + r];
    int64_t rows[kTokenEach];
    int32_t positions[kTokenEach];
    int32_t column = -1;
    int64_t block = -1;
#pragma unroll
    for (int k = 0; k < kTokenEach; ++k) {
      const int64_t i = first + k;
      rows[k] = -1;
      positions[k] = 0;
      if (i >= i1) continue;
      if (i >= cu[r + 1]) {
        do ++r; while (i >= cu[r + 1]);
        q = at.request[r0 + r];
        column = -1;
      }
      int32_t pos = (int32_t)(i - cu[r]);
      if (q.length >= 0) {
        pos += q.length;
        const int32_t here = size.of(pos);
        if (here != column) {
          column = here;
          block = plan.block_of(q, r0 + r, column);
        }
        rows[k] = block * size.n + (pos - column * size.n);
      } else {
        pos = (int32_t)((int64_t)c.length[r0 + r] + pos);
      }
      positions[k] = pos;
    }
    const int count = (int)min((int64_t)kTokenEach, i1 - first);
    store_eight(c.slot + first, rows, count);
    if (c.position) store_eight(c.position + first, positions, count);
  }
  __syncthreads();                                           // the marks, where there is no token
  plan.move_blocks((int64_t)blockIdx.x * kTokenThreads + threadIdx.x, (int64_t)gridDim.x * kTokenThreads);
}

}  // namespace

size_t slots_workspace_bytes(int32_t R) { return (sizeof(Totals) + 15) / 16 * 16 + (size_t)R * (sizeof(Request) + 2 * sizeof(int32_t)) + 32; }

af_status launch_block_slots(af_ctx* ctx, const SlotsCall& c, cudaStream_t s) {
  // One CTA, whose work grows with the tokens, or two launches of about 12 us together.  On the device, 256 threads / 1024 / two
  // launches: 64 requests of 5 tokens 4.0 / 4.9 / 14.2 us, of 16 5.2 / 4.9 / 12.1; 256 of 32 28.5 / 12.7 / 12.3; 1024 of 1
  // - / 5.9 / 15.7, of 8 - / 14.2 / 13.1, of 16 - / 23.5 / 12.9.
  if (c.R <= kFewThreads && c.capacity <= kFewTokens)
    return launch_overlapped(slots_step_kernel<kFewThreads>, 1, kFewThreads, 0, s, c, ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
  if (c.R <= kStepThreads && c.capacity <= kStepTokens)
    return launch_overlapped(slots_step_kernel<kStepThreads>, 1, kStepThreads, 0, s, c, ctx->d_err) == cudaSuccess ? AF_OK
                                                                                                                    : AF_ERR_CUDA;
  const af_status st = ws_grow(ctx->slots_ws, slots_workspace_bytes(c.R));
  if (st != AF_OK) return st;
  Plan plan;
  plan.totals = static_cast<Totals*>(ctx->slots_ws.p);
  plan.request = reinterpret_cast<Request*>(static_cast<char*>(ctx->slots_ws.p) + (sizeof(Totals) + 15) / 16 * 16);
  plan.given_at = reinterpret_cast<int32_t*>(plan.request + c.R);
  plan.wanted_at = plan.given_at + (c.R + 3) / 4 * 4;
  if (launch_overlapped(slots_plan_kernel, 1, kPlanThreads, 0, s, c, plan, ctx->d_err) != cudaSuccess) return AF_ERR_CUDA;
  int64_t tiles = (c.capacity + kTokenTile - 1) / kTokenTile;
  const int64_t most = (int64_t)ctx->sm_count * 6, least = (c.R + 63) / 64 < ctx->sm_count ? (c.R + 63) / 64 : ctx->sm_count;
  tiles = tiles < least ? least : tiles;
  return launch_overlapped(slots_carry_out_kernel, (int)(tiles < most ? tiles : most), kTokenThreads, 0, s, c, plan) == cudaSuccess
             ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
