// af_block_slots: block tables and the rows of new tokens of a paged store, from the requests' lengths.
//
// A plan first (one CTA): what every request gives back and wants, as running sums over the requests, and who gets it.
// Then everything that the sums determine, item by item and in any order: rows of tokens, table entries of new
// blocks, free-list entries of blocks given back.  Blocks given back in a call serve the same call: the k-th wanted one
// comes from place available - 1 - k of the stack, and a place that this call would have pushed is looked up in the
// table it comes from, so nothing that is written here is read here.  Whole numbers only: the answer is unique.
#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

struct Request {                 // one request's share of the plan
  int64_t given_at, wanted_at;   // blocks given back / wanted by the requests before it
  int32_t held, need;            // blocks of its table before, and with the new tokens
  int32_t length;                // tokens kept, -1: the request is refused
  int32_t pad;
};
struct Totals {
  int64_t available, count, given, taken, tokens;   // taken: blocks that leave the stack
};
constexpr int kPlanThreads = 1024;
constexpr int64_t kMostTokens = 0x7fffffff;

struct Sums { int64_t tokens, given, wanted; };
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return {a.tokens + b.tokens, a.given + b.given, a.wanted + b.wanted};
}
__device__ __forceinline__ Sums shfl_up(const Sums& a, int o) {
  return {__shfl_up_sync(0xffffffffu, a.tokens, o), __shfl_up_sync(0xffffffffu, a.given, o), __shfl_up_sync(0xffffffffu, a.wanted, o)};
}
// Sum over the threads before this one (exclusive), and over all of them.  Every thread of the block calls it.
__device__ Sums scan(Sums mine, Sums* total, Sums* warp_sums) {
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
  Sums before{0, 0, 0}, all{0, 0, 0};
  for (int w = 0; w < (int)blockDim.x / 32; ++w) {
    if (w < warp) before = before + warp_sums[w];
    all = all + warp_sums[w];
  }
  *total = all;
  return {before.tokens + run.tokens - mine.tokens, before.given + run.given - mine.given, before.wanted + run.wanted - mine.wanted};
}

struct Wish { int64_t tokens; int32_t held, need, length; bool valid; };
__device__ __forceinline__ Wish wish(const SlotsCall& c, int r) {
  const int32_t length = c.length[r], grow = c.grow[r], held = c.held[r];
  const int64_t end = (int64_t)length + grow;
  Wish w;
  w.tokens = grow > 0 ? grow : 0;
  w.valid = length >= 0 && grow >= 0 && held >= 0 && held <= c.max_blocks && end <= kMostTokens &&
            end <= (int64_t)c.max_blocks * c.block_size;
  w.held = held;
  w.need = w.valid ? (int32_t)((end + c.block_size - 1) / c.block_size) : held;
  w.length = length;
  return w;
}

__device__ void plan(const SlotsCall& c, Request* req, Totals* totals, unsigned int* d_err) {
  __shared__ Sums warp_sums[kPlanThreads / 32];
  unsigned int bad = 0;
  int64_t given = 0;
  for (int r0 = 0; r0 < c.R; r0 += blockDim.x) {             // what comes back, before anything is promised
    const int r = r0 + threadIdx.x;
    Sums mine{0, 0, 0}, all;
    if (r < c.R) {
      const Wish w = wish(c, r);
      if (w.need < w.held) mine.given = w.held - w.need;
    }
    scan(mine, &all, warp_sums);
    given += all.given;
  }
  int64_t count = *c.free_count;
  if (count < 0 || count > c.n_blocks) { bad |= AF_DEVERR_REQUEST; count = count < 0 ? 0 : c.n_blocks; }
  int64_t available = count + given;
  if (available > c.n_blocks) { bad |= AF_DEVERR_REQUEST; available = c.n_blocks; }
  Sums before{0, 0, 0};
  int64_t taken = 0;
  for (int r0 = 0; r0 < c.R; r0 += blockDim.x) {
    const int r = r0 + threadIdx.x;
    Sums mine{0, 0, 0}, all;
    Wish w{};
    if (r < c.R) {
      w = wish(c, r);
      mine.tokens = w.tokens;
      if (w.need < w.held) mine.given = w.held - w.need; else mine.wanted = w.need - w.held;
    }
    const Sums at = before + scan(mine, &all, warp_sums);
    before = before + all;
    if (r < c.R) {
      const bool granted = w.valid && (mine.wanted == 0 || at.wanted + mine.wanted <= available);
      if (!w.valid) bad |= AF_DEVERR_REQUEST;
      else if (!granted) bad |= AF_DEVERR_BLOCKS;
      req[r] = Request{at.given, at.wanted, w.held, w.need, granted ? w.length : -1, 0};
      c.held_out[r] = granted ? w.need : w.held;
      if (c.granted) c.granted[r] = granted;
      c.cu[r] = (int32_t)(at.tokens < kMostTokens ? at.tokens : kMostTokens);
      if (granted && mine.wanted > 0 && at.wanted + mine.wanted > taken) taken = at.wanted + mine.wanted;
    }
  }
  // granted requests come first among those that want blocks: what they take is the largest of their ends
  __shared__ unsigned long long most;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  atomicMax(&most, (unsigned long long)taken);
  if (bad) atomicOr(d_err, bad);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (before.tokens > c.capacity || before.tokens > kMostTokens) atomicOr(d_err, AF_DEVERR_REQUEST);
    c.cu[c.R] = (int32_t)(before.tokens < kMostTokens ? before.tokens : kMostTokens);
    *totals = Totals{available, count, given, (int64_t)most, before.tokens};
    *c.free_count_out = (int32_t)(available - (int64_t)most);
  }
}

// The largest r with key(r) <= x (key non-decreasing, key(0) <= x).
template <class Key>
__device__ __forceinline__ int search(int R, int64_t x, Key key) {
  int lo = 0, hi = R;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (key(mid) <= x) lo = mid; else hi = mid;
  }
  return lo;
}
// The block at place a >= count of the stack: one that this call gives back.
__device__ __forceinline__ int32_t given_block(const SlotsCall& c, const Request* req, int64_t back) {
  const int r = search(c.R, back, [&](int i) { return __ldcg(&req[i].given_at); });
  const int64_t column = __ldcg(&req[r].need) + back - __ldcg(&req[r].given_at);
  return column < c.max_blocks ? c.table[r * c.table_pitch + column] : -1;
}
__device__ __forceinline__ int32_t wanted_block(const SlotsCall& c, const Request* req, const Totals& t, int64_t k) {
  const int64_t place = t.available - 1 - k;
  return place < t.count ? c.free_blocks[place] : given_block(c, req, place - t.count);
}

__device__ void carry_out(const SlotsCall& c, const Request* req, const Totals* totals, int64_t thread, int64_t threads) {
  const Totals t{__ldcg(&totals->available), __ldcg(&totals->count), __ldcg(&totals->given), __ldcg(&totals->taken),
                 __ldcg(&totals->tokens)};
  const int64_t tokens = t.tokens < c.capacity ? (t.tokens < kMostTokens ? t.tokens : kMostTokens) : c.capacity;
  for (int64_t i = thread; i < tokens; i += threads) {       // rows of the new tokens
    const int r = search(c.R, i, [&](int j) { return (int64_t)__ldcg(c.cu + j); });
    const int32_t length = __ldcg(&req[r].length), held = __ldcg(&req[r].held);
    int64_t row = -1;
    const int64_t in = i - __ldcg(c.cu + r);
    const int32_t pos = (int32_t)((int64_t)c.length[r] + in);
    if (length >= 0) {
      const int32_t column = pos / c.block_size;
      const int32_t block = column < held ? c.table[r * c.table_pitch + column]
                                          : wanted_block(c, req, t, __ldcg(&req[r].wanted_at) + column - held);
      row = (int64_t)block * c.block_size + pos % c.block_size;
    }
    c.slot[i] = row;
    if (c.position) c.position[i] = pos;
  }
  for (int64_t k = thread; k < t.taken; k += threads) {      // table entries of the new blocks
    const int r = search(c.R, k, [&](int j) { return __ldcg(&req[j].wanted_at); });
    const int64_t column = __ldcg(&req[r].held) + k - __ldcg(&req[r].wanted_at);
    c.table[r * c.table_pitch + column] = wanted_block(c, req, t, k);
  }
  const int64_t left = t.available - t.taken;
  for (int64_t p = t.count + thread; p < left; p += threads) c.free_blocks[p] = given_block(c, req, p - t.count);
}

__global__ void __launch_bounds__(kPlanThreads) slots_plan_kernel(const SlotsCall c, Request* req, Totals* totals, unsigned int* d_err) {
  wait_for_predecessor();
  let_successor_start();
  plan(c, req, totals, d_err);
}
__global__ void __launch_bounds__(256) slots_carry_out_kernel(const SlotsCall c, const Request* req, const Totals* totals) {
  wait_for_predecessor();
  let_successor_start();
  carry_out(c, req, totals, (int64_t)blockIdx.x * blockDim.x + threadIdx.x, (int64_t)gridDim.x * blockDim.x);
}

}  // namespace

size_t slots_workspace_bytes(int32_t R) { return sizeof(Totals) + 16 + (size_t)R * sizeof(Request); }

af_status launch_block_slots(af_ctx* ctx, const SlotsCall& c, cudaStream_t s) {
  const af_status st = ws_grow(ctx->slots_ws, slots_workspace_bytes(c.R));
  if (st != AF_OK) return st;
  Totals* const totals = static_cast<Totals*>(ctx->slots_ws.p);
  Request* const req = reinterpret_cast<Request*>(static_cast<char*>(ctx->slots_ws.p) + ((sizeof(Totals) + 15) & ~15u));
  if (launch_overlapped(slots_plan_kernel, 1, kPlanThreads, 0, s, c, req, totals, ctx->d_err) != cudaSuccess) return AF_ERR_CUDA;
  const int64_t want = (c.capacity + 255) / 256 + 1, most = (int64_t)ctx->sm_count * 8;
  return launch_overlapped(slots_carry_out_kernel, (int)(want < most ? want : most), 256, 0, s, c, (const Request*)req,
                           (const Totals*)totals) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
