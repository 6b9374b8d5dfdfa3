// af_block_slots: block tables and the rows of new tokens of a paged store, from the requests' lengths.
//
// A plan first (one CTA): what every request gives back and wants, as running sums over the requests, and who gets it.
// Then everything that the sums determine, item by item and in any order: rows of tokens, table entries of new
// blocks, free-list entries of blocks given back.  Blocks given back in a call serve the same call: the k-th wanted one
// comes from place available - 1 - k of the stack, and a place that this call would have pushed is looked up in the
// table it comes from, so nothing that is written here is read here.  Whole numbers only: the answer is unique.
//
// A decoding step (some thousand requests and tokens at most) is one launch of one CTA, all latency: loads, one scan, a search
// per token in shared memory.  A larger batch takes two; in the second a CTA takes 2048 neighbouring tokens, whose
// requests are few, and writes 12 bytes for each: what bounds it.
#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

struct alignas(16) Request {     // one request's share of the plan
  int64_t given_at, wanted_at;   // blocks given back / wanted by the requests before it
  int32_t held, need;            // blocks of its table before, and with the new tokens
  int32_t length;                // tokens kept, -1: the request is refused
  int32_t pad;
};
struct Totals {
  int64_t available, count, given, taken, tokens;   // taken: blocks that leave the stack
};
constexpr int kPlanThreads = 1024;
constexpr int kPerThread = 4;                    // neighbouring requests of a thread
constexpr int kPlanTile = kPlanThreads * kPerThread;
constexpr int kTokenTile = 2048, kTokenThreads = 256;
constexpr int kCached = 1024;                    // running token sums that a tile keeps in shared memory
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

// Block b of a block size that is often a power of two.
struct BlockSize {
  int32_t n, shift;                                          // shift: -1 if n is no power of two
  __device__ __forceinline__ explicit BlockSize(int32_t size) {
    n = size;
    shift = (size & (size - 1)) == 0 ? 31 - __clz(size) : -1;
  }
  __device__ __forceinline__ int32_t of(int32_t pos) const { return shift >= 0 ? pos >> shift : pos / n; }
};

// s_cu (nullable): also receives cu, up to kPlanTile + 1 entries.
__device__ void plan(const SlotsCall& c, Request* req, Totals* totals, int32_t* s_cu, unsigned int* d_err) {
  __shared__ Sums warp_sums[kPlanThreads / 32];
  unsigned int bad = 0;
  Wish w[kPerThread];
  auto wishes = [&](int r0) {
    Sums mine{0, 0, 0};
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int r = r0 + (int)threadIdx.x * kPerThread + k;
      w[k] = Wish{0, 0, 0, 0, true};
      if (r >= c.R) continue;
      w[k] = wish(c, r);
      mine.tokens += w[k].tokens;
      if (w[k].need < w[k].held) mine.given += w[k].held - w[k].need; else mine.wanted += w[k].need - w[k].held;
    }
    return mine;
  };
  int64_t count = *c.free_count;
  int64_t given = 0;
  Sums mine{}, all{}, at{};
  for (int r0 = 0; r0 < c.R; r0 += kPlanTile) {              // what comes back, before anything is promised
    mine = wishes(r0);
    at = scan(mine, &all, warp_sums);
    given += all.given;
  }
  if (count < 0 || count > c.n_blocks) { bad |= AF_DEVERR_REQUEST; count = count < 0 ? 0 : c.n_blocks; }
  int64_t available = count + given;
  if (available > c.n_blocks) { bad |= AF_DEVERR_REQUEST; available = c.n_blocks; }
  Sums before{0, 0, 0};
  int64_t taken = 0;
  for (int r0 = 0; r0 < c.R; r0 += kPlanTile) {
    if (c.R > kPlanTile) {                                   // else all is still at hand
      mine = wishes(r0);
      at = scan(mine, &all, warp_sums);
    }
    Sums here = before + at;
    before = before + all;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int r = r0 + (int)threadIdx.x * kPerThread + k;
      if (r >= c.R) break;
      const int64_t back = w[k].need < w[k].held ? w[k].held - w[k].need : 0, want = w[k].need > w[k].held ? w[k].need - w[k].held : 0;
      const bool granted = w[k].valid && (want == 0 || here.wanted + want <= available);
      if (!w[k].valid) bad |= AF_DEVERR_REQUEST;
      else if (!granted) bad |= AF_DEVERR_BLOCKS;
      req[r] = Request{here.given, here.wanted, w[k].held, w[k].need, granted ? w[k].length : -1, 0};
      c.held_out[r] = granted ? w[k].need : w[k].held;
      if (c.granted) c.granted[r] = granted;
      const int32_t first = (int32_t)(here.tokens < kMostTokens ? here.tokens : kMostTokens);
      c.cu[r] = first;
      if (s_cu) s_cu[r] = first;
      // granted requests come first among those that want blocks: what they take is the largest of their ends
      if (granted && want > 0 && here.wanted + want > taken) taken = here.wanted + want;
      here = here + Sums{w[k].tokens, back, want};
    }
  }
  __shared__ unsigned long long most;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  if (taken > 0) atomicMax(&most, (unsigned long long)taken);
  if (bad) atomicOr(d_err, bad);
  __syncthreads();
  if (threadIdx.x == 0) {
    if (before.tokens > c.capacity || before.tokens > kMostTokens) atomicOr(d_err, AF_DEVERR_REQUEST);
    const int32_t end = (int32_t)(before.tokens < kMostTokens ? before.tokens : kMostTokens);
    c.cu[c.R] = end;
    if (s_cu) s_cu[c.R] = end;
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

// The row of token i of a batch, one of request r's.
__device__ __forceinline__ void place_token(const SlotsCall& c, const Request* req, const Totals& t, const BlockSize& size, int64_t i, int r, int32_t first) {
  const uint4 x = __ldcg(reinterpret_cast<const uint4*>(&req[r].held));        // held, need, length
  const int32_t held = (int32_t)x.x, length = (int32_t)x.z;
  int64_t row = -1;
  int32_t pos;
  if (length >= 0) {
    pos = length + (int32_t)(i - first);
    const int32_t column = size.of(pos);
    const int32_t block = column < held ? c.table[r * c.table_pitch + column]
                                        : wanted_block(c, req, t, __ldcg(&req[r].wanted_at) + column - held);
    row = (int64_t)block * size.n + (pos - column * size.n);
  } else {
    pos = (int32_t)((int64_t)c.length[r] + (i - first));
  }
  c.slot[i] = row;
  if (c.position) c.position[i] = pos;
}
// Table entries of new blocks, and free-list entries of blocks given back.
__device__ __forceinline__ void move_blocks(const SlotsCall& c, const Request* req, const Totals& t, int64_t thread, int64_t threads) {
  for (int64_t k = thread; k < t.taken; k += threads) {
    const int r = search(c.R, k, [&](int j) { return __ldcg(&req[j].wanted_at); });
    const int64_t column = __ldcg(&req[r].held) + k - __ldcg(&req[r].wanted_at);
    c.table[r * c.table_pitch + column] = wanted_block(c, req, t, k);
  }
  const int64_t left = t.available - t.taken;
  for (int64_t p = t.count + thread; p < left; p += threads) c.free_blocks[p] = given_block(c, req, p - t.count);
}
__device__ __forceinline__ Totals totals_of(const Totals* totals) {
  return {__ldcg(&totals->available), __ldcg(&totals->count), __ldcg(&totals->given), __ldcg(&totals->taken), __ldcg(&totals->tokens)};
}
__device__ __forceinline__ int64_t tokens_of(const SlotsCall& c, const Totals& t) {
  const int64_t n = t.tokens < kMostTokens ? t.tokens : kMostTokens;
  return n < c.capacity ? n : c.capacity;
}

__global__ void __launch_bounds__(kPlanThreads) slots_plan_kernel(const SlotsCall c, Request* req, Totals* totals, unsigned int* d_err) {
  wait_for_predecessor();
  let_successor_start();
  plan(c, req, totals, nullptr, d_err);
}
// All of a small batch: at most kPlanTile requests.
__global__ void __launch_bounds__(kPlanThreads) slots_step_kernel(const SlotsCall c, Request* req, Totals* totals, unsigned int* d_err) {
  __shared__ int32_t s_cu[kPlanTile + 1];
  wait_for_predecessor();
  let_successor_start();
  plan(c, req, totals, s_cu, d_err);
  __threadfence_block();
  __syncthreads();
  const Totals t = totals_of(totals);
  const int64_t n = tokens_of(c, t);
  const BlockSize size(c.block_size);
  for (int64_t i = threadIdx.x; i < n; i += kPlanThreads) {
    const int r = search(c.R, i, [&](int j) { return (int64_t)s_cu[j]; });
    place_token(c, req, t, size, i, r, s_cu[r]);
  }
  move_blocks(c, req, t, threadIdx.x, kPlanThreads);
}
// 2048 neighbouring tokens at a time.
__global__ void __launch_bounds__(kTokenThreads) slots_carry_out_kernel(const SlotsCall c, const Request* req, const Totals* totals) {
  __shared__ int32_t s_cu[kCached + 1];
  __shared__ int s_ends[2];
  wait_for_predecessor();
  let_successor_start();
  const Totals t = totals_of(totals);
  const int64_t n = tokens_of(c, t), tiles = (n + kTokenTile - 1) / kTokenTile;
  const BlockSize size(c.block_size);
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t i0 = tile * kTokenTile, i1 = min(i0 + kTokenTile, n);
    __syncthreads();                                         // s_cu of the tile before
    if (threadIdx.x < 64) {                                  // the requests of the first and of the last token, a warp each
      const int r = find_seq_warp(c.cu, c.R, (int)(threadIdx.x < 32 ? i0 : i1 - 1), threadIdx.x & 31);
      if ((threadIdx.x & 31) == 0) s_ends[threadIdx.x >> 5] = r;
    }
    __syncthreads();
    const int r0 = s_ends[0], m = s_ends[1] - r0 + 1;
    if (m <= kCached) {
      for (int k = threadIdx.x; k < m; k += kTokenThreads) s_cu[k] = c.cu[r0 + k];
      __syncthreads();
      for (int64_t i = i0 + threadIdx.x; i < i1; i += kTokenThreads) {
        const int r = search(m, i, [&](int j) { return (int64_t)s_cu[j]; });
        place_token(c, req, t, size, i, r0 + r, s_cu[r]);
      }
    } else {                                                 // a stretch of requests most of which have no token
      for (int64_t i = i0 + threadIdx.x; i < i1; i += kTokenThreads) {
        const int r = r0 + search(m, i, [&](int j) { return (int64_t)c.cu[r0 + j]; });
        place_token(c, req, t, size, i, r, c.cu[r]);
      }
    }
  }
  move_blocks(c, req, t, (int64_t)blockIdx.x * kTokenThreads + threadIdx.x, (int64_t)gridDim.x * kTokenThreads);
}

}  // namespace

size_t slots_workspace_bytes(int32_t R) { return sizeof(Totals) + 16 + (size_t)R * sizeof(Request); }

af_status launch_block_slots(af_ctx* ctx, const SlotsCall& c, cudaStream_t s) {
  const af_status st = ws_grow(ctx->slots_ws, slots_workspace_bytes(c.R));
  if (st != AF_OK) return st;
  Totals* const totals = static_cast<Totals*>(ctx->slots_ws.p);
  Request* const req = reinterpret_cast<Request*>(static_cast<char*>(ctx->slots_ws.p) + ((sizeof(Totals) + 15) & ~15u));
  // one CTA for a small batch: 64 requests of 5 tokens 3 us for 5; it breaks even at some ten thousand tokens
  if (c.R <= kPlanTile && c.capacity <= 2 * kPlanTile)
    return launch_overlapped(slots_step_kernel, 1, kPlanThreads, 0, s, c, req, totals, ctx->d_err) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
  if (launch_overlapped(slots_plan_kernel, 1, kPlanThreads, 0, s, c, req, totals, ctx->d_err) != cudaSuccess) return AF_ERR_CUDA;
  const int64_t tiles = (c.capacity + kTokenTile - 1) / kTokenTile, most = (int64_t)ctx->sm_count * 8;
  return launch_overlapped(slots_carry_out_kernel, (int)(tiles < most ? tiles : most), kTokenThreads, 0, s, c, (const Request*)req,
                           (const Totals*)totals) == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
