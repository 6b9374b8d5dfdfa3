// Lists of candidate ids per token, shared by the scoring kernel and its backward.
//
// A list arrives in any order.  The GEMM epilogues sweep the vocabulary upwards with one output row per
// thread, so each row's list is sorted once beforehand into 32-bit keys, id << 8 | slot: a thread then
// only compares the next key with the end of its columns.  Slots without a valid id sort to the end.
#pragma once

#include "common.cuh"
#include "device_util.cuh"

namespace af {

constexpr uint32_t kNoCandidate = 0xffffffffu;      // id 2^24 - 1, which no vocabulary that is accepted holds
constexpr int32_t kMaxCandidateVocab = (1 << 24) - 256;
static_assert(AF_MAX_CANDIDATES == 256, "a slot has 8 bits of a key");

// Position of the first key whose id is >= col in a sorted row of K keys.
__device__ __forceinline__ int first_candidate(const uint32_t* __restrict__ keys, int K, int col) {
  int lo = 0, hi = K;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if ((int)(__ldg(keys + mid) >> 8) < col) lo = mid + 1; else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ uint32_t candidate_at(const uint32_t* __restrict__ keys, int K, int i) {
  return i < K ? __ldg(keys + i) : kNoCandidate;
}

// Sorts the lists of `rows` tokens.  With g given (the gradients of the listed log-probs) gsum[row]
// receives their sum over the slots with a valid id.
cudaError_t launch_sort_candidates(const int32_t* cand, const float* g, int64_t rows, int32_t K, int32_t V,
                                   uint32_t* keys, float* gsum, cudaStream_t s);

// The one-pass kernel for a few tokens (candidate_stream.cu).
constexpr int kStreamTokens = 16;
struct StreamCall {
  const void* hidden;
  const void* W;
  const int32_t* cand;
  int T, K, d, V;
  float* z;               // [T, V] workspace
  float4* partial;        // [T, CTAs] workspace
  float* cand_logp;
  float* entropy;
  float* lse;
  unsigned int* ticket;   // zero between calls
  unsigned int* d_err;
};
bool stream_fits(int64_t T, int32_t d);
af_status launch_candidate_stream(const StreamCall& c, int sm_count, cudaStream_t s);

}  // namespace af
