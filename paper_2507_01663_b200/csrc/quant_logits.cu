// af_quant_logits: logits of a few tokens from a head in 4 bits, one pass over the codes per 64 of them.
#include "rollout.cuh"

namespace af {

af_status launch_quant_logits(af_ctx* ctx, const void* hidden, const QuantHead& h, int64_t T, void* logits, int32_t type,
                              int64_t pitch, cudaStream_t s) {
  const int64_t element = type == AF_F32 ? 4 : 2;
  for (int64_t t = 0; t < T; t += kQuantTokens) {
    const int n = (int)(T - t < kQuantTokens ? T - t : kQuantTokens);
    const af_status st = launch_quant_umma(ctx, static_cast<const char*>(hidden) + t * h.d * 2, h, n,
                                           static_cast<char*>(logits) + t * pitch * element, type, pitch, s);
    if (st != AF_OK) return st;
  }
  return AF_OK;
}

}  // namespace af
