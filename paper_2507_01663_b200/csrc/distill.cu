// af_distill_loss: the choice of the kernel, and the divergences as listed (see distill_rows.cuh).
#include "distill_rows.cuh"

namespace af {
namespace distill {

cudaError_t launch_listed(const DistillCall& c, int vec, cudaStream_t s) {
  return c.prm.divergence == 0 ? launch_support<0, true>(c, vec, s) : launch_support<0, false>(c, vec, s);
}

}  // namespace distill

cudaError_t launch_distill_loss(const float* cand_logp, const float* teacher_logp, const int32_t* cu, int32_t B,
                                int64_t T, int64_t t0, int64_t rows, int32_t K, const af_distill_params& p,
                                af_distill_out* out, float* token_loss, float* dcand, void* ws, unsigned int* d_err,
                                int sm_count, cudaStream_t s) {
  const uintptr_t inputs = reinterpret_cast<uintptr_t>(cand_logp) | reinterpret_cast<uintptr_t>(teacher_logp);
  const uintptr_t all = inputs | reinterpret_cast<uintptr_t>(dcand);
  const int vec = K % 4 == 0 && (all & 15) == 0 ? 4 : K % 2 == 0 && (all & 7) == 0 ? 2 : 1;
  const distill::DistillCall c{cand_logp, teacher_logp, cu, B, (int)T, (int)t0, (int)rows, K, p, out, token_loss, dcand,
                      static_cast<distill::DistillWs*>(ws), d_err, sm_count, (inputs & 15) ? 0 : (all & 15) ? 1 : 3};
  switch (p.support) {
    case 0: return distill::launch_listed(c, vec, s);
    case 1: return distill::launch_renormalised(c, vec, s);
    default: return distill::launch_tail(c, vec, s);
  }
}

}  // namespace af
