// af_distill_loss, divergences renormalised over the listed ids (see distill_rows.cuh).
#include "distill_rows.cuh"

namespace af {
namespace distill {

cudaError_t launch_renormalised(const DistillCall& c, int vec, cudaStream_t s) {
  return c.prm.divergence == 0 ? launch_support<1, true>(c, vec, s) : launch_support<1, false>(c, vec, s);
}

}  // namespace distill
}  // namespace af
