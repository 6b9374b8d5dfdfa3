// af_distill_loss, divergences with one more outcome for the rest (see distill_rows.cuh).
#include "distill_rows.cuh"

namespace af {
namespace distill {

cudaError_t launch_tail(const DistillCall& c, int vec, cudaStream_t s) {
  return c.prm.divergence == 0 ? launch_support<2, true>(c, vec, s) : launch_support<2, false>(c, vec, s);
}

}  // namespace distill
}  // namespace af
