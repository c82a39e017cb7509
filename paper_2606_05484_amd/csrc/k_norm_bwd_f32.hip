// The backward of the norms around a block (norm_bwd.hpp) on fp32 rows of x.
#include "norm_bwd.hpp"

namespace mapl {

hipError_t launch_norm_bwd_f32(const NormArgs& g, hipStream_t s) {
  if (g.h_f32) return g.once ? pick<float, float, true>(g, s) : pick<float, float, false>(g, s);
  return g.once ? pick<float, bf16_t, true>(g, s) : pick<float, bf16_t, false>(g, s);
}

}  // namespace mapl
