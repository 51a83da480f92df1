// Group-norm backward of bf16 activations with bf16 incoming gradients.
#include "gn_bwd.h"

namespace ckpt {
namespace gnb {

void run_bf16_bf16(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a) {
  p.df ? run_types<__bf16, __bf16, float>(s, p, g, a) : run_types<__bf16, __bf16, __bf16>(s, p, g, a);
}

}  // namespace gnb
}  // namespace ckpt
