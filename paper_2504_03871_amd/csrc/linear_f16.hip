// The dense products' kernels with f16 storage (linear_half.h).
#include "linear_half.h"

namespace moe {

int linear_forward_f16(int act, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) { return LinearHalf<f16>::forward(act, g, p, ws, s); }
int linear_input_grad_f16(bool two, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) { return LinearHalf<f16>::input_grad(two, g, p, ws, s); }
int linear_weight_grad_f16(bool in_type, const GemmArgs& g, const LinearPlan& p, hipStream_t s) { return LinearHalf<f16>::weight_grad(in_type, g, p, s); }
int linear_both_grads_f16(bool two, bool in_type, const GemmArgs& g1, const GemmArgs& g2, const LinearPlan& p, float* ws, hipStream_t s) {
  return LinearHalf<f16>::both_grads(two, in_type, g1, g2, p, ws, s);
}

}  // namespace moe
