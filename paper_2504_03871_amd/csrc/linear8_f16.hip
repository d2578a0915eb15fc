// The products of linear8.hip with results in f16.
#include "gemm_i8_kernel.h"

namespace moe {

int gemm8_f16(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s) { return gemm8_for<f16>(act, g, c, max_tiles, s); }

}  // namespace moe
