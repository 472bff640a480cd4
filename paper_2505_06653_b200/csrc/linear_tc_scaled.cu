// The backward variants of the kernel in linear_tc.cuh that multiply the sums of a token: the gradient of a vocabulary loss.
#include "linear_tc.cuh"

namespace bof4 {

int linear_tc_scaled(const LtLaunch& go) { return lt_launch<true, false, true>(go); }

}  // namespace bof4
