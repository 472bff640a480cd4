// The backward variants of the kernel in linear_tc.cuh.
#include "linear_tc.cuh"

namespace bof4 {

int linear_tc_backward(const LtLaunch& go) { return lt_launch<true, false>(go); }

}  // namespace bof4
