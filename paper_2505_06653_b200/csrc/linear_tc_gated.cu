// The gated variants of the kernel in linear_tc.cuh.
#include "linear_tc.cuh"

namespace bof4 {

int linear_tc_gated(const LtLaunch& go) { return lt_launch<false, true>(go); }

}  // namespace bof4
