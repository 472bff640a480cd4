// The gated variants of the kernel in linear_tc.cuh whose accumulators take a segment of K: results in fp32.
#include "linear_tc.cuh"

namespace bof4 {

int linear_tc_gated_segments(const LtLaunch& go) { return lt_launch<false, true, false, true>(go); }

}  // namespace bof4
