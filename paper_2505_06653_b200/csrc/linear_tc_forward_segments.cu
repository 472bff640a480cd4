// The forward variants of the kernel in linear_tc.cuh whose accumulators take a segment of K: logits in fp32.
#include "linear_tc.cuh"

namespace bof4 {

int linear_tc_forward_segments(const LtLaunch& go) { return lt_launch<false, false, false, true>(go); }

}  // namespace bof4
