// Grouped products in 8-bit integers.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_i8(const GroupedParams &p, hipStream_t st) { return grouped_run<i8_tag, kForward>(p, st); }

}  // namespace alt
