// Products in fp32 with low-rank adapters beside them.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_adapted_f32(const GroupedParams &p, hipStream_t st) { return grouped_run<f32_adapted_tag, kForward>(p, st); }

}  // namespace alt
