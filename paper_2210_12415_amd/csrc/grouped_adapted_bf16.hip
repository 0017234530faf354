// Products in bf16 with low-rank adapters beside them.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_adapted_bf16(const GroupedParams &p, hipStream_t st) { return grouped_run<bf16_adapted_tag, kForward>(p, st); }

}  // namespace alt
