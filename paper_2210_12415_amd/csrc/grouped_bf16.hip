// Grouped products in bf16.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_bf16(int form, const GroupedParams &p, hipStream_t st)
{
    return form == kForward ? grouped_run<bf16_tag, kForward>(p, st) : form == kInput ? grouped_run<bf16_tag, kInput>(p, st) : grouped_run<bf16_tag, kWeights>(p, st);
}

}  // namespace alt
