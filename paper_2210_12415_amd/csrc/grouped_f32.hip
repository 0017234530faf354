// Grouped products in fp32.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_f32(int form, const GroupedParams &p, hipStream_t st)
{
    return form == kForward ? grouped_run<float, kForward>(p, st) : form == kInput ? grouped_run<float, kInput>(p, st) : grouped_run<float, kWeights>(p, st);
}

}  // namespace alt
