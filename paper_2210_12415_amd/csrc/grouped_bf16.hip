// Grouped products in bf16: which kernel a call runs.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_bf16(int form, GroupedParams p, hipStream_t st)
{
    switch (form) {
        case kForward: return grouped_tiles<bf16_tag, kForward, 64, 64, 2, 2, 128>(p, st);
        case kInput: return grouped_tiles<bf16_tag, kInput, 64, 64, 2, 2, 128>(p, st);
        case kWeights: return grouped_tiles<bf16_tag, kWeights, 64, 64, 2, 2, 128>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace alt
