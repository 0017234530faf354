// Grouped products in f32: which kernel a call runs.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_f32(int form, GroupedParams p, hipStream_t st)
{
    switch (form) {
        case kForward: return grouped_tiles<float, kForward, 64, 64, 2, 2, 128>(p, st);
        case kInput: return grouped_tiles<float, kInput, 64, 64, 2, 2, 128>(p, st);
        case kWeights: return grouped_tiles<float, kWeights, 64, 64, 2, 2, 128>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace alt
