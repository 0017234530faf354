// Grouped products in i8: which kernel a call runs.
#include "grouped.h"

namespace alt {

hipError_t grouped_run_i8(GroupedParams p, hipStream_t st)
{
    return grouped_tiles<i8_tag, kForward, 64, 64, 2, 2, 128>(p, st);
}

}  // namespace alt
