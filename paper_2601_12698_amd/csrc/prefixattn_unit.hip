// The attention kernels of one element type (UNIT_DT), cache format (UNIT_FORMAT) and padded head size (UNIT_DP).
#include "prefixattn_kernel.h"

namespace serving {
namespace {

template <int PREFIX, int SUFFIX>
hipError_t launch(const AttnArgs& a, unsigned blocks, hipStream_t s)
{
    return launch_kernel(attn_kernel<UNIT_DT, UNIT_FORMAT, UNIT_DP, PREFIX, SUFFIX>, dim3(blocks), dim3(threads_of(PREFIX, UNIT_DP)), s, a);
}

}  // namespace

// A sequence's rows are some of the prefix's rows, so that its form is never the larger one.
hipError_t ATTN_UNIT(UNIT_DT, UNIT_FORMAT, UNIT_DP)(const AttnArgs& a, int prefix_form, int suffix_form, unsigned blocks, hipStream_t s)
{
    if (prefix_form == FEW_8) return launch<FEW_8, FEW_8>(a, blocks, s);
    if (prefix_form == FEW) return launch<FEW, FEW>(a, blocks, s);
    if constexpr (UNIT_DP <= 128) {
        if (prefix_form == MANY_64) return suffix_form == FEW ? launch<MANY_64, FEW>(a, blocks, s) : launch<MANY_64, MANY_64>(a, blocks, s);
        if (prefix_form == MANY_128 && suffix_form == MANY_64) return launch<MANY_128, MANY_64>(a, blocks, s);
    }
#if UNIT_DP == 128
    if (prefix_form == MANY_256) {
        if (suffix_form == FEW) return launch<MANY_256, FEW>(a, blocks, s);
        if (suffix_form == MANY_64) return launch<MANY_256, MANY_64>(a, blocks, s);
        return suffix_form == MANY_128 ? launch<MANY_256, MANY_128>(a, blocks, s) : launch<MANY_256, MANY_256>(a, blocks, s);
    }
#endif
    return suffix_form == FEW ? launch<MANY_128, FEW>(a, blocks, s) : launch<MANY_128, MANY_128>(a, blocks, s);
}

}  // namespace serving
