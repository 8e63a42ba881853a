// The attention kernels of one element type (UNIT_DT), cache format (UNIT_FORMAT) and padded head size (UNIT_DP).
#include "prefixattn_kernel.h"

namespace serving {
namespace {

template <int PREFIX, int SUFFIX>
void launch(const AttnArgs& a, unsigned blocks, hipStream_t s)
{
    attn_kernel<UNIT_DT, UNIT_FORMAT, UNIT_DP, PREFIX, SUFFIX><<<blocks, threads_of<UNIT_DP>(PREFIX), 0, s>>>(a);
}

}  // namespace

// A sequence's rows are some of the prefix's rows, so that its form is never the larger one.
hipError_t ATTN_UNIT(UNIT_DT, UNIT_FORMAT, UNIT_DP)(const AttnArgs& a, int prefix_form, int suffix_form, unsigned blocks, hipStream_t s)
{
    if (prefix_form == FEW_8) launch<FEW_8, FEW_8>(a, blocks, s);
    else if (prefix_form == FEW) launch<FEW, FEW>(a, blocks, s);
    else if (prefix_form == MANY_64) suffix_form == FEW ? launch<MANY_64, FEW>(a, blocks, s) : launch<MANY_64, MANY_64>(a, blocks, s);
    else if (prefix_form == MANY_128 || UNIT_DP != 128) {
        if (suffix_form == FEW) launch<MANY_128, FEW>(a, blocks, s);
        else if (suffix_form == MANY_64) launch<MANY_128, MANY_64>(a, blocks, s);
        else launch<MANY_128, MANY_128>(a, blocks, s);
    } else {
#if UNIT_DP == 128
        if (suffix_form == FEW) launch<MANY_256, FEW>(a, blocks, s);
        else if (suffix_form == MANY_64) launch<MANY_256, MANY_64>(a, blocks, s);
        else if (suffix_form == MANY_128) launch<MANY_256, MANY_128>(a, blocks, s);
        else launch<MANY_256, MANY_256>(a, blocks, s);
#endif
    }
    return hipGetLastError();
}

}  // namespace serving
