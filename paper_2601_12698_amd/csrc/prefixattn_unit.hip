// The attention kernels of one element type (UNIT_DT), cache format (UNIT_FORMAT) and padded head size (UNIT_DP).
#include "prefixattn_kernel.h"

namespace serving {

hipError_t ATTN_UNIT(UNIT_DT, UNIT_FORMAT, UNIT_DP)(const AttnArgs& a, int prefix_form, int suffix_form, unsigned blocks, hipStream_t s)
{
    if (prefix_form == FEW) attn_kernel<UNIT_DT, UNIT_FORMAT, UNIT_DP, FEW, FEW><<<blocks, kAttnThreads, 0, s>>>(a);
    else if (suffix_form == FEW) attn_kernel<UNIT_DT, UNIT_FORMAT, UNIT_DP, MANY, FEW><<<blocks, kAttnThreads, 0, s>>>(a);
    else attn_kernel<UNIT_DT, UNIT_FORMAT, UNIT_DP, MANY, MANY><<<blocks, kAttnThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace serving
