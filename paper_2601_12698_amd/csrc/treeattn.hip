// Host side of attention of trees of drafted tokens (include/treeattn.h): argument checks and launches.
#include "treeattn_kernel.h"
#include "treeattn_plan.h"
#include "treeattn.h"

using namespace addrms_host;
using namespace serving;

extern "C" {

int64_t treeattn_workspace_bytes(const prefixattn_shape* shape)
{
    Plan p;
    if (const int st = tree_plan_of(shape, &p)) return st;
    return p.bytes;
}

int64_t treeattn_algorithmic_bytes(const prefixattn_shape* shape, int64_t suffix_keys)
{
    Plan p;
    if (const int st = tree_plan_of(shape, &p)) return st;
    if (suffix_keys < 0) return fail(ADDRMS_ERR_INVALID_ARG, "suffix_keys must be >= 0");
    const int64_t key = 2ll * shape->kv_heads * (shape->format == KVCACHE_E4M3 ? shape->d + 1 : 2 * shape->d);
    return (shape->prefix_len + suffix_keys) * key + p.rows * (4ll * shape->d + 4) + 8ll * shape->batch * shape->q_len;
}

int treeattn_run(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale,
                 const int32_t* prefix_pages, const int32_t* suffix_pages, const int32_t* suffix_lens, const int64_t* masks, void* out, float* lse, float scale,
                 const prefixattn_shape* shape, void* workspace, int64_t workspace_bytes, void* stream)
{
    Plan p;
    if (const int st = tree_plan_of(shape, &p)) return st;
    if (const int st = arguments_of(q, q_strides, k_pages, v_pages, k_scale, v_scale, prefix_pages, suffix_pages, suffix_lens, out, lse, scale, shape, workspace,
                                    workspace_bytes, &p))
        return st;
    if (p.rows == 0) return ADDRMS_OK;
    if (!masks) return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if (!aligned_to(masks, 8)) return fail(ADDRMS_ERR_MISALIGNED, "masks must be aligned to 8 bytes");
    AttnArgs& a = p.a;
    a.masks = addr(masks);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    static constexpr AttnLaunch kUnits[2][2][3] = {
        {{TREE_UNIT(0, 0, 64), TREE_UNIT(0, 0, 128), TREE_UNIT(0, 0, 256)}, {TREE_UNIT(0, 1, 64), TREE_UNIT(0, 1, 128), TREE_UNIT(0, 1, 256)}},
        {{TREE_UNIT(1, 0, 64), TREE_UNIT(1, 0, 128), TREE_UNIT(1, 0, 256)}, {TREE_UNIT(1, 1, 64), TREE_UNIT(1, 1, 128), TREE_UNIT(1, 1, 256)}}};
    const AttnLaunch unit = kUnits[shape->dtype == ADDRMS_FP16][shape->format == KVCACHE_E4M3][p.dp == 64 ? 0 : p.dp == 128 ? 1 : 2];
    if (p.finish) {
        if (p.prefix_blocks) SERVING_HIP_TRY(unit(a, p.prefix_form, p.suffix_form, static_cast<unsigned>(p.prefix_blocks), s));
        a.finish = 1;
        a.prefix_blocks = 0;
        SERVING_HIP_TRY(unit(a, p.suffix_form, p.suffix_form, static_cast<unsigned>(p.suffix_blocks), s));
        return ADDRMS_OK;
    }
    if (p.prefix_blocks + p.suffix_blocks) SERVING_HIP_TRY(unit(a, p.prefix_form, p.suffix_form, static_cast<unsigned>(p.prefix_blocks + p.suffix_blocks), s));
    const TreeJoin join = tree_join_of(p);
    const int64_t blocks = join == JOIN_WAVE ? (p.rows + 3) / 4 : join == JOIN_COLUMNS ? p.rows * ((a.d + kJoinColumns - 1) / kJoinColumns) : p.rows;
#define JOIN(DT) (join == JOIN_WAVE ? tree_join_kernel<DT, 1, false> : join == JOIN_COLUMNS ? tree_join_kernel<DT, 4, true> : tree_join_kernel<DT, 4, false>)
    SERVING_HIP_TRY(launch_kernel(shape->dtype == ADDRMS_FP16 ? JOIN(DT_FP16) : JOIN(DT_BF16), dim3(static_cast<unsigned>(blocks)), dim3(kJoinThreads), s, a));
#undef JOIN
    return ADDRMS_OK;
}

}  // extern "C"
