// Host side of attention of trees of drafted tokens (include/treeattn.h): argument checks, and how the work is split.
#include "prefixattn_join.h"
#include "treeattn.h"

using namespace addrms_host;
using namespace serving;

namespace {

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Checks a shape and splits its work.  What a sequence may hold at most counts, for its length is known on the device alone.
int plan_of(const prefixattn_shape* s, Plan* p)
{
    if (const int st = shape_of(s, p)) return st;
    if (s->q_len > TREE_MAX_NODES) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "a tree of %d nodes is beyond the limit (%d)", s->q_len, TREE_MAX_NODES);
    if (p->rows == 0) return ADDRMS_OK;
    AttnArgs& a = p->a;
    const int64_t width = s->suffix_width * s->page_size, all = static_cast<int64_t>(s->batch) * s->q_len * a.group, own = static_cast<int64_t>(s->q_len) * a.group;
    p->suffix_form = form_of(own, p->dp);
    p->prefix_form = form_of(all, p->dp);
    auto wanted = [p](int form) { return form == MANY_256 || (form == MANY_128 && p->dp > 128) ? 256 : 512; };
    auto few = [](int64_t units) { return units <= kFinishUnits ? FEW_8 : FEW; };
    // a short prefix is seen by each sequence's workgroup, by prefixattn.hip's rule
    const int64_t units = static_cast<int64_t>(a.kv_heads) * s->batch, key_bytes = std::max(256, 2 * p->dp * (s->format == KVCACHE_E4M3 ? 1 : 2));
    const int64_t prefix_bytes = a.prefix_len * key_bytes, chain = prefix_bytes + width * key_bytes;
    if (a.pages && a.prefix_len && p->suffix_form == FEW &&
        (units >= kFinishUnits ? units * prefix_bytes <= kInlineBytes : chain <= (units >= kFinishUnits / 2 ? 2 * kInlineChain : kInlineChain))) {
        p->prefix_form = p->suffix_form = few(units);
        p->finish = true;
        a.inline_len = a.prefix_len;
        a.suffix_tiles = a.suffix_splits = 1;
        a.suffix_chunk = static_cast<int32_t>(width);
        p->suffix_blocks = round_up(units, 8);
        return fits(*p);
    }
    // a cache without a page has no key (the kernels read row 0 in the place of one that is not there)
    const bool prefix = a.prefix_len && a.pages, suffix = width && a.pages;
    if (!prefix) p->prefix_form = p->suffix_form;
    a.prefix_tiles = static_cast<int32_t>(tiles_of(all, p->prefix_form));
    a.suffix_tiles = static_cast<int32_t>(tiles_of(own, p->suffix_form));
    const int64_t prefix_units = static_cast<int64_t>(a.prefix_tiles) * a.kv_heads, suffix_units = static_cast<int64_t>(a.suffix_tiles) * a.kv_heads * s->batch;
    a.prefix_splits = prefix ? splits_of(a.prefix_len, prefix_units, wanted(p->prefix_form), kMinChunk, &a.prefix_chunk) : 0;
    p->finish = suffix && suffix_units >= kFinishUnits && a.prefix_splits <= kFinishSplits;
    if (p->finish && p->suffix_form == FEW) p->suffix_form = few(suffix_units);
    if (p->finish && !prefix) p->prefix_form = p->suffix_form;
    if (suffix) {
        a.suffix_splits = splits_of(width, suffix_units, p->finish ? 1 : 2 * wanted(p->suffix_form), 2 * kMinChunk, &a.suffix_chunk);
        p->suffix_blocks = round_up(a.kv_heads * static_cast<int64_t>(s->batch) * a.suffix_splits, 8) * a.suffix_tiles;
    }
    p->prefix_blocks = round_up(static_cast<int64_t>(a.prefix_splits) * a.kv_heads, 8) * a.prefix_tiles;
    const int64_t parts = a.prefix_splits + (p->finish ? 0 : a.suffix_splits);
    p->bytes = parts * p->rows * (4ll * a.d + 8);
    return fits(*p);
}

}  // namespace

extern "C" {

int64_t treeattn_workspace_bytes(const prefixattn_shape* shape)
{
    Plan p;
    if (const int st = plan_of(shape, &p)) return st;
    return p.bytes;
}

int64_t treeattn_algorithmic_bytes(const prefixattn_shape* shape, int64_t suffix_keys)
{
    Plan p;
    if (const int st = plan_of(shape, &p)) return st;
    if (suffix_keys < 0) return fail(ADDRMS_ERR_INVALID_ARG, "suffix_keys must be >= 0");
    const int64_t key = 2ll * shape->kv_heads * (shape->format == KVCACHE_E4M3 ? shape->d + 1 : 2 * shape->d);
    return (shape->prefix_len + suffix_keys) * key + p.rows * (4ll * shape->d + 4) + 8ll * shape->batch * shape->q_len;
}

int treeattn_run(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale,
                 const int32_t* prefix_pages, const int32_t* suffix_pages, const int32_t* suffix_lens, const int64_t* masks, void* out, float* lse, float scale,
                 const prefixattn_shape* shape, void* workspace, int64_t workspace_bytes, void* stream)
{
    Plan p;
    if (const int st = plan_of(shape, &p)) return st;
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
    SERVING_HIP_TRY(launch_join<true>(p, shape->dtype, s));
    return ADDRMS_OK;
}

}  // extern "C"
