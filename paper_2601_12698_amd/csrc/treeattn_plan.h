// How attention of trees of drafted tokens (include/treeattn.h) is cut into workgroups and launches.  Host code alone, and from a shape alone.
#pragma once
#include "prefixattn_plan.h"
#include "treeaccept.h"

namespace serving {

constexpr int64_t kShort = 1024, kShortBytes = 1 << 19, kLong = 1 << 20;      // keys of a sequence, and bytes of a head's (see tree_plan_of)

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

constexpr int64_t kPartKeys = 640;       // that cost as much as a part of 256 rows: below

// Splits of a prefix over `places` workgroups of many rows, `units` of them a split.  Its parts are written and read: each costs what `part_keys`
// keys do (256 rows of 128 in fp32, written and read by all CUs at once, 13 us).  The time of n splits is that of as many rounds of workgroups as
// they need, rounds * keys / n, and of their parts, part_keys * n * units / places; of each number of rounds the most splits it holds are
// looked at, and fewer where parts are dear.  (44 x 16 nodes of 32 heads over 12000 bf16 keys: 88 units; 3 splits need 264 places, and
// with up to 300 keys of their own 263 us a call, 5 splits 186; 64 x 16 of 40 over 8000 e4m3 266 and 205, 40 x 16 of 32 over 20000 332 and 242.)
inline int64_t prefix_splits_of(int64_t keys, int64_t units, int64_t places, int64_t part_keys, int64_t rounds)
{
    int64_t best = std::max<int64_t>(1, std::min(places / units, static_cast<int64_t>(sqrt(static_cast<double>(keys * places) / static_cast<double>(part_keys * units)))));
    const auto cost = [&](int64_t n) { return (n * units + places - 1) / places * keys / n + part_keys * n * units / places; };
    for (int64_t round = 2; round <= rounds; ++round)
        if (const int64_t n = round * places / units; n > 0 && cost(n) < cost(best)) best = n;
    return best;
}

// Checks a shape and splits its work.  What a sequence may hold at most counts, for its length is known on the device alone.
inline int tree_plan_of(const prefixattn_shape* s, Plan* p)
{
    if (const int st = shape_of(s, p)) return st;
    if (s->q_len > TREE_MAX_NODES) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "a tree of %d nodes is beyond the limit (%d)", s->q_len, TREE_MAX_NODES);
    if (p->rows == 0) return ADDRMS_OK;
    AttnArgs& a = p->a;
    const int64_t width = s->suffix_width * s->page_size, all = static_cast<int64_t>(s->batch) * s->q_len * a.group, own = static_cast<int64_t>(s->q_len) * a.group;
    // 128 rows a workgroup where 256 would leave a half without one (40 x 34 nodes of 64 query and 8 key heads over 2000 e4m3 keys 82.6 us in place of 112,
    // 8 x 64 of 48 over 8000 100 and 117; 12 x 7 of 32 beside a prefix of 8000 bf16 keys 33.9 and 38.1).  A sequence's form is never the larger one.
    const auto shape_form = [p](int64_t rows) {
        const int form = form_of(rows, p->dp);
        return form == MANY_256 && tiles_of(rows, MANY_128) < 2 * tiles_of(rows, MANY_256) ? MANY_128 : form;
    };
    p->suffix_form = shape_form(own);
    p->prefix_form = p->suffix_form == MANY_256 ? form_of(all, p->dp) : shape_form(all);
    auto wanted = [p](int form) { return form == MANY_256 || p->dp > 128 ? 256 : 512; };          // one workgroup a CU, or two
    // Eight waves of a workgroup, or four where workgroups fill the chip.  Heads of 256 leave room for one workgroup a CU in either case (60 x 3 nodes of
    // 32 heads over 200 bf16 keys 23.3 us, with four waves 28.5, 64 x 4 over 3000 e4m3 101 and 113; cut into pieces for 256 places, with four waves and for
    // 512, 4 x 2 over 2000 bf16 16.9 and 22.9, 1 x 3 over 30000 44.9 and 52.3).
    auto few = [p](int64_t units) { return p->dp > 128 || units <= kFinishUnits ? FEW_8 : FEW; };
    // Sequences of few keys: 16 rows a workgroup, whose waves share the keys, as often as there are rows; it reads the keys as often, but a
    // form with more rows a workgroup goes over them tile by tile.  Whole calls of 32 query and 8 key heads of 128, us, so and with more rows:
    //   8 x 16 nodes over 300 bf16 keys 10.8, 17.2      8 x 32 over 300 14.2, 22.7    2 x 16 over 700 11.4, 16.0     16 x 16 over 1000 23.6, 26.3
    //   16 x 32 over 1000 e4m3 29.3, 32.5               4 x 16 over 1500 18.5, 16.3   32 x 16 over 2000 53.8, 45.3   64 x 16 over 500 51.8, 25.6
    // and of heads of 256, 15 x 4 of 64 heads over 814 43.5, 25.2, 8 x 8 over 900 25.0, 18.5, 4 x 8 of 40 over 276 11.9, 14.4;
    // one a CU: 48 x 14 of 8 over 36 and up to 1 18.8, 10.5, 10 x 24 of 32 over 400 28.7, 23.9, over 900 e4m3 30.9, 37.1.
    const int64_t units16 = tiles_of(own, FEW) * a.kv_heads * s->batch;
    const int64_t key_bytes = std::max(256, 2 * p->dp * (s->format == KVCACHE_E4M3 ? 1 : 2));
    if (width <= kShort && width * key_bytes <= kShortBytes && units16 <= (p->dp > 128 && width <= kShort / 2 ? 1 : 2) * kFinishUnits) p->suffix_form = FEW;
    // A short prefix is seen by each sequence's workgroups before its own keys, in one launch: with few rows by prefixattn.hip's rule, up to twice the
    // bytes where they fill the chip (64 x 4 nodes over 700 and up to 100 bf16 keys 23.4 us, in two launches 29.4, 32 x 4 over 1400 21.0 and 26.3, over
    // 64 x 1400 33.0 either way); with more rows, where that fills the chip, up to 16 keys for each row of a workgroup, for the work is the same and
    // no part of the prefix's is written (64 x 64 nodes of 64 heads over 300 and up to 500 keys 141 us, so 219, over 2000 359 and 436; 64 x 32
    // nodes of 32 heads over 300 43.7 and 60.3, over 2000 112 and 114, over 8000 349 and 304; 64 x 16 over 600 40.8 and 50.9, over 2000 76.5 and 73.6).
    const int64_t units = tiles_of(own, p->suffix_form) * a.kv_heads * s->batch;
    const int64_t prefix_bytes = a.prefix_len * key_bytes, chain = prefix_bytes + width * key_bytes;
    // Also where a sequence's keys and the prefix's take no longer than apart (30 x 14 of 32 heads over 900 and up to 300 29.8 us and 41.3, 28 x 60 over 3000
    // and 400 e4m3 112 and 156, 60 x 60 of 16 over 3000 and 400 120 and 252, 25 x 40 over 300 and 100 25.5 and 56; not 10 x 30 of 32, 4 of them key heads,
    // over 1500 and 100, 58 and 38, nor 1 x 19 of 8 over 19 and 1072, 39 and 16).
    // What cutting costs, in keys that a workgroup goes over: a place's share, a launch (400; 800 of heads of 64; 200 for two kinds of work) and the parts.
    const auto apart = [p, width](int64_t prefix_len, int64_t units, int64_t places) {
        const int64_t share = std::max<int64_t>(kMinChunk, (2 * prefix_len + width) * units / (2 * places));
        return (p->dp > 64 ? 400 : 800) + (prefix_len ? 200 : 0) + share + ((p->rows * p->a.d * ((prefix_len + width) / share + 1)) >> 15);
    };
    const bool many_together = width && a.prefix_len <= 16 * kFormRows[p->suffix_form] && (units >= kFinishUnits || a.prefix_len + width <= apart(a.prefix_len, units, wanted(p->suffix_form)));
    const bool together = p->suffix_form != FEW ? many_together
                          : units >= kFinishUnits ? prefix_bytes <= 2 * kInlineBytes / units : chain <= (units >= kFinishUnits / 2 ? 2 * kInlineChain : kInlineChain);
    if (a.pages && a.prefix_len && together) {
        if (p->suffix_form == FEW) p->suffix_form = few(units);
        p->prefix_form = p->suffix_form;
        p->finish = true;
        a.inline_len = a.prefix_len;
        a.suffix_splits = 1;
        a.suffix_tiles = static_cast<int32_t>(tiles_of(own, p->suffix_form));
        a.sorted = width && s->batch <= 64 && units > wanted(p->suffix_form);      // without keys of their own there are no lengths to look at
        p->suffix_blocks = round_up(a.kv_heads * static_cast<int64_t>(s->batch), 8) * a.suffix_tiles;
        return fits(*p);
    }
    // a cache without a page has no key (the kernels read row 0 in the place of one that is not there)
    const bool prefix = a.prefix_len && a.pages, suffix = width && a.pages;
    if (!prefix) p->prefix_form = p->suffix_form;
    a.prefix_tiles = static_cast<int32_t>(tiles_of(all, p->prefix_form));
    a.suffix_tiles = static_cast<int32_t>(tiles_of(own, p->suffix_form));
    const int64_t prefix_units = static_cast<int64_t>(a.prefix_tiles) * a.kv_heads, each = static_cast<int64_t>(a.suffix_tiles) * a.kv_heads, suffix_units = each * s->batch;
    auto split_prefix = [&](int64_t n) { a.prefix_splits = prefix ? splits_of(a.prefix_len, prefix_units, n, kMinChunk, &a.prefix_chunk) : 0; };
    const int64_t slots = wanted(p->prefix_form), own_slots = wanted(p->suffix_form);
    const int64_t part_keys = (p->prefix_form == MANY_256 ? kPartKeys : kPartKeys / 2) * all / (static_cast<int64_t>(a.prefix_tiles) * kFormRows[p->prefix_form]) + 1;
    split_prefix(p->prefix_form == FEW || !prefix ? slots : prefix_units * prefix_splits_of(a.prefix_len, prefix_units, slots, part_keys, 4));
    // Where the sequences fill the chip, a workgroup goes over all of a sequence's keys and joins the prefix's parts: no parts of the sequences'
    // own (64 x 8 nodes over 1000 e4m3 keys 26.2 us in place of 38.7, 64 x 64 over 4096 bf16 338 in place of 465).  So also where one launch is
    // all there is to few keys (8 nodes over 301 10.2, with two launches 10.8; over 700 13.6 and 11.6; beside a prefix it is not: 6 x 2 over 4284 and
    // up to 12 of 256 23.0, joined by the sequences 30.3).  With few rows, whose parts are small,
    // long sequences are cut until there are two workgroups a CU (40 sequences over 8000 e4m3 keys 90.6, cut 70.5; 64 x 2 over 4000 the same).
    // Beside a prefix they are so where one launch fills places that they alone leave idle (36 x 4 over 8000 and up to 700 bf16 keys 47.6, joined by the
    // sequences 60.0, 8 x 20 over 4000 and 900 39.6 and 48.5; 64 x 4 over 8000 and 700, which fill the chip, 80 and 70).
    // With many rows, whose parts are large, they are cut where that fills places for long: 32 x 16 nodes of 32 heads (256 workgroups in 512 places)
    // over up to 1500 bf16 keys 34.0 us, cut 39.5, over 2500 50.7 and 48.1, 8000 146 and 112; 48 x 16 over 2500 75.4 and 79.9, 8000 252 and 214; 62 x
    // 16 over 8000 281 and 279.
    // Fewer workgroups than that are cut where a whole sequence takes longer: 12 x 5 nodes of 40 heads of 256 over 740 fp16 keys 16.5 us, whole 24.5, 17 x 40
    // of 16 of 128 over 900 25.2 and 32.7, over 420 24.1 and 21.1, 40 x 40 of 16 over 620 38.5 and 25.8, 60 x 30 of 8 of 64 over 800 e4m3 24.9 and 16.2.
    const bool brief = !prefix && width <= apart(0, suffix_units, own_slots);
    const bool fills = p->suffix_form != FEW ? brief || (suffix_units >= kFinishUnits && width * (own_slots - suffix_units) <= kShort * own_slots)
                                             : suffix_units >= (prefix ? own_slots : width * key_bytes > kLong ? 2 * kFinishUnits : kFinishUnits) || (width <= kShort / 2 && !prefix);
    p->finish = suffix && a.prefix_splits <= kFinishSplits && fills;
    if (p->finish && p->suffix_form == FEW) p->suffix_form = few(suffix_units);
    if (p->finish && !prefix) p->prefix_form = p->suffix_form;
    if (suffix) {
        a.suffix_splits = 1;
        if (!p->finish) {
            // As many pieces as there are places, less the half piece that a sequence ends with; where that is less than a piece a sequence, for
            // twice the places.  (With 16 rows or 4 a sequence over bf16 keys, in place of 4 pieces a sequence: 16 x 16 nodes of 32 heads over up
            // to 4000 37.1 us, so 44.8; 12 x 32 of 40 over 8000 89 and 102; 16 x 4 over 8000 50.3 and 58.6; 12 x 2 of 8 over 20000 e4m3 47.2 and
            // 60.5.  Heads of 256: 16 x 4 of 64 over 3000 40.1 and 56.1, 28 x 8 over 2000 for twice the places 53, else 61.6.)
            // The shortest is two turns; heads of 64, whose turns are short, four (2 x 20 of 64 heads over 1142 15.2 us, with two 16.4; 4 x 32 of 256
            // over 1200 25.6 and 22.6, 1 x 64 of 128 over 2000 22.8 and 20.9).
            a.cut_least = p->suffix_form == FEW || p->dp > 64 ? kMinChunk : 2 * kMinChunk;
            const int64_t most = std::min<int64_t>((width * s->batch + a.cut_least - 1) / a.cut_least, kMaxSplits - 1);
            const int64_t places = own_slots / each, ends = 1 + s->batch / 2, pieces = (places - ends >= s->batch ? places : 2 * places) - ends;
            a.cut_parts = static_cast<int32_t>(std::clamp<int64_t>(std::max<int64_t>(pieces, s->batch), 1, most));
            if (prefix && p->prefix_form == FEW) {
                const int64_t own_blocks = std::min<int64_t>(a.cut_parts + s->batch, (width * s->batch + a.cut_least - 1) / a.cut_least) * each;
                split_prefix(std::max(slots / 2, slots - own_blocks));
            } else if (prefix) {
                // The prefix's share of the places, as if sequences were half as long as they may be (17 x 30 nodes of 16 heads over 10062 fp16 keys of 96
                // and up to 1495 77.8 us, in half the places 93.8; 16 x 16 of 32 over 16000 and 1500 110 and 133, over 2000 and 1500 54.7 in all of them).
                const int64_t share = 2ll * a.prefix_len * slots / (2ll * a.prefix_len + width);
                split_prefix(prefix_units * std::min((share + prefix_units - 1) / prefix_units, prefix_splits_of(a.prefix_len, prefix_units, slots, part_keys, 1)));
            }
        }
        // the longest first where not all start at once (32 x 64 nodes over up to 4096 keys 170 us, in their order 214; where all start, 1.5 us are lost)
        a.sorted = p->finish && s->batch <= 64 && suffix_units > own_slots;
        p->suffix_blocks = round_up(a.kv_heads * (p->finish ? static_cast<int64_t>(s->batch) : a.cut_parts + static_cast<int64_t>(s->batch)), 8) * a.suffix_tiles;
    }
    if (p->dp > 128 && p->prefix_form == FEW) p->suffix_form = p->prefix_form = FEW_8;
    p->prefix_blocks = round_up(static_cast<int64_t>(a.prefix_splits) * a.kv_heads, 8) * a.prefix_tiles;
    // parts of a sequence
    const int64_t parts = static_cast<int64_t>(a.prefix_splits) * s->batch + (a.cut_parts ? a.cut_parts + static_cast<int64_t>(s->batch) : 0);
    p->bytes = parts * s->q_len * s->q_heads * (4ll * a.d + 8);
    return fits(*p);
}

// Up to here a row is joined by several workgroups, each of some of its columns: 15 rows of 256 in 255 parts 20.6 us a call in place of 27.6, 4 of 128
// 20.7 and 22.9; 384 of 256 40.7 and 41.5, 512 of 256 25.1 in place of 24.1.
constexpr int64_t kNarrowRows = 256;

// What joins a row's parts: a wave, a workgroup, or a workgroup for each kJoinColumns of its elements.
enum TreeJoin { JOIN_WAVE, JOIN_GROUP, JOIN_COLUMNS };
inline TreeJoin tree_join_of(const Plan& p)
{
    return p.rows >= kJoinRows ? JOIN_WAVE : p.rows <= kNarrowRows && p.a.d > kJoinColumns ? JOIN_COLUMNS : JOIN_GROUP;
}

}  // namespace serving
