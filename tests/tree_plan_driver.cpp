// Which launches attention of trees takes for a shape, for tests/tree_paths.py.  Host code only.
// One shape per line: batch nodes q_heads kv_heads d page_size pages prefix_len suffix_width dtype format; one line of output for each:
// the status, and where it is 0 the padded head, form of the prefix's rows (- without), form of a sequence's (- without), how the sequences'
// keys come (whole, cut, inline: behind a prefix in the same workgroups, none), splits of the prefix, whether the longest come first, and
// what joins parts (own: the sequences' workgroups; wave, group, columns: see tree_join_of; -: nothing does).
#include <stdarg.h>
#include <stdio.h>

#include "treeattn_plan.h"

int addrms_host::fail(int status, const char*, ...) { return status; }

using namespace serving;

int main()
{
    static const char* const kJoins[] = {"wave", "group", "columns"};
    static const char* const kForms[] = {"few", "64", "128", "256", "few8"};
    prefixattn_shape s = {};
    long long pages, prefix, width;
    while (scanf("%d %d %d %d %d %d %lld %lld %lld %d %d", &s.batch, &s.q_len, &s.q_heads, &s.kv_heads, &s.d, &s.page_size, &pages, &prefix, &width, &s.dtype, &s.format) == 11) {
        s.pages = pages, s.prefix_len = prefix, s.suffix_width = width;
        Plan p;
        const int st = tree_plan_of(&s, &p);
        if (st != ADDRMS_OK || p.rows == 0) {
            printf("%d\n", st);
            continue;
        }
        const AttnArgs& a = p.a;
        const bool own = p.suffix_blocks != 0;
        const char* const join = p.finish ? (a.prefix_splits ? "own" : "-") : kJoins[tree_join_of(p)];
        printf("0 %d %s %s %s %d %d %s\n", p.dp, a.prefix_splits ? kForms[p.prefix_form] : "-", own ? kForms[p.suffix_form] : "-",
               a.inline_len ? "inline" : !own ? "none" : a.cut_parts ? "cut" : "whole", a.prefix_splits, a.sorted, join);
    }
    return 0;
}
