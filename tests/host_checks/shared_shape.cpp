// Prints what csrc/clear_attend_shape.cpp decides for calls with shared prefixes: a call a line on the input (tokens, requests, query heads, key
// heads, head, window, prefixes, prefix columns, columns, page size), and for each the walks, their pieces and the scratch.
#include <cstdio>

#include "clear_internal.h"

int main()
{
    she_attend_shared_args a{};
    while (std::scanf("%u %u %u %u %u %u %u %u %u %u", &a.tokens, &a.requests, &a.q_heads, &a.kv_heads, &a.head, &a.window, &a.prefixes, &a.prefix_width, &a.table_width,
                      &a.page_size) == 10) {
        const she::clear::SharedShape s = she::clear::shared_shape(a, 256);
        std::printf("%s %s %u %u %zu\n", s.whole ? "whole" : s.prefix.few ? "few" : "tile", s.behind.few ? "few" : "tile", s.prefix.splits, s.behind.splits,
                    she::clear::shared_scratch(a, s));
    }
    return 0;
}
