// Whether calls with shared prefixes have at least the bits that attention over the same places in one row has (csrc/clear_attend_shape.cpp): where that
// goes by tiles of few rows, all of their walks do, or take weights as two numbers of the type.
#include <cstdio>

#include "clear_internal.h"

int main()
{
    int bad = 0, fewer = 0, calls = 0;
    for (uint32_t tokens : {1u, 2u, 7u, 16u, 64u, 65u, 250u, 1000u, 4096u, 20000u})
        for (uint32_t requests : {1u, 2u, 5u, 64u, 97u, 1000u})
            for (uint32_t group : {1u, 4u, 7u, 8u, 9u, 28u, 129u})
                for (uint32_t kv_heads : {1u, 8u})
                    for (uint32_t head : {64u, 128u, 256u})
                        for (uint32_t window : {0u, 1u, 100u, 4096u})
                            for (uint32_t prefix : {1u, 10u, 100u, 2048u, 60000u})
                                for (uint32_t own : {1u, 4u, 40u, 1000u})
                                    for (uint32_t prefixes : {0u, 1u, 6u}) {
                                        she_attend_shared_args a{};
                                        a.tokens = tokens, a.requests = requests, a.q_heads = group * kv_heads, a.kv_heads = kv_heads, a.head = head, a.window = window;
                                        a.prefix_width = prefix, a.table_width = own, a.page_size = 16, a.prefixes = prefixes;
                                        she_attend_pages_args b = she::clear::shared_behind(a);
                                        b.table_width += a.prefix_width;
                                        const she::clear::SharedShape s = she::clear::shared_shape(a, 256);
                                        const bool many = !s.behind.few || (!s.whole && prefixes && !s.prefix.few);
                                        calls++;
                                        if (many && !s.two) fewer++;
                                        if (many && !s.two && (she::clear::attend_shape(b, 256).few || tokens * group <= 32 * requests) && bad++ < 10)
                                            std::printf("%u tokens of %u requests, %u heads for each of %u of %u, window %u, %u and %u columns, %u prefixes\n", tokens, requests, group,
                                                        kv_heads, head, window, prefix, own, prefixes);
                                    }
    std::printf("%d calls, %d with one number\n", calls, fewer);
    return bad || !fewer || fewer == calls;
}
