// Prints what attend_shape decides on 256 compute units for each call on the input: tokens, requests, query and key heads, head, window,
// the table's columns and the page size -> the kernel, tiles, places of a piece, pieces of a tile, bytes of scratch.
#include <cstdio>

#include "clear_internal.h"

int main()
{
    unsigned tokens, requests, q_heads, kv_heads, head, window, width, page;
    while (std::scanf("%u %u %u %u %u %u %u %u", &tokens, &requests, &q_heads, &kv_heads, &head, &window, &width, &page) == 8) {
        she_attend_pages_args a{};
        a.tokens = tokens; a.requests = requests; a.q_heads = q_heads; a.kv_heads = kv_heads; a.head = head;
        a.window = window; a.table_width = width; a.page_size = page;
        const she::clear::AttendShape s = she::clear::attend_shape(a, 256);
        std::printf("%s %llu %u %u %zu\n", s.few ? "few" : "tile", (unsigned long long)s.slots, s.chunk, s.splits, she::clear::attend_scratch(a, s));
    }
    return 0;
}
