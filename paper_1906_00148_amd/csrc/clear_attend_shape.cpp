// Which kernel an attention call takes, and the pieces that it is cut into (clear_attend.hip has the kernels).
#include <algorithm>

#include "clear_internal.h"

namespace she { namespace clear {

AttendShape attend_shape(const she_attend_pages_args &a, uint32_t cus)
{
    AttendShape s{};
    const uint64_t group = a.q_heads / a.kv_heads, longest = std::min<uint64_t>((uint64_t)a.table_width * a.page_size, 0x7FFFFFFF);
    const uint64_t rows = a.tokens * group;
    if (!cus) cus = 1;
    // places of a tile at most: a window's, those that its later tokens see further, and those before it down to a multiple of 32
    const auto span = [&](uint64_t tile) { return a.window ? std::min<uint64_t>(longest, (uint64_t)a.window + tile + 31) : longest; };
    // One of the two kernels takes all of a call.  k_attend_tile computes 128 rows whether they are there or not, and k_attend_few reads
    // the places once for every 16 rows.  Either measured (few, tile; 8 key heads of 128, bf16; us; rows of each request at a key head):
    //    one request:    8 rows    16       32       64      128          16 requests:   4 rows     16        32        64
    //    1000 places    13, 23   13, 25   13, 25   15, 26   17, 28         500 places   17, 20    20, 20    24, 20    30, 20
    //    8000           17, 26   18, 26   23, 27   38, 28   57, 30        1000          21, 24    28, 30    34, 30    52, 35
    //    32768          38, 50   40, 51   56, 52   99, 54  172, 59        4000          64, 67    86, 65    92, 66   179, 90
    //                                                                    16384         226, 218  294, 209  325, 211  634, 293
    // Where the work is small the first kernel's short way counts.  It also has single tokens of up to 8 rows, whose caches may have
    // different lengths: its small pieces even them out (200 tokens over 1 to 3000 places 245, 268; 64 over 1 to 16384 421, 429).
    s.few = rows * span(FEW_ROWS) <= 1u << 18 || (a.tokens <= a.requests && group <= FEW_ROWS / 2);
    const uint64_t tile = s.few ? FEW_ROWS : TILE_ROWS, places = span(tile);
    s.slots = a.requests == 1 ? ceil_div(rows, tile) : rows / tile + a.requests;
    if (s.few) {
        // Pieces for two workgroups per compute unit: shorter ones (for eight) cost more to join than they gain, 128 us and not 78 for
        // a token over 32768 places when every row was joined by one wavefront.
        const uint64_t share = ceil_div(s.slots * a.kv_heads * places / (2 * cus), 128) * 128;
        s.chunk = (uint32_t)std::min<uint64_t>(MOST_CHUNK, std::max<uint64_t>(256, share));
        // Up to 32 workgroups for each that runs at once, or eight pieces, even the requests' lengths out.  A table of more places than
        // such pieces have, as wide as a context that few requests fill, does not make scratch and workgroups for more of them: a
        // request that does fill it has longer pieces.  Tables of 131072 places, 8 key heads of 128, in us with a piece for every 2048
        // places, at most 16 workgroups, and 32: one request of 131000 places among 63 of up to 300 841, 915, 855, among 1023 4003,
        // 2160, 2170; 1024 of up to 300 2222, 432, 431; 64 of up to 60000 1503, 1476, 1484.
        const uint64_t most = std::max<uint64_t>(8, ceil_div(32 * 2 * cus, s.slots * a.kv_heads));
        s.splits = (uint32_t)std::max<uint64_t>(1, std::min(most, ceil_div(places, s.chunk)));
        return s;
    }
    // How many tiles there will be: every request has one, and its last is half full on average.
    const uint64_t groups = std::max<uint64_t>({1, s.slots - a.requests / 2, std::min<uint64_t>(a.requests, a.tokens)}) * a.kv_heads;
    // Workgroups that run at once, and pieces that make `rounds` rounds of them: the fewest places one after the other, where a workgroup
    // costs as much as 256 of them beside its own.  Pieces are written and read again, 8 bytes an element of every row where a place is
    // 4, at a quarter of the rate, and a launch more is 128 places.  So tiles of many rows stay whole (24 requests of up to 700 tokens,
    // 16 heads of 64, a window of 1024: 57 us, 82 in two pieces), and few tiles over many places are cut until all compute units have
    // work (64 tokens and one of 100 more over 16384 places each: 1021 us whole, 840 in five pieces).  Single tokens' lengths may
    // differ: half the places on average, and a whole piece at the end.
    const uint64_t at_once = cus * (a.head <= 64 ? 3 : a.head <= 128 ? 2 : 1);
    uint64_t best = ~0ull;
    for (uint64_t rounds = 1; rounds <= 8; rounds++) {
        const uint64_t parts = std::max<uint64_t>(1, rounds * at_once / groups);
        const uint64_t chunk = std::max<uint64_t>(512, ceil_div(ceil_div(places, parts), STEP) * STEP);
        const uint64_t splits = std::max<uint64_t>(1, ceil_div(places, chunk)), longest_piece = std::min(chunk, places);
        uint64_t cost = ceil_div(groups * splits, at_once) * (longest_piece + 256);
        if (a.requests > 1 && a.tokens <= a.requests) cost += groups * (places + (splits + 1) * 256) / (2 * at_once) + longest_piece;
        if (splits > 1) cost += 128 + 8 * rows * a.kv_heads * splits / at_once;
        if (cost >= best) continue;
        best = cost;
        s.chunk = (uint32_t)chunk;
        s.splits = (uint32_t)splits;
    }
    return s;
}

size_t attend_pieces(const she_attend_pages_args &a, const AttendShape &s)
{
    return s.splits > 1 ? (size_t)a.tokens * a.q_heads * s.splits : 0;
}

size_t attend_scratch(const she_attend_pages_args &a, const AttendShape &s)
{
    return attend_pieces(a, s) * (a.head * sizeof(float) + sizeof(float2));
}

}}  // namespace she::clear
