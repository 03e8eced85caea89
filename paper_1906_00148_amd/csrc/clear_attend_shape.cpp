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

she_attend_pages_args shared_behind(const she_attend_shared_args &a)
{
    she_attend_pages_args b{};
    b.type = a.type;
    b.tokens = a.tokens;
    b.requests = a.requests;
    b.q_heads = a.q_heads;
    b.kv_heads = a.kv_heads;
    b.head = a.head;
    b.window = a.window;
    b.scale = a.scale;
    b.q = a.q;
    b.q_token = a.q_token;
    b.q_head = a.q_head;
    b.k_pages = a.k_pages;
    b.v_pages = a.v_pages;
    b.page_stride = a.page_stride;
    b.slot_stride = a.slot_stride;
    b.page_head = a.page_head;
    b.pages = a.pages;
    b.page_size = a.page_size;
    b.table = a.table;
    b.table_stride = a.table_stride;
    b.table_width = a.table_width;
    b.starts = a.starts;
    b.lengths = a.lengths;
    b.out = a.out;
    b.out_token = a.out_token;
    b.out_head = a.out_head;
    return b;
}

SharedShape shared_shape(const she_attend_shared_args &a, uint32_t cus)
{
    SharedShape s{};
    if (!cus) cus = 1;
    const uint64_t group = a.q_heads / a.kv_heads, rows = a.tokens * group, places = (uint64_t)a.prefix_width * a.page_size, own = (uint64_t)a.table_width * a.page_size;
    const she_attend_pages_args call = shared_behind(a);
    s.behind = attend_shape(call, cus);
    // Never fewer bits than she_attend_pages has for the same places, which takes few rows and single tokens with two numbers for a weight: by tiles of many
    // rows with one, these would be off by 0.0023 of a bf16 result and not 0.0017.  The second product costs least where a wavefront waits otherwise, so
    // other calls have it up to 32 rows of a request (one number, two; 8192 places, 8 key heads of 128, bf16; us; rows at a key head on average):
    //    64 requests:  4 rows  32.3, 34.9   6    44.2, 49.0   18   71.7, 83.3   34  108.8, 139.0   66   213.7, 273.5
    //    24 requests:  4 rows  25.3, 27.7   10   30.9, 33.4   18   43.9, 49.2   34   63.9, 74.6    258  294.4, 371.1
    she_attend_pages_args both = call;
    both.table_width += a.prefix_width;
    s.two = rows <= 32 * (uint64_t)a.requests || attend_shape(both, cus).few;
    if (!a.prefixes) return s;
    // Few places, which workgroups that run at once walk in one launch: joining a prefix's pieces with the requests' own takes a second one.
    // (Both, one launch; us on the device; single tokens with 40 places behind a prefix of 60, 330 and 450 places.)
    //    2 requests, 8 / 2 heads of 64     9.9, 6.4   10.9, 9.5   11.3, 10.7       40 requests    10.5, 6.7   11.6, 9.6   11.7, 11.0
    //    2 requests, 32 / 8 of 128        11.7, 7.6   13.7, 11.7  13.7, 13.4       40 requests    13.7, 9.0   16.5, 15.0  16.3, 17.2
    //    2 requests, 8 / 8 of 256         14.3, 10.4  18.6, 18.3  18.5, 20.9       40 requests    23.7, 19.9  24.6, 34.7  24.6, 41.9
    const uint64_t few_slots = a.requests == 1 ? ceil_div(rows, FEW_ROWS) : rows / FEW_ROWS + a.requests, few_groups = few_slots * a.kv_heads;
    const uint64_t few_places = few_groups <= cus ? (a.head <= 128 ? 512 : 384) : few_groups <= 2 * cus && a.head <= 128 ? 384 : 0;
    if (s.behind.few && places + own <= few_places) {
        s.whole = true;
        s.behind.slots = few_slots;
        s.behind.splits = 1;
        s.behind.chunk = 512;
        return s;
    }
    // rows of a prefix: the host knows their average
    const uint64_t each = ceil_div(rows, a.prefixes);
    s.prefix.few = s.behind.few && (each <= FEW_ROWS || each * places <= 1u << 18);
    const uint64_t tile = s.prefix.few ? FEW_ROWS : TILE_ROWS;
    s.prefix.slots = a.prefixes == 1 ? ceil_div(rows, tile) : rows / tile + a.prefixes;
    s.prefix.chunk = s.prefix.few ? 256 : 512;
    // Costs in places that a workgroup with a compute unit to itself walks.  It costs as much as 256 of them beside its own, two on a unit take
    // 1.44 times as long as one, and a row of a piece, written and read again, is a 94th.
    const uint64_t share = a.head > 128 ? 100 : 72, at_most = std::max<uint64_t>(1, std::min<uint64_t>(64, ceil_div(places, s.prefix.chunk)));
    const auto time = [&](uint64_t groups, uint64_t walk, uint64_t beside) {
        return std::max(walk + 256, (ceil_div(groups, cus) * (walk + 256) + beside) * share / 100);
    };
    // the requests' own places, of which the host knows the most that there may be: half of them, a tile of few rows at half the price
    const uint64_t behind = ceil_div(s.behind.slots * a.kv_heads * s.behind.splits, cus) * (own / (2 * s.behind.splits) + 256) / (s.behind.few ? 2 : 1);
    const uint64_t groups = a.prefixes * ceil_div(each, tile) * a.kv_heads, row = rows * a.kv_heads;
    uint64_t best = ~0ull;
    for (uint64_t splits = 1; splits <= at_most; splits++) {
        const uint64_t c = time(groups * splits, ceil_div(places, splits), behind) + row * (splits + s.behind.splits) / 94;
        if (c >= best) continue;
        best = c;
        s.prefix.splits = (uint32_t)splits;
    }
    // Or every request's tiles walk the prefix and its own places as one.
    if (s.behind.few) return s;
    const uint64_t tiles = std::max<uint64_t>(rows / TILE_ROWS + a.requests / 2, std::min<uint64_t>(a.requests, a.tokens)) * a.kv_heads;
    SharedShape w{};
    w.whole = true;
    w.two = s.two;
    w.behind.slots = a.requests == 1 ? ceil_div(rows, TILE_ROWS) : rows / TILE_ROWS + a.requests;
    uint64_t least = ~0ull;
    for (uint64_t splits = 1; splits <= std::max<uint64_t>(1, std::min<uint64_t>(64, ceil_div(places + own, 512))); splits++) {
        const uint64_t c = time(tiles * splits, ceil_div(places + own / 2, splits), 0) * 5 / 4 + (splits > 1 ? 128 + row * splits / 94 : 0);
        if (c >= least) continue;
        least = c;
        w.behind.splits = (uint32_t)splits;
        w.behind.chunk = (uint32_t)(ceil_div(ceil_div(places + own, splits), STEP) * STEP);
    }
    return least <= best ? w : s;
}

size_t shared_pieces(const she_attend_shared_args &a, const SharedShape &s)
{
    if (s.whole) return s.behind.splits > 1 ? (size_t)a.tokens * a.q_heads * s.behind.splits : 0;
    return (size_t)a.tokens * a.q_heads * (s.prefix.splits + s.behind.splits);
}

size_t shared_scratch(const she_attend_shared_args &a, const SharedShape &s)
{
    return shared_pieces(a, s) * (a.head * sizeof(float) + sizeof(float2));
}

}}  // namespace she::clear
