// csrc/clear_reach.h against its definition over places, one by one or in 128 bits, with lengths up to the largest number of 32 bits.
#include <cstdio>

#include "clear_reach.h"

using she::clear::first_behind;
using she::clear::last_behind;

int main()
{
    int bad = 0;
    const auto wrong = [&](const char *what, long long place, long long window, long long own, long long missing, long long got, long long want) {
        if (bad++ < 10) std::printf("%s: place %lld, window %lld, %lld of the prefix and %lld missing: %lld, not %lld\n", what, place, window, own, missing, got, want);
    };
    // small numbers: the first of the row that is less than a window before the token
    for (int place = 0; place < 9; place++)
        for (unsigned window = 0; window < 20; window++)
            for (int own = 0; own < 6; own++)
                for (int missing = 0; missing < 6; missing++) {
                    int want = 0;
                    const auto at = [&](int i) { return i < own ? i : i + missing; };                  // of the place i of the row, counting those that are missing
                    while (window && at(own + place) - at(want) >= (int)window) want++;
                    const int got = first_behind(place, window, own, missing);
                    if (got != want) wrong("first", place, window, own, missing, got, want);
                    if (last_behind(place, own) != own + place) wrong("last", place, window, own, missing, last_behind(place, own), own + place);
                }
    // large ones: as long as a table has a column it is exact, and never before it
    const long long most = 0x7FFFFFFF, table = 1ll << 27;
    for (long long place : {0ll, 1ll, 100ll, table, most / 2, most - 70, most - 1})
        for (long long window : {0ll, 1ll, 40ll, table, most - 60, most, most + 1, 2 * most, 2 * most + 1})
            for (long long own : {0ll, 1ll, 64ll, 1ll << 26})
                for (long long missing : {0ll, 1ll, most - (1ll << 26)}) {
                    const __int128 low = (__int128)place - window + 1;
                    __int128 want = !window ? 0 : low >= 0 ? low + own : low + own + missing;
                    if (window && low < 0) want = want < 0 ? 0 : want > own ? own : want;
                    const int got = first_behind(place, (uint32_t)window, (int)own, missing), end = last_behind(place, (int)own);
                    if (want < table ? got != want : got < table || got == most) wrong("first", place, window, own, missing, got, (long long)want);
                    if (place + own < table ? end != place + own : end < table || end == most) wrong("last", place, window, own, missing, end, place + own);
                }
    return bad != 0;
}
