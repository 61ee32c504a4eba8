// How tiles in a row are shared out among units (csrc/hp_share.hpp) against whole numbers of 128 bits.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "hp_share.hpp"

static void same(const char *what, int64_t got, int64_t want, int total, int unit, int units) {
    if (got == want) return;
    std::printf("%s: %lld instead of %lld, %d tiles, unit or tile %d of %d units\n", what, (long long)got, (long long)want, total, unit, units);
    std::exit(1);
}

static void look(int total, int units) {
    const auto first = [&](int64_t u) { return (int64_t)((__int128)total * u / units); };
    const auto unit = [&](int u) {
        same("first", hp::first_of(total, u, units), first(u), total, u, units);
        if (u == units) return;
        // the unit's first and last tile and the next one's first
        for (int64_t t : {first(u), first(u + 1) - 1, first(u + 1)}) {
            if (t < 0 || t >= total) continue;
            int64_t lo = 0, hi = units - 1;               // the last unit that begins at t or before, and is not empty
            while (lo < hi) {
                const int64_t mid = (lo + hi + 1) / 2;
                if (first(mid) <= t) lo = mid;
                else hi = mid - 1;
            }
            same("unit", hp::unit_of(total, (int)t, units), lo, total, (int)t, units);
        }
    };
    const int most = units < 300 ? units : 300;
    for (int u = 0; u <= most; ++u) unit(u);
    for (int i = 0; i < 300; ++i) unit((int)((int64_t)units * i / 300));
    unit(units);
}

int main() {
    for (int total = 1; total < 400; ++total)
        for (int units = 1; units <= total && units < 70; ++units) look(total, units);
    const int totals[] = {511, 1024, 4097, 65535, 1000003, 16777217, 1 << 30, INT_MAX - 1, INT_MAX};
    const int many[] = {1, 2, 3, 7, 96, 255, 256, 768, 1023, 1024};
    for (int total : totals)
        for (int units : many)
            if (units <= total) look(total, units);
    std::puts("ok");
    return 0;
}
