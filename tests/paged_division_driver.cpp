// Driver for tests/test_paged_division.py: how a paged attention call of many rows is divided over its workgroups, with the
// kernel's own arithmetic (csrc/paged_division.h) on the CPU.  Every tile of every unit has to belong to one workgroup, and what the
// kernel that adds up the partials takes for granted has to hold: a split unit's parts are those of consecutive workgroups, at
// least a tile each, and as many as are described.
//
// quotients | small (random calls, tile by tile) | large (calls whose counts pass 2^39 and 2^53)
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <random>
#include <vector>

#include "paged_division.h"

using namespace pd;

#define CHECK(x, ...)                                            \
    do {                                                         \
        if (!(x)) {                                              \
            printf("FAILED %s:%d %s: ", __FILE__, __LINE__, #x); \
            printf(__VA_ARGS__);                                 \
            printf("\n");                                        \
            exit(1);                                             \
        }                                                        \
    } while (0)

constexpr int R = 256, TK = 64, kLeast = 4;
typedef PagedUnits<R, TK> Units;
struct Seq {
    int rows, len;
};

static void divide(const char *name, int hq, int hkv, const std::vector<Seq> &seqs, int W, bool each_tile)
{
    const int G = hq / hkv;
    struct Held {
        Units s;
        long long at;
        long long unit;
    };
    std::vector<Held> held;
    __int128 exact = 0;
    long long total = 0, units = 0;
    for (const Seq &q : seqs) {
        const Units s((q.rows * G + R - 1) / R, q.rows, q.len, G);
        held.push_back({s, total, units});
        total += hkv * s.all;
        units += (long long)hkv * s.units;
        for (int u = 0; u < s.units && s.units < 100000; ++u) exact += (__int128)hkv * s.count(u);
        if (s.units >= 100000) exact += (__int128)hkv * ((__int128)s.each * s.units + (__int128)R * s.units * (s.units + 1) / 2);
    }
    CHECK(exact == total && units < 1ll << 31, "%s: count %lld", name, total);
    const long long per = paged_part_count<TK>(total, W, kLeast, G), margin = paged_margin<TK>(per, G);
    CHECK(total == 0 || (__int128)per * W > total, "%s: %d parts of %lld do not hold %lld", name, W, per, total);
    CHECK(per == kLeast * TK * G || (__int128)(per - 1) * W <= total, "%s: %d parts of %lld for %lld", name, W, per, total);
    std::vector<PagedCut> cuts;
    for (int w = 0; w <= W; ++w) {
        PagedCut c = {(int)units, 0};
        const __int128 border = (__int128)w * per;
        if (border < total) {
            size_t b = 0;
            while (border >= (__int128)held[b].at + hkv * held[b].s.all) ++b;
            c = held[b].s.cut((long long)border - held[b].at, margin);
            c.unit += (int)held[b].unit;
        }
        cuts.push_back(c);
    }
    CHECK(cuts[0].unit == 0 && cuts[0].tile == 0 && cuts[W].unit == units && cuts[W].tile == 0, "%s: %d.%d to %d.%d of %lld units", name, cuts[0].unit,
          cuts[0].tile, cuts[W].unit, cuts[W].tile, units);
    auto unit_of = [&](int unit, long long *u0, long long *u1, int *tiles) {
        size_t b = held.size() - 1;
        while (held[b].unit > unit || held[b].s.units == 0) --b;
        const Units &s = held[b].s;
        const int in = (int)(unit - held[b].unit), g = in / s.units, i = in % s.units, u = s.tile(i);
        *u0 = held[b].at + g * s.all + s.ahead(i);
        *u1 = *u0 + s.count(u);
        *tiles = s.tiles(s.seen(u));
    };
    int split = 0;
    for (int w = 1; w <= W; ++w) {
        const PagedCut &x = cuts[w - 1], &y = cuts[w];
        CHECK(y.unit > x.unit || (y.unit == x.unit && (y.tile > x.tile || (y.tile == 0 && x.tile == 0))), "%s: border %d at %d.%d behind %d.%d", name, w, y.unit,
              y.tile, x.unit, x.tile);
        if (!y.tile) continue;
        long long u0, u1;
        int tiles, inside = 1;
        unit_of(y.unit, &u0, &u1, &tiles);
        CHECK(y.tile > 0 && y.tile < tiles, "%s: border %d at tile %d of %d", name, w, y.tile, tiles);
        if (x.unit == y.unit && x.tile) continue;
        while (w + inside <= W && cuts[w + inside].unit == y.unit && cuts[w + inside].tile) ++inside;
        CHECK(paged_parts(u0, u1, margin, per) == inside + 1, "%s: unit %d has %d parts, not %d", name, y.unit, inside + 1, paged_parts(u0, u1, margin, per));
        ++split;
    }
    if (each_tile) {
        for (int unit = 0; unit < units; ++unit) {
            long long u0, u1;
            int tiles;
            unit_of(unit, &u0, &u1, &tiles);
            int next = 0;
            for (int w = 0; w < W; ++w) {
                const PagedCut &x = cuts[w], &y = cuts[w + 1];
                const int to = y.unit + (y.tile > 0);
                if (unit < x.unit || unit >= to) continue;
                const int lo = unit == x.unit ? x.tile : 0, hi = unit == to - 1 && y.tile ? y.tile : tiles;
                CHECK(lo == next && hi > lo, "%s: unit %d, workgroup %d: %d .. %d behind %d", name, unit, w, lo, hi, next);
                next = hi;
            }
            CHECK(next == tiles, "%s: unit %d: %d of %d tiles", name, unit, next, tiles);
        }
    }
    if (!each_tile) printf("ok %s: count %.3g, %lld units, %d split, part %.3g\n", name, (double)total, units, split, (double)per);
}

static void quotients()
{
    std::mt19937_64 r(1);
    for (int i = 0; i < 4000000; ++i) {
        const int bits = 1 + (int)(r() % 62), less = (int)(r() % 62);
        const long long b = std::max<long long>(1, (long long)(r() >> 2 >> less));
        long long a = (long long)(r() >> (64 - bits));
        if (i % 3 == 0) a = a / b * b - (i % 2);     // multiples, and one below them
        a = std::max<long long>(a, 0);
        CHECK(paged_quotient64(a, b) == a / b, "%lld / %lld is %lld", a, b, paged_quotient64(a, b));
        if (a / b < 1ll << 31) CHECK(paged_quotient(a, b) == a / b, "%lld / %lld is %d", a, b, paged_quotient(a, b));
    }
}

static void small()
{
    std::mt19937 r(2);
    auto below = [&](int n) { return (int)(r() % (unsigned)n); };
    for (int i = 0; i < 6000; ++i) {
        const int G = 1 + below(i % 5 ? 12 : 300), hkv = 1 + below(6), n = 1 + below(i % 7 ? 6 : 40);
        std::vector<Seq> s;
        for (int b = 0; b < n; ++b) {
            const int rows = below(4) ? 1 + below(i % 3 ? 600 : 60) : 0;
            s.push_back({rows, below(8) ? rows + below(i % 2 ? 9000 : 300) : below(rows + 1)});
        }
        char name[32];
        snprintf(name, sizeof(name), "random call %d", i);
        divide(name, G * hkv, hkv, s, i % 4 ? 256 : 1 + below(256), true);
    }
}

static void large()
{
    const int K = 1024, M = K * K;
    divide("a prompt of 20000, 32 heads on 8", 32, 8, {{20000, 20000}}, 256, false);
    divide("a prompt of 131072, 128 heads on 1", 128, 1, {{128 * K, 128 * K}}, 256, false);
    divide("32768 rows behind 524288, 128 on 1", 128, 1, {{32 * K, 544 * K + 32 * K}}, 256, false);
    divide("1024 rows behind 131072, 1024 on 1", 1024, 1, {{K, 129 * K}}, 256, false);
    divide("8192 rows behind 2^20, 128 on 1", 128, 1, {{8 * K, M + 8 * K}}, 256, false);
    divide("a prompt of 400000, 128 on 8", 128, 8, {{400000, 400000}}, 256, false);
    divide("a prompt of 524288, 128 on 8", 128, 8, {{512 * K, 512 * K}}, 256, false);
    divide("65536 rows behind 2^20, 128 on 8", 128, 8, {{64 * K, M + 64 * K}}, 256, false);
    divide("a prompt of 1.5 million, 32 on 8", 32, 8, {{1500000, 1500000}}, 256, false);
    divide("long and short ones, 128 on 1", 128, 1, {{3, 3}, {200000, 300000}, {0, 7}, {1, 900}, {70000, 200 * M}, {700, 700}}, 256, false);
    divide("2^20 rows at the end of 2^30, 1024 on 1", 1024, 1, {{M, 1 << 30}}, 256, false);
    divide("2^20 rows at the end of 2^30, 1024 on 1024", 1024, 1024, {{M, 1 << 30}}, 256, false);
    divide("the same by three workgroups", 1024, 1, {{M, 1 << 30}}, 3, false);
    divide("4096 sequences of 16 rows at the end of 2^30, 1024 on 64", 1024, 64, std::vector<Seq>(4096, Seq{16, 1 << 30}), 256, false);
}

int main(int argc, char **argv)
{
    if (argc != 2) return 2;
    if (!strcmp(argv[1], "quotients")) quotients();
    else if (!strcmp(argv[1], "small")) small();
    else if (!strcmp(argv[1], "large")) large();
    else return 2;
    return 0;
}
