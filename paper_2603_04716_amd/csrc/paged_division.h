// The arithmetic of the division of a paged attention call with many rows, in whole numbers alone, so that it also runs on the host:
// what a unit counts, what a workgroup's part is, where its borders cut, how many parts a unit has.
//
// Row tile u of a sequence is counted with G (kUnitKeys + before) + R (u + 1), G times the keys that it sees and those that going from one
// unit to the next takes the time of; inside a unit the count is proportional to its tiles.  The units of a sequence and kv head are
// taken from both ends in turn (the last row tile, the first, the last but one, ..), which makes all pairs count the same: what is
// ahead of a unit has a closed form, and where the parts hold whole pairs, as those of equal prompts mostly do, nothing is split.
// A border closer than `margin` to an end of its unit moves there: a partial of few tiles costs more than the
// unevenness.  Every workgroup finds the same cut for a border, and as tiles count less than `per` each, cuts inside a unit are
// different tiles.  Of kUnitKeys 192, 256 and 384 a call of twelve chunks of 1 to 700 tokens behind up to 6000 takes 290, 288 and 290 us,
// with margins of an eighth, a 16th and a 32nd of a part 306, 288 and 289 us.
//
// How large it gets: a call has some 2^30 (token, head) rows at most (of more, queries and results would not fit the memory), so 2^22
// full units, each counted with up to 2^10 (2^30 + 2^9) + 2^30, and the last units of sequences add little: 4096 times the kv heads, with G
// times 2^30 each, are 2^52.  The count of a call thus stays below 2^62.1, but not below 2^53, where doubles are exact, and a
// workgroup's part not below 2^31.
#pragma once
#include <hip/hip_runtime.h>

namespace pd {

constexpr int kUnitKeys = 256;
constexpr int kCutTiles = 8;             // a unit of fewer tiles is never split

struct PagedCut {
    int unit, tile;
};

// floor(a / b), a >= 0, b > 0, of a quotient below 2^31, by way of double: a tenth of the instructions of the compiler's 64-bit
// division.  The quotient in double is off by less than 2^-20, so it is the floor or next to it.
__host__ __device__ inline int paged_quotient(long long a, long long b)
{
    int q = (int)((double)a / (double)b);
    if (a - q * b < 0) --q;
    if (a - q * b >= b) ++q;
    return q;
}
// The same of any quotient, a below 2^63 - 2^12: off by up to 2^11 after the first division, which the second one, of what is left, mends.
__host__ __device__ inline long long paged_quotient64(long long a, long long b)
{
    long long q = (long long)((double)a / (double)b);
    q += (long long)((double)(a - q * b) / (double)b);
    if (a - q * b < 0) --q;
    if (a - q * b >= b) ++q;
    return q;
}

template <int R, int TK>
struct PagedUnits {                      // of a sequence of n_rows rows at the end of len positions, and a kv head
    int units, rows, before, G;
    long long each, pair, all;           // each + R (u + 1): count of row tile u; count of a pair and of all units
    // (no units where another kernel has the sequence)
    __host__ __device__ inline PagedUnits(int n_units, int n_rows, int len, int group)
    {
        units = n_units;
        rows = n_rows * group;
        before = len - n_rows;
        G = group;
        each = (long long)group * (kUnitKeys + (before > 0 ? before : 0));
        pair = 2 * each + (long long)R * (units + 1);
        all = ahead(units);
    }
    __host__ __device__ inline int tile(int i) const { return i & 1 ? i >> 1 : units - 1 - (i >> 1); }      // row tile of unit i
    __host__ __device__ inline long long count(int u) const { return each + (long long)R * (u + 1); }
    __host__ __device__ inline long long ahead(int i) const { return (i >> 1) * pair + (i & 1 ? count(tile(i - 1)) : 0); }
    __host__ __device__ inline int seen(int u) const
    {
        const int end = R * (u + 1) < rows ? R * (u + 1) : rows, keys = before + (end - 1) / G + 1;
        return keys > 0 ? keys : 0;
    }
    __host__ __device__ inline int tiles(int seen) const { return seen > TK ? (seen + TK - 1) / TK : 1; }
    // (more rows than positions: the count says too little about the tiles)
    __host__ __device__ inline bool whole(int tiles) const { return tiles < kCutTiles || before < 0; }
    // the cut of a border y behind the sequence's first count, as a unit of the sequence and a tile of it
    __host__ __device__ inline PagedCut cut(long long y, long long margin) const
    {
        const int g = paged_quotient(y, all);
        y -= g * all;
        int i = 2 * paged_quotient(y, pair);
        y -= (i >> 1) * pair;
        const long long first_of_pair = count(tile(i));
        if (i + 1 < units && y >= first_of_pair) {
            ++i;
            y -= first_of_pair;
        }
        const long long of = count(tile(i));
        const int n = tiles(seen(tile(i)));
        const bool inside = !whole(n) && y >= margin && y <= of - margin;
        const bool next = !inside && 2 * y >= of;
        int at = 0;
        if (inside) {
            at = (int)((double)y * n / (double)of);
            at = at < 1 ? 1 : at > n - 1 ? n - 1 : at;
        }
        return PagedCut{g * units + i + next, at};
    }
};

// count of a workgroup, and what a border keeps from the ends of a unit
template <int TK>
__host__ __device__ inline long long paged_part_count(long long total, int workgroups, int least, int G)
{
    const long long even = paged_quotient64(total, workgroups) + 1, floor = (long long)least * TK * G;
    return even > floor ? even : floor;
}
template <int TK>
__host__ __device__ inline long long paged_margin(long long per, int G)
{
    const long long tiles = (long long)kCutTiles / 2 * TK * G;
    return per / 16 > tiles ? per / 16 : tiles;
}
// parts of a unit that is split, counted from u0 to u1: one more than the borders that cut inside of it
__host__ __device__ inline int paged_parts(long long u0, long long u1, long long margin, long long per)
{
    return 2 + paged_quotient(u1 - margin, per) - paged_quotient(u0 + margin + per - 1, per);
}

}  // namespace pd
