// The division of a paged attention call's keys into work items, on the device (shared by its two kernels).
//
// A unit is a tile of R (token, head) rows of one sequence and kv head; an item is one of the chunks that a unit's keys are
// divided into.  Lengths are known on the device alone, so every workgroup works the division out for itself: the keys that
// all units have to read, divided by the items aimed for, is the chunk; a sequence of len keys and U units makes
// U ceil(len / chunk) items, and since U (len / chunk + 1) <= 2 U len / chunk where there is more than one chunk, the split
// ones are at most twice the items aimed for.  A thread keeps the counts of its own consecutive sequences and the
// sum of those before; nothing is stored per sequence.
#pragma once
#include <type_traits>

#include "paged.h"

namespace pd {

__device__ __forceinline__ float pexp2(float x) { return __builtin_amdgcn_exp2f(x); }

struct PagedItems {
    int chunk, total, split_units;       // keys of a chunk; items and split units of the call, per kv head
    int b0, b1;                          // this thread's sequences
    int first, own;                      // items ahead of them, and theirs
    int split, unit;                     // split items and split units ahead of them
    int start, rows, len;                // the first of them
};
struct PagedFound {
    int seq, at;                         // sequence of an item, and the item's place among the sequence's
    int units, chunks, start, rows, len; // of the sequence
    int split, unit;                     // split items and split units ahead of the sequence
};

// Sum over the lanes up to this one, by data-parallel moves: a cross-lane step through LDS would take ten times as long, and every
// workgroup waits for the division before its first load.
template <typename T>
__device__ __forceinline__ T wave_scan(T v)
{
    auto add = [&](auto CTRL, auto ROWS) {
        const int m = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(CTRL)::value, decltype(ROWS)::value, 0xf, true);
        v += __builtin_bit_cast(T, m);
    };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});    // one lane up, inside rows of 16
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});    // row 0 to 1, 2 to 3
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});    // lane 31 to rows 2 and 3
    return v;
}
// units of a sequence of n rows (none where another kernel has it)
template <int R>
__device__ __forceinline__ int paged_units(const PagedAttnArgs &a, int n)
{
    const int rows = n * a.G;
    return rows > a.rows_above && rows <= a.rows_most ? (rows + R - 1) / R : 0;
}
__device__ __forceinline__ int paged_chunks(int len, int chunk) { return max((len + chunk - 1) / chunk, 1); }
// f(sequence, first row, rows, positions) for a thread's sequences; the first one's fields are kept, most calls have no more
template <typename F>
__device__ __forceinline__ void paged_each(const PagedAttnArgs &a, const PagedItems &r, F f)
{
    if (r.b0 < r.b1) f(r.b0, r.start, r.rows, r.len);
    for (int b = r.b0 + 1; b < r.b1; ++b) {
        const int start = paged_start(a.p, b);
        f(b, start, paged_rows(a.p, b, start), paged_len(a.p, b));
    }
}
// LDS of the division
template <int NT>
struct PagedShared {
    float keys[NT / 64], rows[NT / 64];
    int own[NT / 64], split[NT / 64], unit[NT / 64];
    PagedFound found;
};
// By all NT threads.  Sums that only steer the division are fp32: every workgroup forms them in the same order, and the rows'
// is exact up to 2^24, which no call has more of.
template <int R, int NT>
__device__ __forceinline__ PagedItems paged_divide(const PagedAttnArgs &a, PagedShared<NT> &sh)
{
    const int n = a.p.n_seqs, per = (n + NT - 1) / NT, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    PagedItems r = {64, 0, 0, min((int)threadIdx.x * per, n), 0, 0, 0, 0, 0, 0, 0, 0};
    r.b1 = min(r.b0 + per, n);
    if (r.b0 < n) {
        r.start = paged_start(a.p, r.b0);
        r.rows = paged_rows(a.p, r.b0, r.start);
        r.len = paged_len(a.p, r.b0);
    }
    float keys = 0.f, rows = 0.f;
    paged_each(a, r, [&](int, int, int n_rows, int len) {
        keys += (float)paged_units<R>(a, n_rows) * (float)len;
        rows += (float)n_rows;
    });
    keys = wave_scan(keys);
    rows = wave_scan(rows);
    if (lane == 63) {
        sh.keys[wave] = keys;
        sh.rows[wave] = rows;
    }
    __syncthreads();
    keys = rows = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        keys += sh.keys[w];
        rows += sh.rows[w];
    }
    if (rows > (float)a.p.n_rows) return r;          // the sequences' rows overlap: no such call, and nothing is done
    // (1 + 2^-10: more than the roundings of the sum, so that the bound on the split items holds)
    const float chunk = keys * (float)a.p.Hkv * (1.0009765625f / (float)a.target);
    r.chunk = ((int)ceilf(fminf(fmaxf(chunk, (float)a.least), (float)((1 << 30) - 128))) + 63) & ~63;
    int own = 0, split = 0, unit = 0;
    paged_each(a, r, [&](int, int, int n_rows, int len) {
        const int u = paged_units<R>(a, n_rows), nc = paged_chunks(len, r.chunk);
        own += u * nc;
        split += nc > 1 ? u * nc : 0;
        unit += nc > 1 ? u : 0;
    });
    const int own_to = wave_scan(own), split_to = wave_scan(split), unit_to = wave_scan(unit);
    if (lane == 63) {
        sh.own[wave] = own_to;
        sh.split[wave] = split_to;
        sh.unit[wave] = unit_to;
    }
    __syncthreads();
    r.own = own;
    r.first = own_to - own;
    r.split = split_to - split;
    r.unit = unit_to - unit;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) {
            r.first += sh.own[w];
            r.split += sh.split[w];
            r.unit += sh.unit[w];
        }
        r.total += sh.own[w];
        r.split_units += sh.unit[w];
    }
    r.total = __builtin_amdgcn_readfirstlane(r.total);
    r.chunk = __builtin_amdgcn_readfirstlane(r.chunk);
    return r;
}
// Item t < it.total, written by the thread that has it; ends with a barrier.
template <int R>
__device__ __forceinline__ void paged_find(const PagedAttnArgs &a, const PagedItems &it, int t, PagedFound *f)
{
    if (t >= it.first && t < it.first + it.own) {
        int run = it.first, split = it.split, unit = it.unit;
        paged_each(a, it, [&](int b, int start, int rows, int len) {
            const int u = paged_units<R>(a, rows), nc = paged_chunks(len, it.chunk);
            if (t >= run && t < run + u * nc) {
                f->seq = b; f->at = t - run; f->units = u; f->chunks = nc; f->split = split; f->unit = unit;
                f->start = start; f->rows = rows; f->len = len;
            }
            run += u * nc;
            split += nc > 1 ? u * nc : 0;
            unit += nc > 1 ? u : 0;
        });
    }
    __syncthreads();
}

// ---- the division into equal streams --------------------------------------------------------------------------------------
//
// For the kernel that is bound by reading keys: all units' keys in blocks of `gran`, unit after unit (sequence, kv head, row
// tile), form one stream, and workgroup w of W takes blocks w per .. (w + 1) per - 1 of it, whatever units they belong to.  All
// workgroups then read the same number of keys, a unit is split only where a border falls into it, and a workgroup has at
// most two partials: of the unit that it ends (slot 2 w) and of the one that it begins (slot 2 w + 1).
struct PagedStream {
    int gran, total, per;                // keys of a block; blocks of the call and of a workgroup
    int b0, b1, first;                   // this thread's sequences, and the blocks ahead of them
    int start, rows, len;                // the first of them
};
struct PagedPiece {
    int seq, start, rows, len;           // sequence of a block
    int before, blocks;                  // blocks ahead of the sequence; blocks of each of its units
    int units;                           // row tiles (per kv head)
};
template <int R, int NT, int BASE>
__device__ __forceinline__ PagedStream paged_stream(const PagedAttnArgs &a, PagedShared<NT> &sh)
{
    const int n = a.p.n_seqs, per = (n + NT - 1) / NT, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    PagedItems r = {};
    r.b0 = min((int)threadIdx.x * per, n);
    r.b1 = min(r.b0 + per, n);
    if (r.b0 < n) {
        r.start = paged_start(a.p, r.b0);
        r.rows = paged_rows(a.p, r.b0, r.start);
        r.len = paged_len(a.p, r.b0);
    }
    float blocks = 0.f, rows = 0.f;
    paged_each(a, r, [&](int, int, int n_rows, int len) {
        blocks += (float)paged_units<R>(a, n_rows) * (float)((len + BASE - 1) / BASE);
        rows += (float)n_rows;
    });
    blocks = wave_scan(blocks);
    rows = wave_scan(rows);
    if (lane == 63) {
        sh.keys[wave] = blocks;
        sh.rows[wave] = rows;
    }
    __syncthreads();
    blocks = rows = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        blocks += sh.keys[w];
        rows += sh.rows[w];
    }
    PagedStream st = {BASE, 0, 1, r.b0, r.b1, 0, r.start, r.rows, r.len};
    if (rows > (float)a.p.n_rows) return st;         // the sequences' rows overlap: no such call, and nothing is done
    // larger blocks where their number would not fit an int32 (a sequence without keys is a block too, hence the margin)
    for (float x = blocks * (float)a.p.Hkv; x > (float)(1 << 29); x *= 0.5f) st.gran *= 2;
    int own = 0;
    paged_each(a, r, [&](int, int, int n_rows, int len) { own += a.p.Hkv * paged_units<R>(a, n_rows) * paged_chunks(len, st.gran); });
    const int own_to = wave_scan(own);
    if (lane == 63) sh.own[wave] = own_to;
    __syncthreads();
    st.first = own_to - own;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) st.first += sh.own[w];
        st.total += sh.own[w];
    }
    st.total = __builtin_amdgcn_readfirstlane(st.total);
    st.per = max((st.total + (int)gridDim.x - 1) / (int)gridDim.x, a.least);
    return st;
}
// The sequence that block t < total belongs to, written by the thread that has it; ends with a barrier.
template <int R>
__device__ __forceinline__ void paged_locate(const PagedAttnArgs &a, const PagedStream &st, int t, PagedPiece *f)
{
    PagedItems r = {};
    r.b0 = st.b0; r.b1 = st.b1; r.start = st.start; r.rows = st.rows; r.len = st.len;
    if (t >= st.first) {
        int run = st.first;
        paged_each(a, r, [&](int b, int start, int rows, int len) {
            const int u = paged_units<R>(a, rows), nb = paged_chunks(len, st.gran), n = a.p.Hkv * u * nb;
            if (t >= run && t < run + n) {
                f->seq = b; f->start = start; f->rows = rows; f->len = len; f->before = run; f->blocks = nb; f->units = u;
            }
            run += n;
        });
    }
    __syncthreads();
}

__device__ __forceinline__ void paged_describe(const PagedAttnArgs &a, int unit, int part0, int parts, int start, int r0, int rows, int g,
                                               int before)
{
    int32_t *d = a.parts.desc + (size_t)unit * 8;
    d[0] = part0; d[1] = parts; d[2] = start; d[3] = r0; d[4] = rows; d[5] = g; d[6] = before;
}

}  // namespace pd
