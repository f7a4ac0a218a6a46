// The division of a paged attention call's keys over its workgroups, on the device (shared by its two kernels).
//
// A unit is a tile of R (token, head) rows of one sequence and kv head.  All units' keys, unit after unit, form one stream, and
// workgroup w takes the w-th of equal parts of it, whatever units they belong to.  All workgroups then have the same work, a unit
// is split only where a border falls into it, and a workgroup has at most two partials: of the unit that it ends (slot 2 w) and
// of the one that it begins (slot 2 w + 1).  Lengths are known on the device alone, so every workgroup works the division out for
// itself.  A thread keeps the sums of its own consecutive sequences and of those before; nothing is stored per sequence.
#pragma once
#include <type_traits>

#include "paged.h"
#include "paged_division.h"

namespace pd {

__device__ __forceinline__ float pexp2(float x) { return __builtin_amdgcn_exp2f(x); }

// 2^(score * scale - m) by a fused product: what rounding leaves of m = rounded(largest * scale), up to half a step of m, is in
// all weights of a row alike, and harmless while it is small.  From here on the products are rounded as m is, so that the largest
// weight is 1 however large the scores are.
constexpr float kExactScores = 0x1p24f;

// Sum over the lanes up to this one, by data-parallel moves: a cross-lane step through LDS would take ten times as long, and every
// workgroup waits for the division before its first load.
template <typename T>
__device__ __forceinline__ T wave_scan(T v)
{
    auto add = [&](auto CTRL, auto ROWS) {
        struct W { int w[sizeof(T) / 4]; } m = __builtin_bit_cast(W, v);
#pragma unroll
        for (int &w : m.w) w = __builtin_amdgcn_update_dpp(0, w, decltype(CTRL)::value, decltype(ROWS)::value, 0xf, true);
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
// a thread's sequences, and the first of them
struct PagedOwn {
    int b0, b1, start, rows, len;
};
template <int NT>
__device__ __forceinline__ PagedOwn paged_own(const PagedAttnArgs &a)
{
    const int n = a.p.n_seqs, per = (n + NT - 1) / NT;
    PagedOwn r = {};
    r.b0 = min((int)threadIdx.x * per, n);
    r.b1 = min(r.b0 + per, n);
    if (r.b0 < n) {
        r.start = paged_start(a.p, r.b0);
        r.rows = paged_rows(a.p, r.b0, r.start);
        r.len = paged_len(a.p, r.b0);
    }
    return r;
}
// f(sequence, first row, rows, positions) for a thread's sequences; the first one's fields are kept, most calls have no more
template <typename F>
__device__ __forceinline__ void paged_each(const PagedAttnArgs &a, const PagedOwn &r, F f)
{
    if (r.b0 < r.b1) f(r.b0, r.start, r.rows, r.len);
    for (int b = r.b0 + 1; b < r.b1; ++b) {
        const int start = paged_start(a.p, b);
        f(b, start, paged_rows(a.p, b, start), paged_len(a.p, b));
    }
}

__device__ __forceinline__ void paged_describe(const PagedAttnArgs &a, int unit, int part0, int parts, int start, int r0, int rows, int g,
                                               int before)
{
    int32_t *d = a.parts.desc + (size_t)unit * 8;
    d[0] = part0; d[1] = parts; d[2] = start; d[3] = r0; d[4] = rows; d[5] = g; d[6] = before;
}

// ---- few rows: bound by reading keys; blocks of `gran` keys are counted, each unit of a sequence has as many -------------
template <int NT>
struct PagedShared {
    float blocks[NT / 64], rows[NT / 64];
    int own[NT / 64];
};
struct PagedStream {
    int gran, total, per;                // keys of a block; blocks of the call and of a workgroup
    int first;                           // blocks ahead of this thread's sequences
    PagedOwn own;
};
struct PagedPiece {
    int seq, start, rows, len;           // sequence of a block
    int before, blocks;                  // blocks ahead of the sequence; blocks of each of its units
    int units;                           // row tiles (per kv head)
};
template <int R, int NT, int BASE>
__device__ __forceinline__ PagedStream paged_stream(const PagedAttnArgs &a, PagedShared<NT> &sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const PagedOwn r = paged_own<NT>(a);
    float blocks = 0.f, rows = 0.f;
    paged_each(a, r, [&](int, int, int n_rows, int len) {
        blocks += (float)paged_units<R>(a, n_rows) * (float)((len + BASE - 1) / BASE);
        rows += (float)n_rows;
    });
    blocks = wave_scan(blocks);
    rows = wave_scan(rows);
    if (lane == 63) {
        sh.blocks[wave] = blocks;
        sh.rows[wave] = rows;
    }
    __syncthreads();
    blocks = rows = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        blocks += sh.blocks[w];
        rows += sh.rows[w];
    }
    PagedStream st = {BASE, 0, 1, 0, r};
    if (rows > (float)a.p.n_rows) return st;         // the sequences' rows overlap: no such call, and nothing is done
    if (a.whole) st.gran = 1 << 30;
    // larger blocks where their number would not fit an int32 (a sequence without keys is a block too, hence the margin)
    else for (float x = blocks * (float)a.p.Hkv; x > (float)(1 << 29); x *= 0.5f) st.gran *= 2;
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
    if (t >= st.first) {
        int run = st.first;
        paged_each(a, st.own, [&](int b, int start, int rows, int len) {
            const int u = paged_units<R>(a, rows), nb = paged_chunks(len, st.gran), n = a.p.Hkv * u * nb;
            if (t >= run && t < run + n) {
                f->seq = b; f->start = start; f->rows = rows; f->len = len; f->before = run; f->blocks = nb; f->units = u;
            }
            run += n;
        });
    }
    __syncthreads();
}

// ---- many rows: bound by the matrix pipe; a unit's tiles of keys are what its last row sees ---------------------------------
// (how it is divided: paged_division.h)
constexpr int kListed = 16;
struct PagedTilesItem {
    int seq, g, start, r0;               // sequence, kv head, first row of the sequence, first (token, head) row of the unit
    int rows, before, t_lo, t_hi;        // (token, head) rows of the sequence, position of its first row, tiles
    int seen, slot, len, tok;            // keys that the unit sees; partial, or -1; positions of the sequence; token of row r0
};
struct PagedTilesSeq {
    long long at;                        // count and units ahead of the sequence
    int unit, seq, start, rows, len, pad;
};
template <int NT>
struct PagedTilesShared {
    long long count[NT / 64];
    int units[NT / 64];
    float rows[NT / 64];
    PagedTilesSeq border[2], of[kListed];            // the sequences of the workgroup's borders and listed units
    PagedTilesItem item[NT / 64][kListed];           // each wave's own copy
};
struct PagedTilesPart {
    long long per, margin;               // count of a workgroup; see above
    long long first;                     // count and units ahead of this thread's sequences
    int w;                               // the workgroup's place
    int first_units, from, to;           // units of the workgroup: from .. to - 1, the first from tile `tile`, the last up to tile_to
    int tile, tile_to;
    PagedOwn own;
};
template <int R, int TK>
__device__ __forceinline__ PagedUnits<R, TK> paged_units_of(const PagedAttnArgs &a, int n_rows, int len)
{
    return PagedUnits<R, TK>(paged_units<R>(a, n_rows), n_rows, len, a.G);
}
template <int R, int TK, int NT>
__device__ __forceinline__ PagedTilesPart paged_tiles_part(const PagedAttnArgs &a, PagedTilesShared<NT> &sh)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, Hkv = a.p.Hkv;
    PagedTilesPart r = {};
    r.own = paged_own<NT>(a);
    long long count = 0;
    int units = 0;
    float rows = 0.f;                    // exact up to 2^24, which no call has more of
    paged_each(a, r.own, [&](int, int, int n_rows, int len) {
        const PagedUnits<R, TK> s = paged_units_of<R, TK>(a, n_rows, len);
        count += Hkv * s.all;
        units += Hkv * s.units;
        rows += (float)n_rows;
    });
    // Neighbours in the stream read the same keys, so those of an XCD, which are every eighth workgroup, are neighbours: four
    // prompts of 2048 tokens, 32 heads on 8, take 164 us so and 173 us in the workgroups' own order
    const int W = gridDim.x, xcd = blockIdx.x & 7;
    r.w = xcd * (W >> 3) + min(xcd, W & 7) + (blockIdx.x >> 3);
    const long long count_to = wave_scan(count);
    const int units_to = wave_scan(units);
    rows = wave_scan(rows);
    if (lane == 63) {
        sh.count[wave] = count_to;
        sh.units[wave] = units_to;
        sh.rows[wave] = rows;
    }
    __syncthreads();
    r.first = count_to - count;
    r.first_units = units_to - units;
    long long total = 0;
    int total_units = 0;
    rows = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) {
            r.first += sh.count[w];
            r.first_units += sh.units[w];
        }
        total += sh.count[w];
        total_units += sh.units[w];
        rows += sh.rows[w];
    }
    if (rows > (float)a.p.n_rows) total = 0;         // the sequences' rows overlap: no such call, and nothing is done
    r.per = paged_part_count<TK>(total, W, a.least, a.G);
    r.margin = paged_margin<TK>(r.per, a.G);
    if (total == 0 || r.w * r.per >= total) return r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long long border = (r.w + i) * r.per;
        if (border < r.first || border >= r.first + count) continue;
        long long at = r.first;
        int unit = r.first_units;
        paged_each(a, r.own, [&](int b, int start, int n_rows, int len) {
            const PagedUnits<R, TK> s = paged_units_of<R, TK>(a, n_rows, len);
            if (border >= at && border < at + Hkv * s.all) sh.border[i] = PagedTilesSeq{at, unit, b, start, n_rows, len, 0};
            at += Hkv * s.all;
            unit += Hkv * s.units;
        });
    }
    __syncthreads();
    PagedCut cut = {total_units, 0};                 // of border lane % 2
    const long long border = (r.w + (lane & 1)) * r.per;
    if (border < total) {
        const PagedTilesSeq q = sh.border[lane & 1];
        const PagedUnits<R, TK> s = paged_units_of<R, TK>(a, q.rows, q.len);
        cut = s.cut(border - q.at, r.margin);
        cut.unit += q.unit;
    }
    r.from = __builtin_amdgcn_readlane(cut.unit, 0);
    r.tile = __builtin_amdgcn_readlane(cut.tile, 0);
    r.tile_to = __builtin_amdgcn_readlane(cut.tile, 1);
    r.to = __builtin_amdgcn_readlane(cut.unit, 1) + (r.tile_to > 0);
    return r;
}
// The list of units first .. first + kListed - 1 of the workgroup; a wave writes its copy, thread 0 describes the unit that the
// workgroup begins and does not end.  All threads come here, which is a barrier for what they read of an earlier list.
template <int R, int TK, int NT>
__device__ __forceinline__ void paged_tiles_list(const PagedAttnArgs &a, PagedTilesShared<NT> &sh, const PagedTilesPart &part, int first)
{
    const int Hkv = a.p.Hkv, end = min(first + kListed, part.to), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int unit = part.first_units;
    long long at = part.first;
    __syncthreads();
    if (unit < end)
        paged_each(a, part.own, [&](int b, int start, int n_rows, int len) {
            const PagedUnits<R, TK> s = paged_units_of<R, TK>(a, n_rows, len);
            for (int k = max(first, unit); k < min(end, unit + Hkv * s.units); ++k) sh.of[k - first] = PagedTilesSeq{at, unit, b, start, n_rows, len, 0};
            unit += Hkv * s.units;
            at += Hkv * s.all;
        });
    __syncthreads();
    if (first + lane < end) {
        const PagedTilesSeq q = sh.of[lane];
        const PagedUnits<R, TK> s = paged_units_of<R, TK>(a, q.rows, q.len);
        const int k = first + lane, g = (k - q.unit) / s.units, i = k - q.unit - g * s.units, u = s.tile(i), seen = s.seen(u), tiles = s.tiles(seen);
        const int lo = k == part.from ? part.tile : 0, hi = k == part.to - 1 && part.tile_to ? part.tile_to : tiles;
        const int slot = lo > 0 ? 2 * part.w : hi < tiles ? 2 * part.w + 1 : -1;
        sh.item[wave][lane] = PagedTilesItem{q.seq, g, q.start, u * R, s.rows, s.before, lo, hi, seen, slot, q.len, u * R / a.G};
        if (wave == 0 && k == part.to - 1 && a.parts.desc) {
            int parts = 0;
            if (lo == 0 && hi < tiles) {
                const long long u0 = q.at + g * s.all + s.ahead(i), u1 = u0 + s.count(u);
                parts = paged_parts(u0, u1, part.margin, part.per);
            }
            paged_describe(a, part.w, slot, parts, q.start, u * R, s.rows, g, s.before);
        }
    }
}

}  // namespace pd
