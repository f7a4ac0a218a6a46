// The division of a paged attention call's keys into work items, on the device (shared by its two kernels).
//
// A unit is a tile of R (token, head) rows of one sequence and kv head; an item is one of the chunks that a unit's keys are
// divided into.  Lengths are known on the device alone, so every workgroup works the division out for itself: the keys that
// all units have to read, divided by the items aimed for, is the chunk; a sequence of len keys and U units makes
// U ceil(len / chunk) items, and since U (len / chunk + 1) <= 2 U len / chunk where there is more than one chunk, the split
// ones are at most twice the items aimed for.  A thread keeps the counts of its own consecutive sequences and the
// sum of those before; nothing is stored per sequence.
#pragma once
#include "paged.h"

namespace pd {

__device__ __forceinline__ float pexp2(float x) { return __builtin_amdgcn_exp2f(x); }

struct PagedItems {
    int chunk, total, split_units;       // keys of a chunk; items and split units of the call, per kv head
    int b0, b1;                          // this thread's sequences
    int first, own;                      // items ahead of them, and theirs
    int split, unit;                     // split items and split units ahead of them
};
struct PagedFound {
    int seq, at;                         // sequence of an item, and the item's place among the sequence's
    int units, chunks;                   // of the sequence
    int split, unit;                     // split items and split units ahead of the sequence
};

template <int NT>
__device__ __forceinline__ long block_sum(long v, long *red)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    long s = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) s += red[w];
    return s;
}
// sum over the threads below this one; the sum over all in *all
template <int NT>
__device__ __forceinline__ int block_scan(int v, int *red, int *all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int inc = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int u = __shfl_up(inc, off, 64);
        if (lane >= off) inc += u;
    }
    __syncthreads();
    if (lane == 63) red[wave] = inc;
    __syncthreads();
    int base = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w == wave) base = sum;
        sum += red[w];
    }
    *all = sum;
    return base + inc - v;
}
// units of sequence b (none where another kernel has the sequence)
template <int R>
__device__ __forceinline__ int paged_units(const PagedAttnArgs &a, int b)
{
    const int rows = paged_rows(a.p, b, paged_start(a.p, b)) * a.G;
    return rows > a.rows_above && rows <= a.rows_most ? (rows + R - 1) / R : 0;
}
__device__ __forceinline__ int paged_chunks(const PagedAttnArgs &a, int b, int chunk)
{
    return max((paged_len(a.p, b) + chunk - 1) / chunk, 1);
}
// by all NT threads; red: NT / 64 longs of LDS
template <int R, int NT>
__device__ __forceinline__ PagedItems paged_divide(const PagedAttnArgs &a, long *red)
{
    const int n = a.p.n_seqs, per = (n + NT - 1) / NT;
    PagedItems r = {64, 0, 0, min((int)threadIdx.x * per, n), 0, 0, 0, 0, 0};
    r.b1 = min(r.b0 + per, n);
    long keys = 0, rows = 0;
    for (int b = r.b0; b < r.b1; ++b) {
        keys += (long)paged_units<R>(a, b) * paged_len(a.p, b);
        rows += paged_rows(a.p, b, paged_start(a.p, b));
    }
    keys = block_sum<NT>(keys, red) * a.p.Hkv;
    rows = block_sum<NT>(rows, red);
    if (rows > a.p.n_rows) return r;                 // the sequences' rows overlap: no such call, and nothing is done
    r.chunk = (int)min((max((keys + a.target - 1) / a.target, (long)a.chunk_min) + 63) & ~63l, 1l << 30);
    int split = 0, unit = 0, all;
    for (int b = r.b0; b < r.b1; ++b) {
        const int u = paged_units<R>(a, b), nc = paged_chunks(a, b, r.chunk);
        r.own += u * nc;
        split += nc > 1 ? u * nc : 0;
        unit += nc > 1 ? u : 0;
    }
    r.first = block_scan<NT>(r.own, (int *)red, &r.total);
    r.split = block_scan<NT>(split, (int *)red, &all);
    r.unit = block_scan<NT>(unit, (int *)red, &r.split_units);
    return r;
}
// Item t < it.total, written by the thread that has it; ends with a barrier.
template <int R>
__device__ __forceinline__ void paged_find(const PagedAttnArgs &a, const PagedItems &it, int t, PagedFound *f)
{
    if (t >= it.first && t < it.first + it.own) {
        int run = it.first, split = it.split, unit = it.unit;
        for (int b = it.b0; b < it.b1; ++b) {
            const int u = paged_units<R>(a, b), nc = paged_chunks(a, b, it.chunk);
            if (t < run + u * nc) {
                f->seq = b; f->at = t - run; f->units = u; f->chunks = nc; f->split = split; f->unit = unit;
                break;
            }
            run += u * nc;
            split += nc > 1 ? u * nc : 0;
            unit += nc > 1 ? u : 0;
        }
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
