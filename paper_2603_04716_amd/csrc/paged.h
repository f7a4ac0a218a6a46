// Paged key/value cache: what its kernels share (internal, not part of the C ABI).
#pragma once
#include "pd_internal.h"

namespace pd {

enum PagedKind { PAGED_BF16 = 0, PAGED_E4M3 = 1, PAGED_F32 = 2 };
constexpr int kPagedMaxSeqs = 4096;
constexpr float kPagedMinScale = 0x1p-60f;      // smallest scale of an E4M3 page: its inverse is an ordinary fp32 number

// The pages and the sequences of a call.  starts, lens and the table come from device memory and are not known on the
// host, so every value read from them is brought into its range before it is used: no content of theirs makes a kernel
// leave the tensors.
struct PagedView {
    void *k, *v;                     // [n_pages][Hkv][1 << ps_log][hd]
    float *k_scales, *v_scales;      // [n_pages][Hkv] (E4M3)
    const int32_t *starts;           // [n_seqs + 1], or null: sequence b is row b
    const int32_t *lens;             // [n_seqs]
    const int32_t *table;            // [n_seqs][width]
    int32_t n_seqs, n_rows, width, ps_log, n_pages, Hkv;
};

// What a kernel only reads, as constant memory: at a wave-uniform index the load is a scalar one, which waits for no vector
// load that is still under way.
template <typename T>
__device__ __forceinline__ T load_const(const T *p, size_t i)
{
    return ((const T __attribute__((address_space(4))) *)(uintptr_t)p)[i];
}
__device__ __forceinline__ int paged_start(const PagedView &p, int b)
{
    return p.starts ? min(max(load_const(p.starts, b), 0), p.n_rows) : b;
}
// rows of sequence b (a host check keeps n_rows >= n_seqs where starts is null)
__device__ __forceinline__ int paged_rows(const PagedView &p, int b, int start)
{
    return p.starts ? max(paged_start(p, b + 1) - start, 0) : 1;
}
__device__ __forceinline__ int paged_len(const PagedView &p, int b)
{
    return min(max(load_const(p.lens, b), 0), p.width << p.ps_log);
}

struct PagedAppendArgs {
    PagedView p;
    const void *q, *k, *v;                           // rows; q null: keys and values only
    void *q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;   // elements from row to row
    int32_t Hq, rope;                                // rope 0: keys and queries are stored as they are
    double turns[64];                                // base^(-2c / hd) / (2 pi): turns per position of channel pair c
};
hipError_t launch_paged_append(int kind, int hd, const PagedAppendArgs &a, hipStream_t s);

// Partial results of units - tiles of query rows of one sequence and kv head - whose keys are divided over several workgroups,
// for one attention kernel.
constexpr int kMergeUnits = 4;           // merge_units: at most
struct PagedParts {
    int32_t *desc;      // [..][8]: first partial, partials, first row of the sequence, first (token, head) row of the unit, (token,
                        // head) rows of the sequence, kv head, position of the sequence's first row
    float *ml;          // [..][rows][2] running maximum (log2 domain) and sum
    float *o;           // [..][rows][hd] unnormalised
    int32_t units;      // workgroups that describe one each
    int32_t rows;       // query rows of a unit
    int32_t merge_groups, merge_units;   // workgroups that share the rows of so many described units
};
struct PagedAttnArgs {
    PagedView p;
    const void *q;
    int64_t q_stride;
    void *out;                       // [n_rows][Hq][hd]
    int32_t Hq, G;                   // G = Hq / Hkv
    float scale;
    int32_t rows_above, rows_most;   // this kernel's sequences: more (token, head) rows than the one, at most the other
    int32_t least;                   // fewest blocks (few rows) or tiles (many) of a workgroup
    int32_t whole;                   // (few) no unit is split
    PagedParts parts;
};
// How one of the two kernels is launched, and its part of the workspace: from the host's fields of the call alone.
struct PagedAttnPart {
    bool used, merge;                // launched at all; some of its units may be split
    int rows;                        // query rows of a unit
    int rows_above, rows_most, least, whole, merge_groups, merge_units;
    unsigned grid;
    int cap_units, cap_items;        // units to be merged and their partials: at most
    size_t off_desc, off_ml, off_o;
};
struct PagedAttnPlan {
    PagedAttnPart few, many;
    size_t bytes;
};
PagedAttnPlan paged_attn_plan(int kind, int hd, const PagedView &p, int Hq);
hipError_t launch_paged_attention(int kind, int hd, const PagedAttnArgs &a, const PagedAttnPlan &plan, char *ws, hipStream_t s);
hipError_t launch_paged_tiles(int kind, int hd, const PagedAttnArgs &a, unsigned grid, hipStream_t s);

}  // namespace pd
