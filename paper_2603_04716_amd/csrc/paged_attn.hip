// Attention over a paged key/value cache (grouped queries, causal inside a sequence), any number of query rows.
//
//   o = sum_{j <= p} exp(scale q.k_j - m) v_j / sum_{j <= p} exp(scale q.k_j - m)        p = position of the row
//
// For few query rows the floor is reading the visible keys and values once.  A unit is a tile of R = 16 NR (token, head)
// rows of one sequence and kv head: the whole group's query heads share every byte that is read.  A unit's keys are
// divided into chunks, one workgroup of four waves each; the waves take the chunk's steps of 16 NKB keys in turn, straight
// from the pages into matrix operands, with the running maximum and sum of the softmax per row, and join in LDS at the end.
//
//   S^T[key, row] = K[key, :] . Q[row, :]      A = keys as they lie in the page, B = the unit's query rows
//   O^T[c, row]   = V^T[c, key] . P^T[key, row] A = values transposed in registers, B = the exponentials where the first
//                                              product leaves them
//
// Pages hold values row by row, so that appending a token writes whole rows; the second product wants eight keys of one
// channel per lane.  A lane therefore loads hd / 16 channels of its eight keys and swaps halves of registers
// (v_perm_b32, one per register), which takes no LDS and no lane crossing; accumulator c of a lane is then channel
// (hd / 16) m + c of the matrix row m, 32 (hd 128) neighbouring channels per lane in all.
#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace pd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float pexp2(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- the division of the call's keys into items ------------------------------------------------------------------------
//
// Lengths are known on the device alone, so every workgroup works the division out for itself: the keys that all units
// have to read, divided by the items aimed for, is the chunk; a sequence of len keys and U units makes U ceil(len / chunk)
// items, and since U (len / chunk + 1) <= 2 U len / chunk where there is more than one chunk, the split ones are at most
// twice the items aimed for.  pre[0 .. 2][b]: items, split items and split units (per kv head) ahead of sequence b.
struct PagedItems {
    int chunk, total, split_items, split_units;
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
// sum over the threads below this one
template <int NT>
__device__ __forceinline__ int block_scan(int v, int *red)
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
    int base = 0;
    for (int w = 0; w < wave; ++w) base += red[w];
    return base + inc - v;
}
// units of sequence b
template <int R>
__device__ __forceinline__ int paged_units(const PagedAttnArgs &a, int b)
{
    return (paged_rows(a.p, b, paged_start(a.p, b)) * a.G + R - 1) / R;
}
template <int R, int NT>
__device__ __forceinline__ PagedItems paged_divide(const PagedAttnArgs &a, int *pre, void *red)
{
    const int n = a.p.n_seqs, per = (n + NT - 1) / NT, b0 = min((int)threadIdx.x * per, n), b1 = min(b0 + per, n);
    long keys = 0, rows = 0;
    for (int b = b0; b < b1; ++b) {
        keys += (long)paged_units<R>(a, b) * paged_len(a.p, b);
        rows += paged_rows(a.p, b, paged_start(a.p, b));
    }
    keys = block_sum<NT>(keys, (long *)red) * a.p.Hkv;
    rows = block_sum<NT>(rows, (long *)red);
    PagedItems r = {64, 0, 0, 0};
    if (rows > a.p.n_rows) return r;                 // the sequences' rows overlap: no such call, and nothing is done
    r.chunk = (int)min((max((keys + a.target - 1) / a.target, (long)a.chunk_min) + 63) & ~63l, 1l << 30);
    int c[3] = {0, 0, 0};
    for (int b = b0; b < b1; ++b) {
        const int u = paged_units<R>(a, b), nc = max((paged_len(a.p, b) + r.chunk - 1) / r.chunk, 1);
        c[0] += u * nc;
        if (nc > 1) {
            c[1] += u * nc;
            c[2] += u;
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int run = block_scan<NT>(c[k], (int *)red);
        int *q = pre + k * (n + 1);
        for (int b = b0; b < b1; ++b) {
            q[b] = run;
            const int u = paged_units<R>(a, b), nc = max((paged_len(a.p, b) + r.chunk - 1) / r.chunk, 1);
            run += k == 0 ? u * nc : nc == 1 ? 0 : k == 1 ? u * nc : u;
        }
        if (b1 == n && b0 < n) q[n] = run;
    }
    __syncthreads();
    r.total = pre[n];
    r.split_items = pre[2 * n + 1];
    r.split_units = pre[3 * n + 2];
    return r;
}

// ---- one step of NKB * 16 keys in registers -------------------------------------------------------------------------------
//
// Lane (m, kg) = (lane % 16, lane / 16).  Keys: row m of each 16-key block, as the A operand wants it; which channels a
// k-step takes is free as long as the queries agree (q_channel).  Values: keys 16 kb + 4 kg + i of the step, channels CPL m ..
// CPL m + CPL - 1: the keys whose exponentials the first product leaves in lanes kg.
//
// A value that is infinite or not a number must not reach a row that does not see it, but 0 * infinity would: a step that
// its rows see in part takes such values out of the product (take_odd) and adds them to the rows that see them one by one.
__device__ __forceinline__ unsigned finite_part2(unsigned x)      // of two bf16 values
{
    return ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
}

template <typename STEP, int HD>
struct Step16 {                                      // bf16 operands, 32 keys: what both 16-bit and 8-bit pages share
    static constexpr int NKB = 2, CPL = HD / 16, NQ = HD / 32;
    typedef bf16x8 qfrag;
    static __device__ __forceinline__ void load_q(const void *q, int kg, qfrag (&f)[NQ])
    {
#pragma unroll
        for (int s = 0; s < NQ; ++s) f[s] = *(const bf16x8 *)((const uint16_t *)q + STEP::q_channel(s, kg));
    }
    static __device__ __forceinline__ void no_q(qfrag (&f)[NQ])
    {
#pragma unroll
        for (int s = 0; s < NQ; ++s) f[s] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
    }
    __device__ __forceinline__ void scores(const qfrag (&q)[NQ], f32x4 (&sacc)[NKB]) const
    {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            sacc[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < NQ; ++s)
                sacc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(((const STEP *)this)->kfrag(kb, s), q[s], sacc[kb], 0, 0, 0);
        }
    }
    // eight values of one channel: halves of the registers of neighbouring keys
    __device__ __forceinline__ u32x4 column(int c) const
    {
        const STEP &me = *(const STEP *)this;
        u32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            r[j] = __builtin_amdgcn_perm(me.pair(2 * j + 1, c >> 1), me.pair(2 * j, c >> 1), c & 1 ? 0x07060302u : 0x05040100u);
        return r;
    }
    static __device__ __forceinline__ bf16x8 operand(const f32x4 (&p)[NKB])
    {
        return __builtin_bit_cast(bf16x8, u32x4{pack2bf(p[0][0], p[0][1]), pack2bf(p[0][2], p[0][3]), pack2bf(p[1][0], p[1][1]), pack2bf(p[1][2], p[1][3])});
    }
    template <int NR>
    __device__ __forceinline__ void values(const f32x4 (&p)[NR][NKB], f32x4 (&o)[NR][CPL]) const
    {
        bf16x8 pf[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) pf[r] = operand(p[r]);
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const bf16x8 vf = __builtin_bit_cast(bf16x8, column(c));
#pragma unroll
            for (int r = 0; r < NR; ++r) o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r], o[r][c], 0, 0, 0);
        }
    }
};

template <int KIND, int HD>
struct Step;

template <int HD>
struct Step<PAGED_BF16, HD> : Step16<Step<PAGED_BF16, HD>, HD> {
    static constexpr int CPL = HD / 16;
    typedef uint16_t elem;
    u32x4 k[2][HD / 32];
    unsigned v[8][CPL / 2];
    static __device__ __forceinline__ int q_channel(int s, int kg) { return 32 * s + 8 * kg; }
    // kp, vp: rows of the 16-key block kb
    __device__ __forceinline__ void load(int kb, const elem *kp, const elem *vp, float, float, int m, int kg)
    {
#pragma unroll
        for (int s = 0; s < HD / 32; ++s) k[kb][s] = *(const u32x4 *)(kp + m * HD + 32 * s + 8 * kg);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const elem *src = vp + (4 * kg + i) * HD + CPL * m;
            if (CPL == 8) {
                const u32x4 w = *(const u32x4 *)src;
#pragma unroll
                for (int d = 0; d < CPL / 2; ++d) v[4 * kb + i][d] = w[d];
            } else {
                const u32x2 w = *(const u32x2 *)src;
#pragma unroll
                for (int d = 0; d < CPL / 2; ++d) v[4 * kb + i][d] = w[d];
            }
        }
    }
    __device__ __forceinline__ void clear_keys(int kb)
    {
#pragma unroll
        for (int s = 0; s < HD / 32; ++s) k[kb][s] = u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void clear_value(int i)
    {
#pragma unroll
        for (int d = 0; d < CPL / 2; ++d) v[i][d] = 0u;
    }
    __device__ __forceinline__ bool take_odd()
    {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int d = 0; d < CPL / 2; ++d) {
                const unsigned x = finite_part2(v[i][d]);
                odd |= x != v[i][d];
                v[i][d] = x;
            }
        return odd;
    }
    static __device__ __forceinline__ float value(elem x, float) { return bfbits2f(x); }
    __device__ __forceinline__ bf16x8 kfrag(int kb, int s) const { return __builtin_bit_cast(bf16x8, k[kb][s]); }
    __device__ __forceinline__ unsigned pair(int i, int d) const { return v[i][d]; }   // channels 2 d, 2 d + 1 of the lane's key i
};

// E4M3: a code times its page's scale (a power of two) is exact in bf16, and one instruction widens two of them.
template <int HD>
struct Step<PAGED_E4M3, HD> : Step16<Step<PAGED_E4M3, HD>, HD> {
    static constexpr int CPL = HD / 16;
    typedef uint8_t elem;
    u32x4 k[2][HD / 64];
    unsigned v[8][CPL / 4];
    float ks[2], vs[2];
    // 16 consecutive channels per lane and load: k-steps 2 t and 2 t + 1
    static __device__ __forceinline__ int q_channel(int s, int kg) { return 64 * (s >> 1) + 16 * kg + 8 * (s & 1); }
    __device__ __forceinline__ void load(int kb, const elem *kp, const elem *vp, float k_scale, float v_scale, int m, int kg)
    {
        ks[kb] = k_scale;
        vs[kb] = v_scale;
#pragma unroll
        for (int t = 0; t < HD / 64; ++t) k[kb][t] = *(const u32x4 *)(kp + m * HD + 64 * t + 16 * kg);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const elem *src = vp + (4 * kg + i) * HD + CPL * m;
            if (CPL == 8) {
                const u32x2 w = *(const u32x2 *)src;
#pragma unroll
                for (int d = 0; d < CPL / 4; ++d) v[4 * kb + i][d] = w[d];
            } else {
                v[4 * kb + i][0] = *(const unsigned *)src;
            }
        }
    }
    __device__ __forceinline__ void clear_keys(int kb)
    {
#pragma unroll
        for (int t = 0; t < HD / 64; ++t) k[kb][t] = u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void clear_value(int i)
    {
#pragma unroll
        for (int d = 0; d < CPL / 4; ++d) v[i][d] = 0u;
    }
    __device__ __forceinline__ bool take_odd()       // the codes 0x7f and 0xff are not numbers; there are no infinities
    {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int d = 0; d < CPL / 4; ++d)
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    if ((v[i][d] >> e & 0x7fu) == 0x7fu) {
                        v[i][d] &= ~(0xffu << e);
                        odd = true;
                    }
        return odd;
    }
    static __device__ __forceinline__ float value(elem x, float scale) { return e4m3_decode(x) * scale; }
    static __device__ __forceinline__ unsigned widen(unsigned w, float scale, bool high)
    {
        return high ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))
                    : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    }
    __device__ __forceinline__ bf16x8 kfrag(int kb, int s) const
    {
        const unsigned a = k[kb][s >> 1][2 * (s & 1)], b = k[kb][s >> 1][2 * (s & 1) + 1];
        return __builtin_bit_cast(bf16x8, u32x4{widen(a, ks[kb], false), widen(a, ks[kb], true), widen(b, ks[kb], false), widen(b, ks[kb], true)});
    }
    __device__ __forceinline__ unsigned pair(int i, int d) const { return widen(v[i][d >> 1], vs[i >> 2], d & 1); }
};

// fp32: 16 keys a step on v_mfma_f32_16x16x4_f32, whose operands are one value per lane: nothing to transpose.
template <int HD>
struct Step<PAGED_F32, HD> {
    static constexpr int NKB = 1, CPL = HD / 16, NQ = HD / 4;
    typedef float elem;
    typedef float qfrag;
    f32x4 k[HD / 16], v[4][CPL / 4];
    static __device__ __forceinline__ void load_q(const void *q, int kg, qfrag (&f)[NQ])
    {
#pragma unroll
        for (int t = 0; t < HD / 16; ++t) {
            const f32x4 w = *(const f32x4 *)((const float *)q + 16 * t + 4 * kg);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * t + e] = w[e];
        }
    }
    static __device__ __forceinline__ void no_q(qfrag (&f)[NQ])
    {
#pragma unroll
        for (int s = 0; s < NQ; ++s) f[s] = 0.f;
    }
    __device__ __forceinline__ void load(int, const elem *kp, const elem *vp, float, float, int m, int kg)
    {
#pragma unroll
        for (int t = 0; t < HD / 16; ++t) k[t] = *(const f32x4 *)(kp + m * HD + 16 * t + 4 * kg);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < CPL / 4; ++d) v[i][d] = *(const f32x4 *)(vp + (4 * kg + i) * HD + CPL * m + 4 * d);
    }
    __device__ __forceinline__ void clear_keys(int)
    {
#pragma unroll
        for (int t = 0; t < HD / 16; ++t) k[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void clear_value(int i)
    {
#pragma unroll
        for (int d = 0; d < CPL / 4; ++d) v[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void scores(const qfrag (&q)[NQ], f32x4 (&sacc)[1]) const
    {
        sacc[0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < HD / 16; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sacc[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][e], q[4 * t + e], sacc[0], 0, 0, 0);
    }
    template <int NR>
    __device__ __forceinline__ void values(const f32x4 (&p)[NR][1], f32x4 (&o)[NR][CPL]) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < CPL; ++c)
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    o[r][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j][c >> 2][c & 3], p[r][0][j], o[r][c], 0, 0, 0);
    }
    __device__ __forceinline__ bool take_odd()
    {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < CPL; ++c)
                if (!(fabsf(v[i][c >> 2][c & 3]) < INFINITY)) {
                    v[i][c >> 2][c & 3] = 0.f;
                    odd = true;
                }
        return odd;
    }
    static __device__ __forceinline__ float value(elem x, float) { return x; }
};

// four consecutive channels of an output row
__device__ __forceinline__ void store4(uint16_t *p, f32x4 x) { *(uint2 *)p = make_uint2(pack2bf(x[0], x[1]), pack2bf(x[2], x[3])); }
__device__ __forceinline__ void store4(float *p, f32x4 x) { *(f32x4 *)p = x; }
template <int KIND>
struct RowElem { typedef uint16_t type; };
template <>
struct RowElem<PAGED_F32> { typedef float type; };

constexpr int kWaves = 4;

template <int KIND, int HD, int NR>
__global__ __launch_bounds__(256, KIND == PAGED_F32 ? 1 : 2) void paged_rows_kernel(PagedAttnArgs a)
{
    typedef Step<KIND, HD> S;
    typedef typename RowElem<KIND>::type T;
    constexpr int R = 16 * NR, NKB = S::NKB, KS = 16 * NKB, CPL = S::CPL, NQ = S::NQ, LD = HD + 4;
    extern __shared__ __attribute__((aligned(16))) float sm[];
    float *os = sm, *ml = sm + kWaves * R * LD;      // per wave: O [R][LD]; (maximum, sum) [R]
    int *pre = (int *)(ml + kWaves * R * 2);         // [3][n_seqs + 1]
    __shared__ long red[kWaves];
    const PagedView &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedItems it = paged_divide<R, 256>(a, pre, red);
    const int *pre_split = pre + p.n_seqs + 1, *pre_unit = pre_split + p.n_seqs + 1;
    if (blockIdx.x == 0 && tid == 0 && a.parts.head) a.parts.head[0] = it.split_units * p.Hkv;
    const float sl2e = a.scale * 1.4426950408889634f;

    for (int item = blockIdx.x; item < it.total * p.Hkv; item += gridDim.x) {
        const int t = item / p.Hkv, g = item - t * p.Hkv;
        int b = 0;
        for (int hi = p.n_seqs; hi - b > 1;) {       // last sequence whose items start at or before t
            const int mid = (b + hi) >> 1;
            if (pre[mid] <= t) b = mid; else hi = mid;
        }
        b = __builtin_amdgcn_readfirstlane(b);
        const int start = paged_start(p, b), rows = paged_rows(p, b, start), len = paged_len(p, b);
        const int units = (rows * a.G + R - 1) / R, nc = max((len + it.chunk - 1) / it.chunk, 1);
        // row tiles that read the same keys are neighbours, the one that sees most first
        const int c = (t - pre[b]) / units, u = units - 1 - (t - pre[b] - c * units);
        const int r0 = u * R, nrows = min(R, rows * a.G - r0);
        const int before = len - rows;               // position of the sequence's first row (negative: it is not held)
        const int vis_min = before + r0 / a.G + 1, vis_max = max(before + (r0 + nrows - 1) / a.G + 1, 0);
        const int nc_u = max((vis_max + it.chunk - 1) / it.chunk, 1);
        if (c >= nc_u) continue;
        const int c0 = c * it.chunk, c1 = min(vis_max, c0 + it.chunk);

        typename S::qfrag q[NR][NQ];
        int limit[NR];                               // the row sees keys 0 .. limit - 1
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = r0 + 16 * r + n, tok = row / a.G;
            const bool ok = row < r0 + nrows;
            limit[r] = ok ? before + tok + 1 : 0;
            S::no_q(q[r]);
            if (ok) S::load_q((const T *)a.q + (start + tok) * a.q_stride + (g * a.G + row - tok * a.G) * HD, kg, q[r]);
        }
        f32x4 o[NR][CPL];
        float m_run[NR], l_run[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            m_run[r] = -INFINITY;
            l_run[r] = 0.f;
#pragma unroll
            for (int i = 0; i < CPL; ++i) o[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int32_t *pages = p.table + (size_t)b * p.width;
        for (int k0 = c0 + wave * KS; k0 < c1; k0 += kWaves * KS) {
            S st;
            bool gone[NKB];
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const int key = k0 + 16 * kb, at = min(key, len - 1);
                const int id = pages[at >> p.ps_log];
                gone[kb] = id < 0 || id >= p.n_pages;
                const size_t unit = (size_t)(gone[kb] ? 0 : id) * p.Hkv + g;
                const size_t off = ((unit << p.ps_log) + (key & ((1 << p.ps_log) - 1))) * HD;
                st.load(kb, (const typename S::elem *)p.k + off, (const typename S::elem *)p.v + off,
                        KIND == PAGED_E4M3 ? p.k_scales[unit] : 1.f, KIND == PAGED_E4M3 ? p.v_scales[unit] : 1.f, n, kg);
            }
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                if (gone[kb]) {                      // a page that is not there reads as zeros
                    st.clear_keys(kb);
#pragma unroll
                    for (int i = 0; i < 4; ++i) st.clear_value(4 * kb + i);
                }
            }
            const bool past = k0 + KS > c1, part = k0 + KS > vis_min;
            if (past)                                // nobody's keys: whatever the page holds there must not meet a weight of 0
#pragma unroll
                for (int i = 0; i < 4 * NKB; ++i)
                    if (k0 + 16 * (i >> 2) + 4 * kg + (i & 3) >= c1) st.clear_value(i);
            f32x4 s[NR][NKB];
            const auto sees = [&](int r, int i) { return k0 + 16 * (i >> 2) + 4 * kg + (i & 3) < min(limit[r], c1); };
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                st.scores(q[r], s[r]);
                float mx = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if ((past || part) && !sees(r, 4 * kb + j)) s[r][kb][j] = -INFINITY;
                        mx = fmaxf(mx, s[r][kb][j]);
                    }
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float m_new = fmaxf(m_run[r], mx * sl2e);
                const float m_ref = m_new == -INFINITY ? 0.f : m_new;      // nothing seen yet: every weight is 0
                const float alpha = pexp2(m_run[r] - m_ref);
                m_run[r] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[r][kb][j] = pexp2(fmaf(s[r][kb][j], sl2e, -m_ref));
                        sum += s[r][kb][j];
                    }
                l_run[r] = l_run[r] * alpha + sum;
#pragma unroll
                for (int i = 0; i < CPL; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[r][i][j] *= alpha;
            }
            const bool odd = part && vis_min != vis_max && __any(st.take_odd());
            st.template values<NR>(s, o);
            if (odd)
#pragma unroll 1
                for (int key = k0; key < min(k0 + KS, c1); ++key) {
                    const int id = pages[key >> p.ps_log];
                    if (id < 0 || id >= p.n_pages) continue;
                    const size_t unit = (size_t)id * p.Hkv + g;
                    const typename S::elem *src = (const typename S::elem *)p.v + ((unit << p.ps_log) + (key & ((1 << p.ps_log) - 1))) * HD + 4 * CPL * kg;
                    const float scale = KIND == PAGED_E4M3 ? p.v_scales[unit] : 1.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < CPL; ++i) {
                            const float x = S::value(src[CPL * j + i], scale);
                            if (!(fabsf(x) < INFINITY))
#pragma unroll
                                for (int r = 0; r < NR; ++r)
                                    if (key < limit[r]) o[r][i][j] += x;
                        }
                }
        }

        // ---- join the waves -------------------------------------------------------------------------------------------------
        const int nw = max(min((c1 - c0 + KS - 1) / KS, kWaves), 1);       // waves that had a step
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float l = l_run[r] + __shfl_xor(l_run[r], 16, 64);
            l += __shfl_xor(l, 32, 64);
            if (wave < nw && 16 * r + n < nrows) {
                if (kg == 0) {
                    ml[(wave * R + 16 * r + n) * 2] = m_run[r];
                    ml[(wave * R + 16 * r + n) * 2 + 1] = l;
                }
                float *dst = os + (wave * R + 16 * r + n) * LD + 4 * CPL * kg;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int d = 0; d < CPL / 4; ++d)
                        *(f32x4 *)(dst + CPL * j + 4 * d) = f32x4{o[r][4 * d][j], o[r][4 * d + 1][j], o[r][4 * d + 2][j], o[r][4 * d + 3][j]};
            }
        }
        __syncthreads();
        const int part0 = ((pre_split[b] + u * nc) * p.Hkv) + g * nc_u;    // first partial of the unit
        for (int e = tid; e < nrows * (HD / 4); e += 256) {
            const int row = e / (HD / 4), d = (e & (HD / 4 - 1)) * 4;
            float M = -INFINITY, L = 0.f;
            for (int i = 0; i < nw; ++i) M = fmaxf(M, ml[(i * R + row) * 2]);
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            for (int i = 0; i < nw; ++i) {
                const float m = ml[(i * R + row) * 2];
                const float w = m == -INFINITY ? 0.f : pexp2(m - M);
                L += w * ml[(i * R + row) * 2 + 1];
                const f32x4 y = *(const f32x4 *)(os + (i * R + row) * LD + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] += w * y[j];
            }
            const int tok = (r0 + row) / a.G, head = g * a.G + r0 + row - tok * a.G;
            if (nc_u == 1) {
                const float inv = 1.f / L;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = before + tok < 0 ? 0.f : x[j] * inv;
                store4((T *)a.out + ((size_t)(start + tok) * a.Hq + head) * HD + d, x);
            } else {
                const size_t at = (size_t)(part0 + c) * R + row;
                *(f32x4 *)(a.parts.o + at * HD + d) = x;
                if (d == 0) *(float2 *)(a.parts.ml + at * 2) = make_float2(M, L);
            }
        }
        if (nc > 1 && c == 0 && tid < 8) {
            const int vals[8] = {part0, nc_u, start, r0, rows * a.G, g, before, 0};
            int v = vals[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) v = tid == i ? vals[i] : v;
            a.parts.desc[(size_t)((pre_unit[b] + u) * p.Hkv + g) * 8 + tid] = v;
        }
        __syncthreads();
    }
}

// Adds up the partials of a split unit: o = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c.  A workgroup takes a row at a
// time, its four waves the row's partials in turn.
template <int KIND, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a)
{
    typedef typename std::conditional<KIND == PAGED_F32, float, bf16_t>::type T;
    constexpr int CH = HD / 64;
    __shared__ float xs[kWaves][HD], ls[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, R = a.parts.rows;
    const int tasks = a.parts.head[0] * R;
    for (int t = blockIdx.x; t < tasks; t += gridDim.x) {
        const int32_t *desc = a.parts.desc + (size_t)(t / R) * 8;
        const int part0 = desc[0], nc = desc[1], start = desc[2], r = desc[3] + t % R, rows = desc[4], g = desc[5], before = desc[6];
        if (nc == 1 || r >= rows) continue;
        float M = -INFINITY;
        for (int c = lane; c < nc; c += 64) M = fmaxf(M, a.parts.ml[((size_t)(part0 + c) * R + t % R) * 2]);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
        float x[CH] = {}, L = 0.f;
#pragma unroll 4
        for (int c = wave; c < nc; c += kWaves) {
            const size_t at = (size_t)(part0 + c) * R + t % R;
            const float2 ml = *(const float2 *)(a.parts.ml + at * 2);
            const float w = ml.x == -INFINITY ? 0.f : pexp2(ml.x - M);
            L += w * ml.y;
#pragma unroll
            for (int i = 0; i < CH; ++i) x[i] += w * a.parts.o[at * HD + CH * lane + i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < CH; ++i) xs[wave][CH * lane + i] = x[i];
        if (lane == 0) ls[wave] = L;
        __syncthreads();
        const int tok = r / a.G, head = g * a.G + r - tok * a.G;
        if (threadIdx.x < HD) {
            const int d = threadIdx.x;
            const float y = before + tok < 0 ? 0.f : (xs[0][d] + xs[1][d] + xs[2][d] + xs[3][d]) * (1.f / (ls[0] + ls[1] + ls[2] + ls[3]));
            Elem<T>::st((T *)a.out + ((size_t)(start + tok) * a.Hq + head) * HD + d, y);
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
constexpr int kChunkMin = 256;      // keys: two steps for each of the four waves
constexpr int kTarget = 1024;       // items to aim for: two workgroups on each of the 256 CUs, twice over

PagedAttnPlan paged_attn_plan(int kind, int hd, const PagedView &p, int Hq)
{
    PagedAttnPlan r;
    const int G = Hq / p.Hkv;
    r.rows = !p.starts && G <= 16 ? 16 : 32;
    r.chunk_min = kChunkMin;
    r.target = kTarget;
    const int64_t max_len = (int64_t)p.width << p.ps_log;
    const int64_t units = ((int64_t)p.n_rows * G / r.rows + p.n_seqs) * p.Hkv;
    const int64_t chunks = (max_len + kChunkMin - 1) / kChunkMin;
    r.merge = chunks > 1 && units > 0;
    r.cap_items = r.merge ? (int)std::min<int64_t>(2 * kTarget, units * chunks) : 0;
    r.cap_units = r.merge ? (int)std::min<int64_t>(kTarget, units) : 0;
    const size_t al = 255;
    r.off_desc = 256;
    r.off_ml = (r.off_desc + (size_t)r.cap_units * 32 + al) & ~al;
    r.off_o = (r.off_ml + (size_t)r.cap_items * r.rows * 8 + al) & ~al;
    r.bytes = r.merge ? r.off_o + (size_t)r.cap_items * r.rows * hd * 4 : 0;
    return r;
}

template <int KIND, int HD, int NR>
static hipError_t launch_rows(const PagedAttnArgs &a, unsigned grid, hipStream_t s)
{
    const size_t lds = (size_t)(kWaves * 16 * NR * (HD + 6) + 3 * (a.p.n_seqs + 1)) * 4;
    static OncePerDevice attr;
    int dev;
    if (attr.need(&dev)) {
        const size_t most = (size_t)(kWaves * 16 * NR * (HD + 6) + 3 * (kPagedMaxSeqs + 1)) * 4;
        hipError_t e = hipFuncSetAttribute((const void *)paged_rows_kernel<KIND, HD, NR>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
        if (e != hipSuccess) return e;
        attr.mark(dev);
    }
    paged_rows_kernel<KIND, HD, NR><<<grid, 256, lds, s>>>(a);
    return hipGetLastError();
}

template <int KIND, int HD>
static hipError_t launch_kind(const PagedAttnArgs &a, const PagedAttnPlan &plan, hipStream_t s)
{
    const int64_t units = ((int64_t)a.p.n_rows * a.G / plan.rows + a.p.n_seqs) * a.p.Hkv;
    const unsigned grid = (unsigned)std::min<int64_t>(units + (plan.merge ? plan.target : 0), 1 << 20);
    hipError_t e = plan.rows == 16 ? launch_rows<KIND, HD, 1>(a, grid, s) : launch_rows<KIND, HD, 2>(a, grid, s);
    if (e != hipSuccess || !plan.merge) return e;
    paged_merge_kernel<KIND, HD><<<std::min(plan.cap_units * plan.rows, 2048), 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_attention(int kind, int hd, PagedAttnArgs a, const PagedAttnPlan &plan, char *ws, hipStream_t s)
{
    a.chunk_min = plan.chunk_min;
    a.target = plan.target;
    a.parts.head = plan.merge ? (int32_t *)ws : nullptr;
    a.parts.desc = (int32_t *)(ws + plan.off_desc);
    a.parts.ml = (float *)(ws + plan.off_ml);
    a.parts.o = (float *)(ws + plan.off_o);
    a.parts.cap_units = plan.cap_units;
    a.parts.rows = plan.rows;
    if (kind == PAGED_BF16) return hd == 128 ? launch_kind<PAGED_BF16, 128>(a, plan, s) : launch_kind<PAGED_BF16, 64>(a, plan, s);
    if (kind == PAGED_E4M3) return hd == 128 ? launch_kind<PAGED_E4M3, 128>(a, plan, s) : launch_kind<PAGED_E4M3, 64>(a, plan, s);
    return hd == 128 ? launch_kind<PAGED_F32, 128>(a, plan, s) : launch_kind<PAGED_F32, 64>(a, plan, s);
}

}  // namespace pd
