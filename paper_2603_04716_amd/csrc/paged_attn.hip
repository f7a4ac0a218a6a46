// Attention over a paged key/value cache (grouped queries, causal inside a sequence), any number of query rows.
//
//   o = sum_{j <= p} exp(scale q.k_j - m) v_j / sum_{j <= p} exp(scale q.k_j - m)        p = position of the row
//
// For few query rows the floor is reading the visible keys and values once.  A unit is a tile of R = 16 NR (token, head)
// rows of one sequence and kv head: the whole group's query heads share every byte that is read.  All units' keys form one
// stream, which is cut into equal parts, a workgroup of four waves each; the waves take the steps of 16 NKB keys in turn,
// straight from the pages into matrix operands, with the running maximum and sum of the softmax per row, and join in LDS at the
// end of each unit.
//
//   S^T[key, row] = K[key, :] . Q[row, :]      A = keys as they lie in the page, B = the unit's query rows
//   O^T[c, row]   = V^T[c, key] . P^T[key, row] A = values transposed in registers, B = the exponentials where the first
//                                              product leaves them
//
// Pages hold values row by row, so that appending a token writes whole rows; the second product wants eight keys of one
// channel per lane.  A lane therefore loads hd / 16 channels of its eight keys and swaps halves of registers
// (v_perm_b32, one per register), which takes no LDS and no lane crossing; accumulator c of a lane is then channel
// (hd / 16) m + c of the matrix row m, 32 (hd 128) neighbouring channels per lane in all.
//
// Measured, 32 heads on 8 of 128 channels, one row per sequence: 64 sequences of 100 to 8000 positions 175 us or 5.6 TB/s, one of 131000
// 94 us or 5.7 TB/s, 256 of 1500 to 2600 on E4M3 pages 193 us or 5.5 TB/s (a stream of reads reaches 6.2), and 5 us each for the partials.
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "paged_items.h"

namespace pd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

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

// largest value, and sum, over the four lanes of a column (m, m + 16, m + 32, m + 48), in each of them
__device__ __forceinline__ float across_kg(float x)
{
    const unsigned u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned y = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_across_kg(float x)
{
    const unsigned u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned y = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
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
    // The exponentials are rounded to bf16, to be an operand of the matrix pipe (in fp32 the second product would take eight times
    // as long): each weight by up to 2^-8 of itself, so that a result is off by at most that share of sum p |v| / sum p, and mostly by
    // much less, as the roundings are of both signs.  The sum below the fraction adds them unrounded.
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
    bool there[2];
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
    bool there[2];
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
        ks[kb] = vs[kb] = 1.f;                       // (the scale that was loaded is another page's, and may be no number)
    }
    __device__ __forceinline__ void clear_value(int i)
    {
#pragma unroll
        for (int d = 0; d < CPL / 4; ++d) v[i][d] = 0u;
    }
    __device__ __forceinline__ bool take_odd()       // the codes 0x7f and 0xff are not numbers, and 256 * 2^120 is infinite
    {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned least = vs[i >> 2] < 0x1p120f ? 0x7fu : 0x78u;
#pragma unroll
            for (int d = 0; d < CPL / 4; ++d)
#pragma unroll
                for (int e = 0; e < 32; e += 8)
                    if ((v[i][d] >> e & 0x7fu) >= least) {
                        v[i][d] &= ~(0xffu << e);
                        odd = true;
                    }
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
    bool there[1];
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
    __shared__ PagedShared<256> sh;
    __shared__ PagedPiece piece;
    const PagedView &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float sl2e = a.scale * 1.4426950408889634f;
    const PagedStream st = paged_stream<R, 256, kWaves * KS>(a, sh);
    if (a.parts.desc && tid == 0) a.parts.desc[(size_t)blockIdx.x * 8 + 1] = 0;      // no unit of its own to be merged
    const int end = min((int)(blockIdx.x + 1) * st.per, st.total);

    for (int at = blockIdx.x * st.per, next; at < end; at = next) {
        paged_locate<R>(a, st, at, &piece);
        const int b = __builtin_amdgcn_readfirstlane(piece.seq), start = __builtin_amdgcn_readfirstlane(piece.start);
        const int rows = __builtin_amdgcn_readfirstlane(piece.rows), len = __builtin_amdgcn_readfirstlane(piece.len);
        const int nb = __builtin_amdgcn_readfirstlane(piece.blocks), units = __builtin_amdgcn_readfirstlane(piece.units);
        const int first = __builtin_amdgcn_readfirstlane(piece.before);
        const int unit = (at - first) / nb, from = at - first - unit * nb;         // the unit, and its first block here
        const int g = unit / units, u = unit - g * units;
        const int unit0 = first + unit * nb;                                        // its first block in the stream
        next = min(unit0 + nb, end);
        const int r0 = u * R, nrows = min(R, rows * a.G - r0);
        const int before = len - rows;               // position of the sequence's first row (negative: it is not held)
        const int vis_min = before + r0 / a.G + 1, vis_max = max(before + (r0 + nrows - 1) / a.G + 1, 0);
        const int c0 = from * st.gran, c1 = min(vis_max, (next - unit0) * st.gran);   // keys: none where c1 <= c0
        const int w0 = unit0 / st.per, parts = (unit0 + nb - 1) / st.per - w0 + 1;      // the workgroups that share the unit

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
        // Page numbers are asked for a step ahead of the loads, the loads of a step (where the registers hold two of them) a step
        // ahead of its products.  Past the end the last step is asked for again: after a conditional load the compiler would no
        // longer know which loads are the older ones, and wait for all.
        constexpr bool TWO = NR == 1 || KIND == PAGED_F32;
        const int last = c0 + wave * KS + max(c1 - 1 - c0 - wave * KS, 0) / (kWaves * KS) * (kWaves * KS);     // the wave's last step
        int ids[NKB];
        auto ask = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) ids[kb] = load_const(pages, (unsigned)min(min(k0, last) + 16 * kb, len - 1) >> p.ps_log);
        };
        auto load = [&](S &st, int k0) __attribute__((always_inline)) {       // the step at k0, whose pages were asked for
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb) {
                const bool there = (unsigned)ids[kb] < (unsigned)p.n_pages;
                const size_t unit = (size_t)(there ? ids[kb] : 0) * p.Hkv + g;
                const size_t off = ((unit << p.ps_log) + ((min(k0, last) + 16 * kb) & ((1 << p.ps_log) - 1))) * HD;
                st.there[kb] = there;
                st.load(kb, (const typename S::elem *)p.k + off, (const typename S::elem *)p.v + off,
                        KIND == PAGED_E4M3 ? load_const(p.k_scales, unit) : 1.f, KIND == PAGED_E4M3 ? load_const(p.v_scales, unit) : 1.f, n, kg);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        auto process = [&](S &st, int k0) __attribute__((always_inline)) {
#pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
                if (!st.there[kb]) {                 // a page that is not there reads as zeros
                    st.clear_keys(kb);
#pragma unroll
                    for (int i = 0; i < 4; ++i) st.clear_value(4 * kb + i);
                }
            const bool past = k0 + KS > c1, part = k0 + KS > vis_min;
            if (past)                                // nobody's keys: whatever the page holds there must not meet a weight of 0
#pragma unroll
                for (int i = 0; i < 4 * NKB; ++i)
                    if (k0 + 16 * (i >> 2) + 4 * kg + (i & 3) >= c1) st.clear_value(i);
            f32x4 s[NR][NKB];
#pragma unroll
            for (int r = 0; r < NR; ++r) st.scores(q[r], s[r]);
            if (past || part)
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    int seen = min(limit[r], c1) - k0 - 4 * kg;
                    asm volatile("" : "+v"(seen));   // keeps the branch
#pragma unroll
                    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (16 * kb + j >= seen) s[r][kb][j] = -INFINITY;
                }
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                float mx = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) mx = fmaxf(mx, s[r][kb][j]);
                mx = across_kg(mx);
                const float m_new = fmaxf(m_run[r], mx * sl2e);
                const float m_ref = m_new == -INFINITY ? 0.f : m_new;      // nothing seen yet: every weight is 0
                const float alpha = pexp2(m_run[r] - m_ref);
                m_run[r] = m_new;
                float sum = 0.f, factor = sl2e;
                if (__any(fabsf(m_ref) > kExactScores)) {
                    factor = 1.f;
#pragma unroll
                    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[r][kb][j] *= sl2e;
                }
#pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[r][kb][j] = pexp2(fmaf(s[r][kb][j], factor, -m_ref));
                        sum += s[r][kb][j];
                    }
                l_run[r] = l_run[r] * alpha + sum;
                if (__any(alpha != 1.f))             // a NaN is not 1 either
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
                    const int id = load_const(pages, (unsigned)key >> p.ps_log);
                    if (id < 0 || id >= p.n_pages) continue;
                    const size_t unit = (size_t)id * p.Hkv + g;
                    const typename S::elem *src = (const typename S::elem *)p.v + ((unit << p.ps_log) + (key & ((1 << p.ps_log) - 1))) * HD + 4 * CPL * kg;
                    const float scale = KIND == PAGED_E4M3 ? load_const(p.v_scales, unit) : 1.f;
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
        };
        constexpr int D = kWaves * KS;
        int k0 = c0 + wave * KS;
        if (k0 < c1) {
            S sa, sb;
            ask(k0);
            if (TWO) {
                load(sa, k0);
                ask(k0 + D);
                for (;; k0 += 2 * D) {
                    load(sb, k0 + D);
                    ask(k0 + 2 * D);
                    process(sa, k0);
                    if (k0 + D >= c1) break;
                    load(sa, k0 + 2 * D);
                    ask(k0 + 3 * D);
                    process(sb, k0 + D);
                    if (k0 + 2 * D >= c1) break;
                }
            } else {
                for (; k0 < c1; k0 += D) {
                    load(sa, k0);
                    ask(k0 + D);
                    process(sa, k0);
                }
            }
        }

        // ---- join the waves -------------------------------------------------------------------------------------------------
        const int nw = max(min((c1 - c0 + KS - 1) / KS, kWaves), 1);       // waves that had a step
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const float l = sum_across_kg(l_run[r]);
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
        const int slot = 2 * (int)blockIdx.x + (from == 0);
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
            if (parts == 1) {
                const float inv = 1.f / L;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = before + tok < 0 ? 0.f : x[j] * inv;
                store4((T *)a.out + ((size_t)(start + tok) * a.Hq + head) * HD + d, x);
            } else {
                const size_t to = (size_t)slot * R + row;
                *(f32x4 *)(a.parts.o + to * HD + d) = x;
                if (d == 0) *(float2 *)(a.parts.ml + to * 2) = make_float2(M, L);
            }
        }
        if (parts > 1 && from == 0 && tid == 0) paged_describe(a, blockIdx.x, 2 * w0 + 1, parts, start, r0, rows * a.G, g, before);
        __syncthreads();                             // piece, os and ml are read
    }
}

// Adds up the partials of split units: o = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.  `groups` workgroups share the rows of merge_units
// descriptions, most of which name no split unit.  hd / 4 threads, four channels each, take a partial of a row.  Of up to
// kWavePartials partials a wave takes four rows together, whose loads are under way at the same time; of more (one long sequence)
// the workgroup takes one row.
constexpr int kWavePartials = 16;
// partial i of a unit: slot 2 w + 1 of the first workgroup, slot 2 w of the following ones
__device__ __forceinline__ int merge_at(int i) { return max(2 * i - 1, 0); }
template <int KIND, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a, PagedParts few, PagedParts many)
{
    typedef typename RowElem<KIND>::type T;
    constexpr int TPR = HD / 4, NG = 256 / TPR, WG = 64 / TPR;
    __shared__ f32x4 xs[NG][TPR];
    __shared__ float ls[NG];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = threadIdx.x / TPR, d4 = threadIdx.x & (TPR - 1);
    const int blocks_few = few.units ? (few.units + few.merge_units - 1) / few.merge_units * few.merge_groups : 0;
    const bool is_few = (int)blockIdx.x < blocks_few;
    const int block = is_few ? blockIdx.x : blockIdx.x - blocks_few, groups = is_few ? few.merge_groups : many.merge_groups;
    const int units = is_few ? few.units : many.units, most = is_few ? few.merge_units : many.merge_units, unit = block / groups * most;
    const int64_t stride = is_few ? few.rows : many.rows;
    const int32_t *d = is_few ? few.desc : many.desc;
    const float *ml0 = is_few ? few.ml : many.ml, *o0 = is_few ? few.o : many.o;
    int4 lo[kMergeUnits], hi[kMergeUnits];
#pragma unroll
    for (int i = 0; i < kMergeUnits; ++i) {
        const int32_t *di = d + (size_t)min(unit + i, units - 1) * 8;
        lo[i] = *(const int4 *)di;
        hi[i] = *(const int4 *)(di + 4);
    }
#pragma unroll
    for (int i = 0; i < kMergeUnits; ++i) {
        const int parts = lo[i].y, rows = min(hi[i].x - lo[i].w, (int)stride), g = hi[i].y, before = hi[i].z;
        if (i >= most || unit + i >= units || parts <= 1) continue;
        const float *ml = ml0 + (size_t)lo[i].x * stride * 2, *o = o0 + (size_t)lo[i].x * stride * HD + 4 * d4;
        auto store = [&](int r, f32x4 x, float L) {
            const int row = lo[i].w + r, tok = row / a.G, head = g * a.G + row - tok * a.G;
            const float inv = 1.f / L;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = before + tok < 0 ? 0.f : x[j] * inv;
            store4((T *)a.out + ((size_t)(lo[i].z + tok) * a.Hq + head) * HD + 4 * d4, x);
        };
        if (parts <= kWavePartials) {
            for (int r = 16 * (block % groups) + 4 * ((wave + i) & 3); r < rows; r += 16 * groups) {      // units of few rows: each another wave
                // 16 lanes have a row's weights
                const int wr = min(r + (lane >> 4), rows - 1), wp = lane & 15;
                const float2 f = *(const float2 *)(ml + (merge_at(min(wp, parts - 1)) * stride + wr) * 2);
                float M = f.x;
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
                const float w = wp < parts && f.x != -INFINITY ? pexp2(f.x - M) : 0.f;
                float L = w * f.y;
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) L += __shfl_xor(L, off, 64);
                f32x4 x[4] = {};
                for (int p = 0; p < parts; p += WG) {
                    const int mine = p + lane / TPR;
                    const float *op = o + merge_at(min(mine, parts - 1)) * stride * HD;
                    f32x4 y[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) y[q] = *(const f32x4 *)(op + (size_t)min(r + q, rows - 1) * HD);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float wq = __shfl(w, 16 * q + (mine & 15), 64);
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[q][j] += wq * y[q][j];
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int off = TPR; off < 64; off *= 2)
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[q][j] += __shfl_xor(x[q][j], off, 64);
                    const float Lq = __shfl(L, 16 * q, 64);
                    if (r + q < rows && lane < TPR) store(r + q, x[q], Lq);
                }
            }
            continue;
        }
        for (int r = block % groups; r < rows; r += groups) {
            float M = -INFINITY, L = 0.f;
            for (int p = lane; p < parts; p += 64) M = fmaxf(M, ml[(merge_at(p) * stride + r) * 2]);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int p = group; p < parts; p += NG) {
                const float2 f = *(const float2 *)(ml + (merge_at(p) * stride + r) * 2);
                const f32x4 y = *(const f32x4 *)(o + (merge_at(p) * stride + r) * HD);
                const float w = f.x == -INFINITY ? 0.f : pexp2(f.x - M);
                L += w * f.y;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] += w * y[j];
            }
            xs[group][d4] = x;
            if (d4 == 0) ls[group] = L;
            __syncthreads();
            if (group == 0) {
                for (int n = 1; n < NG; ++n) {
                    L += ls[n];
                    const f32x4 y = xs[n][d4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] += y[j];
                }
                store(r, x, L);
            }
            __syncthreads();
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
constexpr int kFewRows = 32;        // (token, head) rows of a sequence and kv head up to which paged_rows_kernel takes it
// Its workgroups: two on each of the 256 CUs.  64 sequences of 2000 positions take 97 us so, 100 us with half as many, and 100 us with
// twice as many, whose partials are twice as many too (32 sequences of 4 rows: 66, 61 and 73 us).
constexpr int kStreams = 512;
// Most blocks that a table has room for (the host knows no lengths: a wide table is planned for long ones) up to which no unit is
// split, which saves the partials and the kernel that adds them up; for fewer than 32 units, which leave most CUs idle, and for more.  8 kv heads, bf16, one sequence of 700 positions: 12.1 us so and
// 12.9 us split, of 1000: 14.6 and 12.3 us; 64 sequences of up to 1000: 41 and 51 us, 256: 154 and 152 us.  (fp32, nine chunks of up to
// 60 rows at up to 960 positions, 15 blocks: 25 and 16 us.)
constexpr int kWholeBlocksFew = 6, kWholeBlocks = 8;
constexpr int kTileStreams = 256;   // workgroups of the other kernel, each of which fills a CU
constexpr int kStreamBlocks = 1;    // fewest blocks (a step for each wave) of one

static size_t take(size_t *end, size_t bytes)
{
    const size_t at = *end;
    *end = (at + bytes + 255) & ~(size_t)255;
    return at;
}
// units that a call can have: those of its rows, and a last one in part for each sequence that can have so many rows
static int64_t most_units(int rows, int rows_above, int rows_most, const PagedView &p, int G)
{
    const int64_t all = (int64_t)p.n_rows * G, seqs = std::min<int64_t>(p.n_seqs, all / (rows_above + 1));
    return std::min(all / rows + seqs, seqs * ((rows_most - 1) / rows + 1)) * p.Hkv;
}

// Sequences of up to kFewRows rows are bound by reading their keys, the others by the matrix pipe: one kernel for each kind,
// and as the host does not know which a call has, both are launched unless every sequence has one row.  fp32 has the first
// kernel alone.  At the border, 32 heads on 8 of 128 channels, 64 sequences of 2000 positions: 8 rows each (32 with their heads) take
// 110 us by the one and 170 us by the other, 16 rows each 203 us and 174 us.
PagedAttnPlan paged_attn_plan(int kind, int hd, const PagedView &p, int Hq)
{
    const int G = Hq / p.Hkv, most = 0x7fffffff;
    const int64_t max_len = (int64_t)p.width << p.ps_log;
    PagedAttnPlan r;
    memset(&r, 0, sizeof(r));
    const bool one = !p.starts, tiles = kind != PAGED_F32;
    if (!one || !tiles || G <= kFewRows) {
        PagedAttnPart &t = r.few;
        t.rows = one && G <= 16 ? 16 : 32;
        t.rows_most = tiles && !one ? kFewRows : most;
        t.least = kStreamBlocks;
        const int64_t units = most_units(t.rows, 0, t.rows_most, p, G), block = kWaves * (kind == PAGED_F32 ? 16 : 32);
        const int64_t blocks = (max_len + block - 1) / block;
        t.whole = blocks <= (units < 32 ? kWholeBlocksFew : kWholeBlocks);
        t.grid = (unsigned)std::min<int64_t>(kStreams, t.whole ? units : units * blocks);
        t.used = units > 0;
        t.merge = t.used && !t.whole && blocks > 1 && t.grid > 1;
        if (t.merge) {
            t.cap_units = (int)t.grid;
            t.cap_items = 2 * (int)t.grid;
            t.merge_groups = std::min(one ? std::min(G, t.rows) : t.rows, 8);
            t.merge_units = kMergeUnits;
        }
    }
    if (tiles && (!one || G > kFewRows)) {
        PagedAttnPart &t = r.many;
        t.rows = 256;
        t.rows_above = one ? 0 : kFewRows;
        t.rows_most = most;
        t.least = 4;                // (a prompt of 200 tokens: 27 us, 35 us with eight)
        const int64_t units = most_units(t.rows, t.rows_above, t.rows_most, p, G), parts = (max_len + 255) / 256;
        t.grid = (unsigned)std::min<int64_t>(kTileStreams, units * std::max<int64_t>(parts, 1));
        t.used = units > 0;
        t.merge = t.used && max_len > 448 && t.grid > 1;        // (a unit of fewer than eight tiles is never split)
        if (t.merge) {
            t.cap_units = (int)t.grid;
            t.cap_items = 2 * (int)t.grid;
            t.merge_groups = 16;
            t.merge_units = 2;
        }
    }
    for (PagedAttnPart *t : {&r.few, &r.many}) {
        t->off_desc = take(&r.bytes, (size_t)t->cap_units * 32);
        t->off_ml = take(&r.bytes, (size_t)t->cap_items * t->rows * 8);
        t->off_o = take(&r.bytes, (size_t)t->cap_items * t->rows * hd * 4);
    }
    return r;
}

static PagedAttnArgs part_args(PagedAttnArgs a, const PagedAttnPart &t, char *ws)
{
    a.rows_above = t.rows_above; a.rows_most = t.rows_most; a.least = t.least; a.whole = t.whole;
    if (!t.merge) return a;
    a.parts.desc = (int32_t *)(ws + t.off_desc);
    a.parts.ml = (float *)(ws + t.off_ml);
    a.parts.o = (float *)(ws + t.off_o);
    a.parts.units = t.cap_units;
    a.parts.rows = t.rows;
    a.parts.merge_groups = t.merge_groups;
    a.parts.merge_units = t.merge_units;
    return a;
}

template <int KIND, int HD, int NR>
static hipError_t launch_rows(const PagedAttnArgs &a, unsigned grid, hipStream_t s)
{
    constexpr int lds = kWaves * 16 * NR * (HD + 6) * 4;
    static OncePerDevice attr;
    int dev;
    if (attr.need(&dev)) {
        hipError_t e = hipFuncSetAttribute((const void *)paged_rows_kernel<KIND, HD, NR>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        attr.mark(dev);
    }
    paged_rows_kernel<KIND, HD, NR><<<grid, 256, lds, s>>>(a);
    return hipGetLastError();
}

template <int KIND, int HD>
static hipError_t launch_kind(const PagedAttnArgs &a, const PagedAttnPlan &plan, char *ws, hipStream_t s)
{
    const PagedAttnArgs few = part_args(a, plan.few, ws), many = part_args(a, plan.many, ws);
    hipError_t e = hipSuccess;
    if (plan.many.used) e = launch_paged_tiles(KIND, HD, many, plan.many.grid, s);
    if (e == hipSuccess && plan.few.used)
        e = plan.few.rows == 16 ? launch_rows<KIND, HD, 1>(few, plan.few.grid, s) : launch_rows<KIND, HD, 2>(few, plan.few.grid, s);
    auto merge_blocks = [](const PagedParts &p) { return p.units ? (p.units + p.merge_units - 1) / p.merge_units * p.merge_groups : 0; };
    const int blocks = merge_blocks(few.parts) + merge_blocks(many.parts);
    if (e != hipSuccess || blocks == 0) return e;
    paged_merge_kernel<KIND, HD><<<blocks, 256, 0, s>>>(a, few.parts, many.parts);
    return hipGetLastError();
}

hipError_t launch_paged_attention(int kind, int hd, const PagedAttnArgs &a, const PagedAttnPlan &plan, char *ws, hipStream_t s)
{
    if (kind == PAGED_BF16) return hd == 128 ? launch_kind<PAGED_BF16, 128>(a, plan, ws, s) : launch_kind<PAGED_BF16, 64>(a, plan, ws, s);
    if (kind == PAGED_E4M3) return hd == 128 ? launch_kind<PAGED_E4M3, 128>(a, plan, ws, s) : launch_kind<PAGED_E4M3, 64>(a, plan, ws, s);
    return hd == 128 ? launch_kind<PAGED_F32, 128>(a, plan, ws, s) : launch_kind<PAGED_F32, 64>(a, plan, ws, s);
}

}  // namespace pd
