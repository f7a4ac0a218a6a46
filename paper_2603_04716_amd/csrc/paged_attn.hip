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
    __shared__ PagedShared<256> sh;
    const PagedView &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedItems it = paged_divide<R, 256>(a, sh);
    if (blockIdx.x == 0 && tid == 0 && a.parts.head) a.parts.head[0] = it.split_units * p.Hkv;
    const float sl2e = a.scale * 1.4426950408889634f;

    const int t = blockIdx.x / p.Hkv, g = blockIdx.x - t * p.Hkv;
    if (t >= it.total) return;
    paged_find<R>(a, it, t, &sh.found);
    const int b = __builtin_amdgcn_readfirstlane(sh.found.seq), units = __builtin_amdgcn_readfirstlane(sh.found.units);
    const int nc = __builtin_amdgcn_readfirstlane(sh.found.chunks), at = __builtin_amdgcn_readfirstlane(sh.found.at);
    const int start = __builtin_amdgcn_readfirstlane(sh.found.start), rows = __builtin_amdgcn_readfirstlane(sh.found.rows);
    const int len = __builtin_amdgcn_readfirstlane(sh.found.len);
    // row tiles that read the same keys are neighbours, the one that sees most first
    const int c = at / units, u = units - 1 - (at - c * units);
    const int r0 = u * R, nrows = min(R, rows * a.G - r0);
    const int before = len - rows;               // position of the sequence's first row (negative: it is not held)
    const int vis_min = before + r0 / a.G + 1, vis_max = max(before + (r0 + nrows - 1) / a.G + 1, 0);
    const int nc_u = max((vis_max + it.chunk - 1) / it.chunk, 1);
    if (c >= nc_u) return;
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
            const int id = load_const(pages, at >> p.ps_log);
            gone[kb] = id < 0 || id >= p.n_pages;
            const size_t unit = (size_t)(gone[kb] ? 0 : id) * p.Hkv + g;
            const size_t off = ((unit << p.ps_log) + (key & ((1 << p.ps_log) - 1))) * HD;
            st.load(kb, (const typename S::elem *)p.k + off, (const typename S::elem *)p.v + off,
                    KIND == PAGED_E4M3 ? load_const(p.k_scales, unit) : 1.f, KIND == PAGED_E4M3 ? load_const(p.v_scales, unit) : 1.f, n, kg);
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
                const int id = load_const(pages, key >> p.ps_log);
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
    const int part0 = (sh.found.split + u * nc) * p.Hkv + g * nc_u;       // first partial of the unit
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
    if (nc > 1 && c == 0 && tid == 0)
        paged_describe(a, (sh.found.unit + u) * p.Hkv + g, part0, nc_u, start, r0, rows * a.G, g, before);
}

// Adds up the partials of a split unit: o = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c.  A workgroup takes a row at a
// time, its four waves the row's partials in turn; first the few-row kernel's units, then the other's.
template <int KIND, int HD>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a, PagedParts few, PagedParts many)
{
    typedef typename std::conditional<KIND == PAGED_F32, float, bf16_t>::type T;
    constexpr int CH = HD / 64;
    __shared__ float xs[kWaves][HD], ls[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tasks_few = few.head ? few.head[0] * few.rows : 0, tasks = tasks_few + (many.head ? many.head[0] * many.rows : 0);
    for (int t = blockIdx.x; t < tasks; t += gridDim.x) {
        const PagedParts &from = t < tasks_few ? few : many;
        const int at_task = t < tasks_few ? t : t - tasks_few, R = from.rows, lr = at_task % R;
        const int32_t *desc = from.desc + (size_t)(at_task / R) * 8;
        const int part0 = desc[0], nc = desc[1], start = desc[2], r = desc[3] + lr, rows = desc[4], g = desc[5], before = desc[6];
        if (nc == 1 || r >= rows) continue;
        float M = -INFINITY;
        for (int c = lane; c < nc; c += 64) M = fmaxf(M, from.ml[((size_t)(part0 + c) * R + lr) * 2]);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
        float x[CH] = {}, L = 0.f;
#pragma unroll 4
        for (int c = wave; c < nc; c += kWaves) {
            const size_t at = (size_t)(part0 + c) * R + lr;
            const float2 ml = *(const float2 *)(from.ml + at * 2);
            const float w = ml.x == -INFINITY ? 0.f : pexp2(ml.x - M);
            L += w * ml.y;
#pragma unroll
            for (int i = 0; i < CH; ++i) x[i] += w * from.o[at * HD + CH * lane + i];
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
constexpr int kFewRows = 32;        // (token, head) rows of a sequence and kv head up to which paged_rows_kernel takes it

static PagedAttnPart plan_part(int rows, int rows_above, int rows_most, int chunk_min, int target, int hd, const PagedView &p, int G, size_t *end)
{
    PagedAttnPart r;
    r.rows = rows; r.rows_above = rows_above; r.rows_most = rows_most; r.chunk_min = chunk_min; r.target = target;
    // a unit of each sequence may be in part, and no sequence has more rows than rows_most
    const int64_t all = (int64_t)p.n_rows * G;
    const int64_t seqs = std::min<int64_t>(p.n_seqs, all / (rows_above + 1));
    r.units = std::min(all / rows + seqs, seqs * ((rows_most - 1) / rows + 1)) * p.Hkv;
    r.used = r.units > 0;
    r.chunks = (((int64_t)p.width << p.ps_log) + chunk_min - 1) / chunk_min;
    r.merge = r.used && r.chunks > 1;
    r.cap_items = r.merge ? (int)std::min<int64_t>(2 * target, r.units * r.chunks) : 0;
    r.cap_units = r.merge ? (int)std::min<int64_t>(target, r.units) : 0;
    auto take = [&](size_t bytes) {
        const size_t at = *end;
        *end = (at + bytes + 255) & ~(size_t)255;
        return at;
    };
    r.off_head = take(r.merge ? 4 : 0);
    r.off_desc = take((size_t)r.cap_units * 32);
    r.off_ml = take((size_t)r.cap_items * rows * 8);
    r.off_o = take((size_t)r.cap_items * rows * hd * 4);
    return r;
}

// Sequences of up to kFewRows rows are bound by reading their keys, the others by the matrix pipe: one kernel for each kind,
// and as the host does not know which a call has, both are launched unless every sequence has one row.  fp32 has the first
// kernel alone.
PagedAttnPlan paged_attn_plan(int kind, int hd, const PagedView &p, int Hq)
{
    const int G = Hq / p.Hkv, most = 0x7fffffff;
    PagedAttnPlan r;
    r.bytes = 0;
    r.few.used = r.many.used = r.few.merge = r.many.merge = false;
    const bool one = !p.starts, tiles = kind != PAGED_F32;
    // 256 keys are two steps for each of the four waves; 1024 items two workgroups on each of 256 CUs, twice over
    if (!one || !tiles || G <= kFewRows)
        r.few = plan_part(one && G <= 16 ? 16 : 32, 0, tiles && !one ? kFewRows : most, 256, 1024, hd, p, G, &r.bytes);
    // 512 keys are eight tiles; 256 items one workgroup on each CU
    if (tiles && (!one || G > kFewRows)) r.many = plan_part(256, one ? 0 : kFewRows, most, 512, 256, hd, p, G, &r.bytes);
    return r;
}

static PagedAttnArgs part_args(PagedAttnArgs a, const PagedAttnPart &t, char *ws)
{
    a.rows_above = t.rows_above; a.rows_most = t.rows_most; a.chunk_min = t.chunk_min; a.target = t.target;
    a.parts.head = t.merge ? (int32_t *)(ws + t.off_head) : nullptr;
    a.parts.desc = (int32_t *)(ws + t.off_desc);
    a.parts.ml = (float *)(ws + t.off_ml);
    a.parts.o = (float *)(ws + t.off_o);
    a.parts.rows = t.rows;
    return a;
}
static unsigned part_grid(const PagedAttnPart &t)
{
    // items of a call: a chunk more than len / chunk for every unit, and no more than all chunks of all units
    return (unsigned)std::min(t.units + t.target, t.units * t.chunks);
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
    if (plan.many.used) e = launch_paged_tiles(KIND, HD, many, part_grid(plan.many), s);
    if (e == hipSuccess && plan.few.used)
        e = plan.few.rows == 16 ? launch_rows<KIND, HD, 1>(few, part_grid(plan.few), s) : launch_rows<KIND, HD, 2>(few, part_grid(plan.few), s);
    const int tasks = std::max(plan.few.merge ? plan.few.cap_units * plan.few.rows : 0, plan.many.merge ? plan.many.cap_units * plan.many.rows : 0);
    if (e != hipSuccess || tasks == 0) return e;
    paged_merge_kernel<KIND, HD><<<std::min(tasks, 2048), 256, 0, s>>>(a, few.parts, many.parts);
    return hipGetLastError();
}

hipError_t launch_paged_attention(int kind, int hd, const PagedAttnArgs &a, const PagedAttnPlan &plan, char *ws, hipStream_t s)
{
    if (kind == PAGED_BF16) return hd == 128 ? launch_kind<PAGED_BF16, 128>(a, plan, ws, s) : launch_kind<PAGED_BF16, 64>(a, plan, ws, s);
    if (kind == PAGED_E4M3) return hd == 128 ? launch_kind<PAGED_E4M3, 128>(a, plan, ws, s) : launch_kind<PAGED_E4M3, 64>(a, plan, ws, s);
    return hd == 128 ? launch_kind<PAGED_F32, 128>(a, plan, ws, s) : launch_kind<PAGED_F32, 64>(a, plan, ws, s);
}

}  // namespace pd
