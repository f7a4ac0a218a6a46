// Attention over a paged cache for many query rows of a sequence (chunks, whole prompts): bf16 rows, bf16 or E4M3 pages.
//
// With hundreds of query rows the matrix pipe is the bound, and what has to be kept from it is the delivery of keys and values.
// A unit is 256 (token, head) rows of one sequence and kv head, 32 for each of eight waves, so that a tile of 64 keys and
// values comes through the L2 once for 256 rows; heads of a group share it.  Everything is computed transposed:
//
//   S^T[key, row] = K[key, :] . Q[row, :]       A = key rows from LDS, B = the wave's rows, in registers throughout
//   O^T[c, row]   = V^T[c, key] . P^T[key, row]  A = value columns from LDS, B = the exponentials in the registers and the
//                                               order in which the first product leaves them
//
// and a lane's column is one row in both, so that the softmax's maximum and sum are lane-local but for the other half of the
// wave.  Pages hold values row by row; gfx950 reads an LDS tile by columns (ds_read_b64_tr_b16: 16 lanes fetch four rows of 16
// values and each gets one column), so no transposed copy of the values is made anywhere, and any four rows can be
// taken together, which is how the second product takes keys in the accumulators' order without moving the exponentials.
//
// bf16 tiles go from the pages to LDS directly, four (hd 128) or eight (hd 64) rows an instruction - a page holds at least
// 16 - in a ring of four tiles, one barrier a tile.  E4M3 tiles are loaded two tiles ahead into registers, widened (a code
// times its page's scale is exact in bf16) and written to a ring of two: widened by the workgroup once, not by every wave.
#include <type_traits>

#include "paged_items.h"

namespace pd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef const void __attribute__((address_space(1))) *gptr_t;
typedef void __attribute__((address_space(3))) *lptr_t;
typedef s16x4 __attribute__((address_space(3))) *trptr_t;

// s_waitcnt with only the vector-memory count set: at most n of the wave's loads still in flight
#define PD_TILE_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (15 << 8) | (((n) >> 4) << 14))

constexpr int kTileRows = 256, kTileKeys = 64;
constexpr float kNoScore = -3.0e38f;             // running maximum before any score: finite, so that differences are defined
constexpr float kLazyRaise = 8.0f;               // the maximum is raised when a score exceeds it by 2^8: sums stay exact in fp32
__device__ __align__(16) unsigned char paged_zeros[16];     // what keys and values that are not there are loaded from

// Byte offset of the 16-byte piece c of row r in a K or V tile.  K is read 32 rows at one piece index, V four rows at 64
// bytes' worth of neighbouring pieces; the exclusive-ors spread both over all banks.
template <int HD>
__device__ __forceinline__ int k_off(int r, int c) { return r * HD * 2 + (HD == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7)) * 16; }
template <int HD>
__device__ __forceinline__ int v_off(int r, int c) { return r * HD * 2 + (HD == 128 ? c ^ ((r & 3) << 2) : c ^ (((r >> 1) & 1) << 2)) * 16; }

template <int KIND, int HD>
__global__ __launch_bounds__(512, 1) void paged_tiles_kernel(PagedAttnArgs a)
{
    constexpr int NST = KIND == PAGED_BF16 ? 4 : 2, TILE = kTileKeys * HD * 2, STAGE = 2 * TILE;
    constexpr int NK = HD / 16, NDB = HD / 32;       // k-steps of a score, 32-channel blocks of the output
    constexpr int AHEAD = NST - 1;
    constexpr int LPW = TILE / 1024 / 8;             // bf16: load instructions per wave for each of K and V
    constexpr int RPI = 1024 / (HD * 2);             // ... rows of one
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ PagedShared<512> sh;
    const PagedView &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedItems it = paged_divide<kTileRows, 512>(a, sh);
    if (blockIdx.x == 0 && tid == 0 && a.parts.head) a.parts.head[0] = it.split_units * p.Hkv;
    const float sl2e = a.scale * 1.4426950408889634f;
    const int ps_mask = (1 << p.ps_log) - 1;

    const int t = blockIdx.x / p.Hkv, g = blockIdx.x - t * p.Hkv;
    if (t >= it.total) return;
    paged_find<kTileRows>(a, it, t, &sh.found);
    const int b = __builtin_amdgcn_readfirstlane(sh.found.seq), units = __builtin_amdgcn_readfirstlane(sh.found.units);
    const int nc = __builtin_amdgcn_readfirstlane(sh.found.chunks), at = __builtin_amdgcn_readfirstlane(sh.found.at);
    const int start = paged_start(p, b), rows = paged_rows(p, b, start), len = paged_len(p, b);
    const int c = at / units, u = units - 1 - (at - c * units);     // the tile that sees most keys first
    const int r0 = u * kTileRows, nrows = min(kTileRows, rows * a.G - r0);
    const int before = len - rows;
    const int vis_max = max(before + (r0 + nrows - 1) / a.G + 1, 0);
    const int nc_u = max((vis_max + it.chunk - 1) / it.chunk, 1);
    const int part0 = (sh.found.split + u * nc) * p.Hkv + g * nc_u;
    if (tid == 0 && nc > 1 && c == 0)
        paged_describe(a, (sh.found.unit + u) * p.Hkv + g, part0, nc_u, start, r0, rows * a.G, g, before);
    const int c0 = c * it.chunk, c1 = min(vis_max, c0 + it.chunk);
    if (c >= nc_u) return;

    // ---- the wave's rows
    const int w0 = wave * 32, row = r0 + w0 + n, tok = row / a.G;
    const bool ok = w0 + n < nrows;
    const int limit = ok ? before + tok + 1 : 0;                    // the row sees keys 0 .. limit - 1
    // keys that the wave's first and last row see
    const int w_min = before + (r0 + w0) / a.G + 1, w_max = w0 < nrows ? before + (r0 + min(w0 + 31, nrows - 1)) / a.G + 1 : 0;
    bf16x8 qf[NK];
    {
        const uint16_t *q = (const uint16_t *)a.q + (start + tok) * a.q_stride + (g * a.G + row - tok * a.G) * HD + 8 * h;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            u32x4 w = {0u, 0u, 0u, 0u};
            if (ok) w = *(const u32x4 *)(q + 16 * k);
            qf[k] = __builtin_bit_cast(bf16x8, w);
        }
    }
    f32x16 o[NDB];
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float m_run = kNoScore, l_run = 0.f;

    const int32_t *pages = p.table + (size_t)b * p.width;
    const int t_lo = c0 / kTileKeys, t_hi = (c1 + kTileKeys - 1) / kTileKeys;

    // ---- tile loaders ----
    // bf16: instruction i of a wave brings rows RPI (8 i + wave) .. of the tile.  Its page number is asked for one tile
    // before its rows are.
    int ids[LPW > 0 ? LPW : 1];
    auto ask = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LPW; ++i) ids[i] = load_const(pages, min(j * kTileKeys + RPI * (8 * i + wave), len - 1) >> p.ps_log);
    };
    auto issue = [&](int j, unsigned char *st) __attribute__((always_inline)) {
        const int lr = lane / (64 / RPI), slot = lane & (64 / RPI - 1);
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = RPI * (8 * i + wave), key = j * kTileKeys + r;
            const bool there = ids[i] >= 0 && ids[i] < p.n_pages;
            const size_t base = ((((size_t)(there ? ids[i] : 0) * p.Hkv + g) << p.ps_log) + (key & ps_mask)) * (HD * 2);
            const char *kp = (const char *)p.k + base + (k_off<HD>(r + lr, slot) - r * HD * 2);
            const char *vp = (const char *)p.v + base + (v_off<HD>(r + lr, slot) - r * HD * 2);
            if (!there || key + RPI > c1) {      // keys that nobody sees, or whose page is not there: zeros
                const bool in = there && key + lr < c1;
                kp = in ? kp : (const char *)paged_zeros;
                vp = in ? vp : (const char *)paged_zeros;
            }
            __builtin_amdgcn_global_load_lds((gptr_t)kp, (lptr_t)(st + r * HD * 2), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((gptr_t)vp, (lptr_t)(st + TILE + r * HD * 2), 16, 0, 0);
        }
    };
    // E4M3: eight threads a row, HD / 8 codes each
    constexpr int CW = HD / 32;                  // registers of codes
    unsigned kc[CW], vc[CW];
    float k_sc = 1.f, v_sc = 1.f;
    const int cr = tid >> 3, cp = tid & 7;
    auto fetch = [&](int j) __attribute__((always_inline)) {
        const int key = j * kTileKeys + cr;
        const int id = load_const(pages, min(j * kTileKeys + (wave << 3), len - 1) >> p.ps_log);
        const bool there = id >= 0 && id < p.n_pages;
        const size_t unit = (size_t)(there ? id : 0) * p.Hkv + g;
        const size_t off = ((unit << p.ps_log) + (key & ps_mask)) * HD + cp * (HD / 8);
        k_sc = load_const(p.k_scales, unit);
        v_sc = load_const(p.v_scales, unit);
        const bool in = there && key < c1;
        if (HD == 128) {
            const u32x4 kw = *(const u32x4 *)((const uint8_t *)p.k + off), vw = *(const u32x4 *)((const uint8_t *)p.v + off);
#pragma unroll
            for (int i = 0; i < CW; ++i) {
                kc[i] = in ? kw[i & 3] : 0u;
                vc[i] = in ? vw[i & 3] : 0u;
            }
        } else {
            const u32x2 kw = *(const u32x2 *)((const uint8_t *)p.k + off), vw = *(const u32x2 *)((const uint8_t *)p.v + off);
#pragma unroll
            for (int i = 0; i < CW; ++i) {
                kc[i] = in ? kw[i & 1] : 0u;
                vc[i] = in ? vw[i & 1] : 0u;
            }
        }
    };
    auto widen4 = [](unsigned lo, unsigned hi, float s) {
        return u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true))};
    };
    auto commit = [&](unsigned char *st) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CW / 2; ++i) {
            *(u32x4 *)(st + k_off<HD>(cr, cp * (CW / 2) + i)) = widen4(kc[2 * i], kc[2 * i + 1], k_sc);
            *(u32x4 *)(st + TILE + v_off<HD>(cr, cp * (CW / 2) + i)) = widen4(vc[2 * i], vc[2 * i + 1], v_sc);
        }
    };

    // ---- one tile out of stage st of the ring, while the one for which there is room goes to st_to; PART: some row of the unit
    // does not see all of its keys ----
    auto tile = [&](const int j, const unsigned char *st, unsigned char *st_to, auto PART) __attribute__((always_inline)) {
        if (KIND == PAGED_BF16) {
            // Loads retire in order: with at most the requests of the AHEAD - 1 later tiles in flight this wave's part of
            // tile j has landed, after the barrier every wave's, and every wave is done with tile j - 1, whose stage
            // the request for tile j + AHEAD overwrites.  Past the last tile it is requested again, so that the count
            // stays the same.
            PD_TILE_VMCNT((AHEAD - 1) * 2 * LPW);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            issue(min(j + AHEAD, t_hi - 1), st_to);
            ask(min(j + AHEAD + 1, t_hi - 1));
        } else {
            __syncthreads();                     // tile j is written, and tile j - 1 read
            commit(st_to);
            fetch(min(j + 2, t_hi - 1));
        }
        __builtin_amdgcn_sched_barrier(0);
        const int k0 = j * kTileKeys;
        if (k0 >= w_max) return;                 // wave-uniform: no row of the wave sees a key of this tile
        f32x16 s[2];
        bf16x8 kf[2 * NK];
#pragma unroll
        for (int i = 0; i < 2 * NK; ++i) kf[i] = *(const bf16x8 *)(st + k_off<HD>(32 * (i / NK) + n, 2 * (i % NK) + h));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * NK; ++i) s[i / NK] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i % NK], s[i / NK], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        // Value columns: operand (db, ks) is channels 32 db .. + 31 of the keys whose exponentials are registers
        // 8 (ks % 2) .. + 7 of s[ks / 2]: keys 16 ks + 4 h + {0 .. 3, 8 .. 11}, four rows a read.
        // Half of them are requested here and land during the softmax, the others behind it, when the scores' registers are
        // free, and land during the first half's products.
        u32x4 vf[NDB][4];
        auto load_v = [&](int ks) {
#pragma unroll
            for (int db = 0; db < NDB; ++db) {
                const int r = 16 * ks + 4 * h + ((lane & 15) >> 2), piece = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((trptr_t)(st + TILE + v_off<HD>(r, piece) + 8 * (lane & 1))));
                const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((trptr_t)(st + TILE + v_off<HD>(r + 8, piece) + 8 * (lane & 1))));
                vf[db][ks] = u32x4{lo[0], lo[1], hi[0], hi[1]};
            }
        };
        load_v(0);
        load_v(1);
        __builtin_amdgcn_sched_barrier(0);
        // ---- softmax: p = 2^(s scale log2 e - m) ----
        const bool part = decltype(PART)::value && k0 + kTileKeys > w_min;   // ... and of the wave
        if (part)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + 32 * kb + 8 * (r >> 2) + 4 * h + (r & 3) >= limit) s[kb][r] = -INFINITY;
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
        {
            const unsigned mb = __builtin_bit_cast(unsigned, mx);
            auto sw = __builtin_amdgcn_permlane32_swap(mb, mb, false, false);
            mx = fmaxf(__builtin_bit_cast(float, (unsigned)sw[0]), __builtin_bit_cast(float, (unsigned)sw[1]));
        }
        const float m_cand = fmaxf(m_run, mx * sl2e);
        if (__any(m_cand - m_run > kLazyRaise)) {
            const float alpha = pexp2(m_run - m_cand);
            m_run = m_cand;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < NDB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
        }
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = pexp2(fmaf(s[kb][r], sl2e, -m_run));
                sum += s[kb][r];
            }
        l_run += sum;
        bf16x8 pf[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int r = 8 * (ks & 1);
            pf[ks] = __builtin_bit_cast(bf16x8, u32x4{pack2bf(s[ks >> 1][r], s[ks >> 1][r + 1]), pack2bf(s[ks >> 1][r + 2], s[ks >> 1][r + 3]),
                                                      pack2bf(s[ks >> 1][r + 4], s[ks >> 1][r + 5]), pack2bf(s[ks >> 1][r + 6], s[ks >> 1][r + 7])});
        }
        __builtin_amdgcn_sched_barrier(0);
        load_v(2);
        load_v(3);
        __builtin_amdgcn_sched_barrier(0);
        // A value that is not finite must not reach a row that does not see it, but 0 * infinity would: in a tile seen in
        // part such values leave the product and are added to the rows that see them one by one.
        bool odd = false;
        if (part)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned x = vf[db][ks][i];
                        const unsigned fin = ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
                        odd |= fin != x;
                        vf[db][ks][i] = fin;
                    }
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int db = 0; db < NDB; ++db)
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[db][ks]), pf[ks], o[db], 0, 0, 0);
        if (decltype(PART)::value && __any(odd))
#pragma unroll 1
            for (int key = k0; key < min(k0 + kTileKeys, c1); ++key) {
#pragma unroll
                for (int db = 0; db < NDB; ++db)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        const u32x2 w = *(const u32x2 *)(st + TILE + v_off<HD>(key - k0, 4 * db + q4) + 8 * h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = bfbits2f((w[e >> 1] >> (16 * (e & 1))) & 0xffffu);
                            if (!(fabsf(x) < INFINITY) && key < limit) o[db][4 * q4 + e] += x;
                        }
                    }
            }
    };
    if (t_lo < t_hi) {
        if (KIND == PAGED_BF16) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                ask(min(t_lo + i, t_hi - 1));
                issue(min(t_lo + i, t_hi - 1), smem + i * STAGE);
                __builtin_amdgcn_sched_barrier(0);
            }
            ask(min(t_lo + AHEAD, t_hi - 1));
        } else {
            fetch(t_lo);
            commit(smem);
            fetch(min(t_lo + 1, t_hi - 1));
        }
        // the unit's first row sees keys 0 .. vis_min - 1: the tiles below are seen whole by every row, and their stages are
        // constants, so that a tile's LDS addresses are registers plus immediates
        const int t_full = max(t_lo, min(t_hi, (before + r0 / a.G + 1) / kTileKeys));
        auto full = [&](int j, auto STG) __attribute__((always_inline)) {
            constexpr int stg = decltype(STG)::value;
            if (j < t_full) tile(j, smem + stg * STAGE, smem + (stg + AHEAD) % NST * STAGE, std::false_type{});
        };
        for (int j = t_lo; j < t_full; j += NST) {
            full(j, std::integral_constant<int, 0>{});
            full(j + 1, std::integral_constant<int, 1>{});
            if (NST == 4) {
                full(j + 2, std::integral_constant<int, 2 % NST>{});
                full(j + 3, std::integral_constant<int, 3 % NST>{});
            }
        }
        for (int j = t_full; j < t_hi; ++j) tile(j, smem + (j - t_lo) % NST * STAGE, smem + (j - t_lo + AHEAD) % NST * STAGE, std::true_type{});
        // the repeated requests of the last tile: none may outlive the workgroup's LDS
        if (KIND == PAGED_BF16) PD_TILE_VMCNT(0);
    }

    // ---- a lane holds row `row`, channels 32 db + 8 (r / 4) + 4 h + r % 4 ----
    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    if (ok && nc_u == 1) {
        const float inv = 1.f / l_tot;
        uint16_t *op = (uint16_t *)a.out + ((size_t)(start + tok) * a.Hq + g * a.G + row - tok * a.G) * HD + 4 * h;
        const bool none = limit <= 0;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : o[db][4 * q4 + e] * inv;
                *(uint2 *)(op + 32 * db + 8 * q4) = make_uint2(pack2bf(x[0], x[1]), pack2bf(x[2], x[3]));
            }
    } else if (ok) {
        const size_t at_part = (size_t)(part0 + c) * kTileRows + w0 + n;
        float *op = a.parts.o + at_part * HD + 4 * h;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *(float4 *)(op + 32 * db + 8 * q4) = make_float4(o[db][4 * q4], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]);
        if (h == 0) *(float2 *)(a.parts.ml + at_part * 2) = make_float2(m_run, l_tot);
    }
}

template <int KIND, int HD>
static hipError_t launch_tiles(const PagedAttnArgs &a, unsigned grid, hipStream_t s)
{
    constexpr int lds = (KIND == PAGED_BF16 ? 4 : 2) * 2 * kTileKeys * HD * 2;
    static OncePerDevice attr;
    int dev;
    if (attr.need(&dev)) {
        hipError_t e = hipFuncSetAttribute((const void *)paged_tiles_kernel<KIND, HD>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        attr.mark(dev);
    }
    paged_tiles_kernel<KIND, HD><<<grid, 512, lds, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_tiles(int kind, int hd, const PagedAttnArgs &a, unsigned grid, hipStream_t s)
{
    if (kind == PAGED_E4M3) return hd == 128 ? launch_tiles<PAGED_E4M3, 128>(a, grid, s) : launch_tiles<PAGED_E4M3, 64>(a, grid, s);
    return hd == 128 ? launch_tiles<PAGED_BF16, 128>(a, grid, s) : launch_tiles<PAGED_BF16, 64>(a, grid, s);
}

}  // namespace pd
