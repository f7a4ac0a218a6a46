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
typedef void __attribute__((address_space(3))) *lptr_t;
typedef s16x4 __attribute__((address_space(3))) *trptr_t;

// s_waitcnt with only the vector-memory count set: at most n of the wave's loads still in flight
#define PD_TILE_VMCNT(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (15 << 8) | (((n) >> 4) << 14))

// s_waitcnt for the wave's own LDS accesses
#define PD_TILE_LGKM0() __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14))

constexpr int kTileRows = 256, kTileKeys = 64;
constexpr float kNoScore = -3.0e38f;             // running maximum before any score: finite, so that differences are defined
constexpr float kLazyRaise = 8.0f;               // the maximum is raised when a score exceeds it by 2^8: sums stay exact in fp32

// Byte offset of the 16-byte piece c of row r in a K or V tile.  K is read 32 rows at one piece index, V four rows at 64
// bytes' worth of neighbouring pieces; the exclusive-ors spread both over all banks.
template <int HD>
__device__ __forceinline__ int k_off(int r, int c) { return r * HD * 2 + (HD == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7)) * 16; }
template <int HD>
__device__ __forceinline__ int v_off(int r, int c) { return r * HD * 2 + (HD == 128 ? c ^ ((r & 3) << 2) : c ^ (((r >> 1) & 1) << 2)) * 16; }

template <int KIND, int HD>
__global__ __launch_bounds__(512, 1) void paged_tiles_kernel(PagedAttnArgs a)
{
    // stages of the ring: K tiles, then V tiles, so that all stages of either lie within an LDS instruction's 64 KB immediate
    constexpr int NST = 4, TILE = kTileKeys * HD * 2, VRING = NST * TILE;
    constexpr int NK = HD / 16, NDB = HD / 32;       // k-steps of a score, 32-channel blocks of the output
    constexpr int LPW = TILE / 1024 / 8;             // bf16: load instructions per wave for each of K and V
    constexpr int RPI = 1024 / (HD * 2);             // ... rows of one
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ PagedShared<512> sh;
    __shared__ int again;
    const PagedView &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63;
    int n = lane & 31, h = lane >> 5;
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
    const int start = __builtin_amdgcn_readfirstlane(sh.found.start), rows = __builtin_amdgcn_readfirstlane(sh.found.rows);
    const int len = __builtin_amdgcn_readfirstlane(sh.found.len);
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
    const int w_min = before + (r0 + w0) / a.G + 1;                     // ... and the wave's first row 0 .. w_min - 1
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
    // bf16: instruction i of a wave brings rows RPI (8 i + wave) .. of the tile, as a buffer that ends behind the last of them that
    // somebody sees: the lanes behind it, and all lanes where the page is not there, write zeros.  A page number is asked
    // for one tile before its rows are.
    const unsigned page_bytes = (unsigned)p.Hkv << p.ps_log << (HD == 128 ? 8 : 7);
    const size_t head_bytes = ((size_t)g << p.ps_log) * (HD * 2);
    const char *k_head = (const char *)p.k + head_bytes, *v_head = (const char *)p.v + head_bytes;
    unsigned k_lane, v_lane;                         // the same for every i: rows 8 RPI apart have the same swizzle
    {
        const int r = RPI * wave, lr = lane / (64 / RPI), slot = lane & (64 / RPI - 1);
        k_lane = k_off<HD>(r + lr, slot) - r * HD * 2;
        v_lane = v_off<HD>(r + lr, slot) - r * HD * 2;
    }
    int ids[LPW];
    auto ask = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LPW; ++i) ids[i] = load_const(pages, (unsigned)min(j * kTileKeys + RPI * (8 * i + wave), len - 1) >> p.ps_log);
    };
    auto issue = [&](int j, unsigned char *st) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = RPI * (8 * i + wave), key = j * kTileKeys + r;
            const bool there = (unsigned)ids[i] < (unsigned)p.n_pages;
            const size_t off = (size_t)(there ? (unsigned)ids[i] : 0u) * page_bytes + (unsigned)((key & ps_mask) * (HD * 2));
            const int bytes = __builtin_amdgcn_readfirstlane(there ? max(min(c1 - key, RPI), 0) * (HD * 2) : 0);
            auto kb = __builtin_amdgcn_make_buffer_rsrc((void *)(k_head + off), 0, bytes, 0x00020000);
            auto vb = __builtin_amdgcn_make_buffer_rsrc((void *)(v_head + off), 0, bytes, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kb, (lptr_t)(st + r * HD * 2), 16, k_lane, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vb, (lptr_t)(st + VRING + r * HD * 2), 16, v_lane, 0, 0, 0);
        }
    };
    // E4M3: a wave brings rows 8 wave .. + 7, eight threads a row, HD / 8 codes each; the same buffers, into registers
    constexpr int CW = HD / 32;                      // registers of codes
    unsigned kc[CW], vc[CW];
    float k_sc = 1.f, v_sc = 1.f;
    const int cr = tid >> 3, cp = tid & 7;
    auto ask_codes = [&](int j) __attribute__((always_inline)) {
        ids[0] = load_const(pages, (unsigned)min(j * kTileKeys + 8 * wave, len - 1) >> p.ps_log);
    };
    auto fetch = [&](int j) __attribute__((always_inline)) {     // the rows of tile j, whose page was asked for
        const int key = j * kTileKeys + 8 * wave;
        const bool there = (unsigned)ids[0] < (unsigned)p.n_pages;
        const unsigned id = there ? (unsigned)ids[0] : 0u;
        const size_t off = (size_t)id * (page_bytes / 2) + (unsigned)((key & ps_mask) * HD);
        const int bytes = __builtin_amdgcn_readfirstlane(there ? max(min(c1 - key, 8), 0) * HD : 0);
        k_sc = load_const(p.k_scales, (size_t)id * p.Hkv + g);
        v_sc = load_const(p.v_scales, (size_t)id * p.Hkv + g);
        auto kb = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)p.k + head_bytes / 2 + off), 0, bytes, 0x00020000);
        auto vb = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)p.v + head_bytes / 2 + off), 0, bytes, 0x00020000);
        const int at_lane = (cr & 7) * HD + cp * (HD / 8);
        if constexpr (HD == 128) {
            const u32x4 kw = __builtin_amdgcn_raw_buffer_load_b128(kb, at_lane, 0, 0), vw = __builtin_amdgcn_raw_buffer_load_b128(vb, at_lane, 0, 0);
#pragma unroll
            for (int i = 0; i < CW; ++i) { kc[i] = kw[i]; vc[i] = vw[i]; }
        } else {
            const u32x2 kw = __builtin_amdgcn_raw_buffer_load_b64(kb, at_lane, 0, 0), vw = __builtin_amdgcn_raw_buffer_load_b64(vb, at_lane, 0, 0);
#pragma unroll
            for (int i = 0; i < CW; ++i) { kc[i] = kw[i]; vc[i] = vw[i]; }
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
            *(u32x4 *)(st + VRING + v_off<HD>(cr, cp * (CW / 2) + i)) = widen4(vc[2 * i], vc[2 * i + 1], v_sc);
        }
    };

    // ---- a tile in two phases ----
    // M(j): the products, V^T P^T of tile j - 1 and K Q^T of tile j;  S(j): the softmax of tile j.  The two waves of a SIMD (wave
    // and wave + 4) are one phase apart, so that one's matrix instructions run under the other's exponentials; a barrier ends
    // every phase: the early waves' M(j) is phase 2 j, the late ones' phase 2 j + 1.  In S(j) a wave asks for its part of tile
    // j + 2, in the stage of tile j - 2, whose values the late waves read for the last time in phase 2 j - 1.  Tile j has
    // to be there in phase 2 j: before the barrier ahead of it an early wave (at the end of S(j - 1)) waits for all but the
    // tile asked for last, a late one (at the end of M(j - 1)) for all.
    f32x16 s[2];
    bf16x8 pf[4];
    u32x4 vf[NDB][4];
    const bool late = wave >= 4;
    auto phase_end = [&](auto M) __attribute__((always_inline)) {
        if (KIND != PAGED_BF16) {
            if (decltype(M)::value) PD_TILE_LGKM0();     // codes written in S(j) are needed after the wave's M(j + 1)
        } else if (!decltype(M)::value) {
            PD_TILE_VMCNT(2 * LPW);
        } else if (late) {
            PD_TILE_VMCNT(0);
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto ahead = [&](int j, auto stage) __attribute__((always_inline)) {      // in S(j); stage(i): the LDS of tile i
        if (KIND == PAGED_BF16) {
            issue(min(j + 2, t_hi - 1), stage(j + 2));
            ask(min(j + 3, t_hi - 1));
        } else {
            commit(stage(j + 2));
            fetch(min(j + 3, t_hi - 1));
            ask_codes(min(j + 4, t_hi - 1));
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // Value columns: operand (db, ks) is channels 32 db .. + 31 of the keys whose exponentials are registers 8 (ks % 2) .. + 7 of
    // s[ks / 2]: keys 16 ks + 4 h + {0 .. 3, 8 .. 11}, four rows a read.
    auto load_v = [&](const unsigned char *st, int ks) __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
            const int r = 16 * ks + 4 * h + ((lane & 15) >> 2), piece = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((trptr_t)(st + VRING + v_off<HD>(r, piece) + 8 * (lane & 1))));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((trptr_t)(st + VRING + v_off<HD>(r + 8, piece) + 8 * (lane & 1))));
            vf[db][ks] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    };
    bf16x8 kf[2][NK];
    auto load_k = [&](const unsigned char *st, int half) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int k = half * (NK / 2); k < (half + 1) * (NK / 2); ++k) kf[kb][k] = *(const bf16x8 *)(st + k_off<HD>(32 * kb + n, 2 * k + h));
    };
    auto mul_k = [&](int half) __attribute__((always_inline)) {
#pragma unroll
        for (int k = half * (NK / 2); k < (half + 1) * (NK / 2); ++k)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kb][k], qf[k], s[kb], 0, 0, 0);
    };
    auto mul_v = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[db][ks]), pf[ks], o[db], 0, 0, 0);
    };
    auto clear_s = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
    };
    // p = 2^(s scale log2 e - m); the first half of the values is requested behind it
    auto softmax = [&](int j, const unsigned char *st) __attribute__((always_inline)) {
        const int k0 = j * kTileKeys;
        if (k0 + kTileKeys > w_min) {                // some row of the wave does not see all of the tile
            int seen = limit - k0 - 4 * h;
            asm volatile("" : "+v"(seen));           // keeps the branch
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * kb + 8 * (r >> 2) + (r & 3) >= seen) s[kb][r] = -INFINITY;
        }
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
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int r = 8 * (ks & 1);
            u32x4 w = {pack2bf(s[ks >> 1][r], s[ks >> 1][r + 1]), pack2bf(s[ks >> 1][r + 2], s[ks >> 1][r + 3]),
                       pack2bf(s[ks >> 1][r + 4], s[ks >> 1][r + 5]), pack2bf(s[ks >> 1][r + 6], s[ks >> 1][r + 7])};
            asm volatile("" : "+v"(w));              // formed in this phase, not where it is used
            pf[ks] = __builtin_bit_cast(bf16x8, w);
        }
        asm volatile("" : "+v"(l_run));
        __builtin_amdgcn_sched_barrier(0);
        load_v(st, 0);
        load_v(st, 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    // the rest of V^T P^T out of st and, unless this was the last tile, K Q^T out of st_k: operands are requested a quarter ahead
    auto products = [&](const unsigned char *st, const unsigned char *st_k, auto NEXT) __attribute__((always_inline)) {
        load_v(st, 2);
        load_v(st, 3);
        __builtin_amdgcn_sched_barrier(0);
        mul_v(0);
        mul_v(1);
        __builtin_amdgcn_sched_barrier(0);
        if (decltype(NEXT)::value) load_k(st_k, 0);
        __builtin_amdgcn_sched_barrier(0);
        mul_v(2);
        mul_v(3);
        __builtin_amdgcn_sched_barrier(0);
        if (decltype(NEXT)::value) {
            load_k(st_k, 1);
            clear_s();
            __builtin_amdgcn_sched_barrier(0);
            mul_k(0);
            mul_k(1);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // A weight of 0 times a value that is infinite or NaN is NaN: such a value would reach rows that do not see it.  The results
    // tell: where one is not finite, the tiles are gone through again with the values in question taken out in LDS, and these
    // are then added to the rows that see them.
    bool clean = false;
    auto clean_v = [&](unsigned char *st) __attribute__((always_inline)) {    // by the early half of the waves in M(j), before any S(j)
        if (!late)
#pragma unroll 1
            for (int i = tid; i < TILE / 16; i += 256) {
                u32x4 w = *(u32x4 *)(st + VRING + i * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = ((w[e] & 0x7f80u) == 0x7f80u ? 0u : w[e] & 0xffffu) | ((w[e] & 0x7f800000u) == 0x7f800000u ? 0u : w[e] & 0xffff0000u);
                *(u32x4 *)(st + VRING + i * 16) = w;
            }
        PD_TILE_LGKM0();
    };
    while (t_lo < t_hi) {
        asm volatile("" : "+v"(n), "+v"(h));         // addresses are formed here, not kept from before a loop that rarely runs twice
        auto stage_at = [&](int j) __attribute__((always_inline)) { return smem + (j - t_lo) % NST * TILE; };
        if (KIND == PAGED_BF16) {
            ask(t_lo);
            issue(t_lo, smem);
            ask(min(t_lo + 1, t_hi - 1));
            issue(min(t_lo + 1, t_hi - 1), smem + TILE);
            ask(min(t_lo + 2, t_hi - 1));
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                ask_codes(min(t_lo + i, t_hi - 1));
                fetch(min(t_lo + i, t_hi - 1));
                if (i < 2) commit(smem + i * TILE);
            }
            ask_codes(min(t_lo + 3, t_hi - 1));
        }
        __builtin_amdgcn_sched_barrier(0);
        if (tid == 0) again = 0;
        if (KIND == PAGED_BF16) PD_TILE_VMCNT(2 * LPW);
        PD_TILE_LGKM0();
        __builtin_amdgcn_s_barrier();
        if (late) phase_end(std::false_type{});
        // M(t_lo)
        if (clean) clean_v(smem);
        load_k(smem, 0);
        load_k(smem, 1);
        clear_s();
        mul_k(0);
        mul_k(1);
        __builtin_amdgcn_sched_barrier(0);
        phase_end(std::true_type{});
        // S(j), M(j + 1); the stages are constants, so that LDS addresses are registers plus immediates
        int j = t_lo;
        auto step = [&](auto STG) __attribute__((always_inline)) {
            auto stage = [&](int i) __attribute__((always_inline)) { return smem + (decltype(STG)::value + i - j) % NST * TILE; };
            ahead(j, stage);
            softmax(j, stage(j));
            phase_end(std::false_type{});
            if (clean) clean_v(stage(j + 1));
            products(stage(j), stage(j + 1), std::true_type{});
            phase_end(std::true_type{});
            return ++j < t_hi - 1;
        };
        if (j < t_hi - 1)
            while (step(std::integral_constant<int, 0>{}) && step(std::integral_constant<int, 1>{}) && step(std::integral_constant<int, 2>{}) &&
                   step(std::integral_constant<int, 3>{})) {
            }
        softmax(j, stage_at(j));
        if (!late) phase_end(std::false_type{});
        products(stage_at(j), nullptr, std::false_type{});
        // (infinity or NaN) * 0 is NaN, and no sum removes it
        float zero = 0.f;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) zero = fmaf(o[db][r], 0.f, zero);
        if (__any(ok && zero != 0.f) && lane == 0) again = 1;
        // the repeated requests of the last tile: none may land in another round's tiles or outlive the workgroup's LDS
        if (KIND == PAGED_BF16) PD_TILE_VMCNT(0);
        __syncthreads();
        if (clean || !again) break;
        __syncthreads();
        clean = true;
        m_run = kNoScore;
        l_run = 0.f;
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    }
    if (clean)
#pragma unroll 1
        for (int key = c0; key < c1; ++key) {
            const int id = load_const(pages, key >> p.ps_log);
            if (id < 0 || id >= p.n_pages) continue;
            const size_t unit = (size_t)id * p.Hkv + g, at_v = ((unit << p.ps_log) + (key & ps_mask)) * HD;
            const float v_scale = KIND == PAGED_E4M3 ? load_const(p.v_scales, unit) : 1.f;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const size_t i = at_v + 32 * db + 8 * (r >> 2) + 4 * h + (r & 3);
                    const float x = KIND == PAGED_E4M3 ? e4m3_decode(((const uint8_t *)p.v)[i]) * v_scale : bfbits2f(((const uint16_t *)p.v)[i]);
                    if (!(fabsf(x) < INFINITY) && key < limit) o[db][r] += x;
                }
        }

    // ---- a lane holds row `row`, channels 32 db + 8 (r / 4) + 4 h + r % 4 ----
    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    if (nc_u == 1) {
        // halves of the wave trade registers, so that a lane stores eight consecutive channels
        const float inv = limit <= 0 ? 0.f : 1.f / l_tot;
        uint16_t *op = (uint16_t *)a.out + ((size_t)(start + tok) * a.Hq + g * a.G + row - tok * a.G) * HD + 8 * h;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; q4 += 2) {
                unsigned w[2][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) w[i][e] = pack2bf(o[db][4 * (q4 + i) + 2 * e] * inv, o[db][4 * (q4 + i) + 2 * e + 1] * inv);
                const auto lo = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), hi = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                if (ok) *(u32x4 *)(op + 32 * db + 8 * q4) = u32x4{lo[0], hi[0], lo[1], hi[1]};
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
    constexpr int lds = 4 * 2 * kTileKeys * HD * 2;
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
