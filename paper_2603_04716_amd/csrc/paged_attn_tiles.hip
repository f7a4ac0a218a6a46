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
// 16 - in a ring of four tiles.  E4M3 tiles are loaded into registers a tile earlier, widened (a code times its page's scale is exact
// in bf16) and written to the same ring: widened by the workgroup once, not by every wave.
//
// A workgroup fills a CU (128 KB of ring, 256 registers a lane) and stays: it takes an equal part of all units' tiles and goes
// from unit to unit with the ring full, which saves the division of the call, the first loads' latency and an empty pipe, some
// 13 us, for each unit but its first.
//
// Measured, 32 heads on 8 of 128 channels: calls of four prompts of 2048 tokens in 163 us, 840 TFLOP/s of what the rows see (large library
// products reach 1230 to 1500 here, by their data); 512 tokens behind 32000 in 276 us, 980 TFLOP/s.  A tile takes some 4000 clocks, of which the
// matrix pipe is busy for 2048: M, the two products, takes 1750 and S, the softmax, 1600 beside it, with 130 for a barrier each.
// From unit to unit takes 4.5 us, from the launch to the first products 12 us.  Four waves of 64 rows, which read every operand half as
// often but leave a SIMD one wave, took 5300 clocks a tile.
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
constexpr float kNoScore = -0x1.fffffep127f;      // running maximum before any score: the least finite number, so that differences are defined
constexpr float kLazyRaise = 8.0f;               // the maximum is raised when a score exceeds it by 2^8: sums stay exact in fp32

// Byte offset of the 16-byte piece c of row r in a K or V tile.  K is read 32 rows at one piece index, V four rows at 64
// bytes' worth of neighbouring pieces; the exclusive-ors spread both over all banks.
template <int HD>
__device__ __forceinline__ int k_off(int r, int c) { return r * HD * 2 + (HD == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7)) * 16; }
template <int HD>
__device__ __forceinline__ int v_off(int r, int c) { return r * HD * 2 + (HD == 128 ? c ^ ((r & 3) << 2) : c ^ (((r >> 1) & 1) << 2)) * 16; }

// x[i] of lane n + 32 h: piece 2 i + h (16 bytes) of row n.  Afterwards x[4 k + i] of a lane: piece 8 k + rows_piece() of row 8 i + lane % 8,
// so that a store or load covers eight rows' whole cache lines: 32 rows at 32 bytes each took four times as long.  Its own inverse.
__device__ __forceinline__ int rows_piece(int lane) { return ((lane & 8) >> 1) + ((lane & 16) >> 3) + (lane >> 5); }
template <int N>
__device__ __forceinline__ void rows_swap16(u32x4 (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto s = __builtin_amdgcn_permlane16_swap(x[i][e], x[i + 1][e], false, false);
            x[i][e] = s[0];
            x[i + 1][e] = s[1];
        }
}
template <int N>
__device__ __forceinline__ void rows_swap8(u32x4 (&x)[N])      // lanes 8 .. 15 of each 16 of x[i] with lanes 0 .. 7 of x[i + 2]
{
#pragma unroll
    for (int i = 0; i < N; i += i & 1 ? 3 : 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int lo = x[i][e], hi = x[i + 2][e];
            x[i][e] = __builtin_amdgcn_update_dpp(lo, hi, 0x128, 0xf, 0xc, false);       // row_ror:8
            x[i + 2][e] = __builtin_amdgcn_update_dpp(hi, lo, 0x128, 0xf, 0x3, false);
        }
}

template <int KIND, int HD>
__global__ __launch_bounds__(512, 1) void paged_tiles_kernel(PagedAttnArgs a)
{
    // stages of the ring: K tiles, then V tiles, so that all stages of either lie within an LDS instruction's 64 KB immediate
    constexpr int NST = 4, TILE = kTileKeys * HD * 2, VRING = NST * TILE;
    constexpr int NK = HD / 16, NDB = HD / 32;       // k-steps of a score, 32-channel blocks of the output
    constexpr int LPW = TILE / 1024 / 8;             // bf16: load instructions per wave for each of K and V
    constexpr int RPI = 1024 / (HD * 2);             // ... rows of one
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ PagedTilesShared<512> sh;
    __shared__ unsigned bad;                         // listed units with results that are not finite
    const PagedView &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63;
    int n = lane & 31, h = lane >> 5;
    int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedTilesPart part = paged_tiles_part<kTileRows, kTileKeys>(a, sh);
    if (part.from >= part.to) {
        if (tid == 0 && a.parts.desc) a.parts.desc[(size_t)part.w * 8 + 1] = 0;      // no unit of its own to be merged
        return;
    }
    const float sl2e = a.scale * 1.4426950408889634f;
    int n_listed = 0;
    auto field = [&](int i, int at) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(((const int *)&sh.item[wave][i])[at]); };
#define PD_ITEM(i, f) field(i, offsetof(PagedTilesItem, f) / 4)

    // the lane, for addresses that are formed where they are used: registers for them are not to be had
    auto lane_now = [&]() __attribute__((always_inline)) {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    };
    // what is used at the ends of units alone is read there: scalar registers are short as well
    auto rare = [&]() __attribute__((always_inline)) {
        const PagedAttnArgs __attribute__((address_space(4))) *args = (const PagedAttnArgs __attribute__((address_space(4))) *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(args));
        return args;
    };

    // ---- the wave's rows of a unit ----
    const int w0 = wave * 32;
    int item, j, t_hi, w_min, limit;                 // of the products: listed unit, its tile, the end of them; the wave's first row sees keys
    bf16x8 qf[NK];                                   // 0 .. w_min - 1, the lane's row 0 .. limit - 1
    f32x16 o[NDB];
    float m_run, l_run;
    bool large;                                      // some row's maximum is beyond kExactScores
    // A unit's row w is (token, head) row r0 + w of its sequence: token tok + (rest + w) / G, where G tok + rest = r0.  The quotient by
    // way of fp32 is exact for dividends up to 2^21.
    struct Unit {
        int r0, rows, tok, rest, start, head, G;
        float per_G;
        __device__ __forceinline__ int token(int w) const { return (int)(((float)(rest + w) + 0.5f) * per_G); }
    };
    auto unit_of = [&](int i, int G) __attribute__((always_inline)) {
        Unit u = {PD_ITEM(i, r0), PD_ITEM(i, rows), PD_ITEM(i, tok), 0, PD_ITEM(i, start), PD_ITEM(i, g) * G, G, 1.f / (float)G};
        u.rest = u.r0 - u.tok * G;
        return u;
    };
    // four rows of the wave in the layout of whole cache lines: 8 i + lane % 8 for x[4 k + {0, 2, 1, 3}[i]]
    auto row_of = [&](int i) __attribute__((always_inline)) { return w0 + 8 * (i >> 1 | (i & 1) << 1) + (lane_now() & 7); };
    auto load_q = [&](int i) __attribute__((always_inline)) {
        const auto args = rare();
        const Unit u = unit_of(i, args->G);
        const int64_t stride = args->q_stride;
        const uint16_t *q = (const uint16_t *)args->q + (u.start + u.tok) * stride + (u.head + u.rest) * HD;
        const int piece = 8 * rows_piece(lane_now());
        u32x4 x[NK];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = min(row_of(i), u.rows - 1 - u.r0), tok = u.token(w);    // (rows behind the last are not stored)
            const uint16_t *at = q + tok * stride + ((w - tok * u.G) * HD + piece);
#pragma unroll
            for (int k = 0; k < NK / 4; ++k) x[4 * k + i] = *(const u32x4 *)(at + 64 * k);
        }
#pragma unroll
        for (int k = 0; k < NK; ++k) qf[k] = __builtin_bit_cast(bf16x8, x[k]);
    };
    auto turn_q = [&]() __attribute__((always_inline)) {
        u32x4 x[NK];
#pragma unroll
        for (int k = 0; k < NK; ++k) x[k] = __builtin_bit_cast(u32x4, qf[k]);
        rows_swap8(x);
        rows_swap16(x);
#pragma unroll
        for (int k = 0; k < NK; ++k) qf[k] = __builtin_bit_cast(bf16x8, x[k]);
    };
    // what the products need of a unit
    struct Bounds { int t_lo, t_hi, w_min, limit; };
    auto bounds_of = [&](int i) __attribute__((always_inline)) {
        const Unit u = unit_of(i, rare()->G);
        const int first = PD_ITEM(i, before) + u.tok + 1;
        return Bounds{PD_ITEM(i, t_lo), PD_ITEM(i, t_hi), first + __builtin_amdgcn_readfirstlane(u.token(w0)), w0 + n < u.rows - u.r0 ? first + u.token(w0 + n) : 0};
    };
    auto begin = [&](int i, const Bounds &x) __attribute__((always_inline)) {
        item = i;
        j = x.t_lo;
        t_hi = x.t_hi;
        w_min = x.w_min;
        limit = x.limit;
        m_run = kNoScore;
        l_run = 0.f;
        large = false;
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    };

    // ---- tile loaders ----
    // bf16: instruction i of a wave brings rows RPI (8 i + wave) .. of the tile, as a buffer that ends behind the last of them that
    // somebody sees: the lanes behind it, and all lanes where the page is not there, write zeros.  A page number is asked
    // for one tile before its rows are.  Page numbers and rows run ahead of the products, over the ends of units, each at a
    // place of its own.
    const void *k_pages = p.k, *v_pages = p.v;
    const float *k_scales = p.k_scales, *v_scales = p.v_scales;
    int n_pages = p.n_pages, ps_log = p.ps_log, Hkv = p.Hkv;
    unsigned page_bytes = (unsigned)Hkv << ps_log << (HD == 128 ? 8 : 7);
    struct Place { int item, j, t_hi; } pg, at;      // next page numbers, next rows
    const int32_t *pages;
    int last_key, seen;                              // of pg's unit: positions - 1; of at's: keys that it sees, kv head
    unsigned head;
    auto page_of = [&](int i) __attribute__((always_inline)) {
        pg = Place{i, PD_ITEM(i, t_lo), PD_ITEM(i, t_hi)};
        last_key = PD_ITEM(i, len) - 1;
        // (without positions: any number will do, no key is seen)
        const auto r = rare();
        pages = last_key < 0 ? r->p.lens : r->p.table + (size_t)PD_ITEM(i, seq) * r->p.width;
        last_key = max(last_key, 0);
    };
    auto rows_of = [&](int i) __attribute__((always_inline)) {
        at = Place{i, PD_ITEM(i, t_lo), PD_ITEM(i, t_hi)};
        seen = PD_ITEM(i, seen);
        head = PD_ITEM(i, g);
    };
    // onto the next unit, where the place is behind its own; at the end of the list it goes on, over keys that nobody sees
    auto settle = [&](Place &x, auto next) __attribute__((always_inline)) {
        if (x.j < x.t_hi) return;
        if (x.item + 1 < n_listed) next(x.item + 1);
        else x.t_hi = 0x7fffffff;
    };
    auto settle_all = [&]() __attribute__((always_inline)) {
        settle(at, rows_of);
        settle(pg, page_of);
    };
    unsigned k_lane, v_lane;                         // the same for every i: rows 8 RPI apart have the same swizzle
    {
        const int r = RPI * wave, lr = lane / (64 / RPI), slot = lane & (64 / RPI - 1);
        k_lane = k_off<HD>(r + lr, slot) - r * HD * 2;
        v_lane = v_off<HD>(r + lr, slot) - r * HD * 2;
    }
    int ids[LPW];
    auto ask = [&](int (&ids)[LPW]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LPW; ++i) ids[i] = load_const(pages, (unsigned)min(pg.j * kTileKeys + RPI * (8 * i + wave), last_key) >> ps_log);
        ++pg.j;
    };
    auto issue = [&](unsigned char *st, int i, const int (&ids)[LPW]) __attribute__((always_inline)) {
        const int r = RPI * (8 * i + wave), key = at.j * kTileKeys + r;
        const bool there = (unsigned)ids[i] < (unsigned)n_pages;
        const size_t off = (size_t)(there ? (unsigned)ids[i] : 0u) * page_bytes + ((head << ps_log) + (unsigned)(key & ((1 << ps_log) - 1))) * (HD * 2);
        const int bytes = __builtin_amdgcn_readfirstlane(there ? max(min(seen - key, RPI), 0) * (HD * 2) : 0);
        auto kb = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)k_pages + off), 0, bytes, 0x00020000);
        auto vb = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)v_pages + off), 0, bytes, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kb, (lptr_t)(st + r * HD * 2), 16, k_lane, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vb, (lptr_t)(st + VRING + r * HD * 2), 16, v_lane, 0, 0, 0);
        if (i == LPW - 1) ++at.j;
    };
    // E4M3: a wave brings rows 8 wave .. + 7, eight threads a row, HD / 8 codes each; the same buffers, into registers
    constexpr int CW = HD / 32;                      // registers of codes
    unsigned kc[CW], vc[CW];
    float k_sc = 1.f, v_sc = 1.f;
    auto ask_codes = [&](int &id) __attribute__((always_inline)) {
        id = load_const(pages, (unsigned)min(pg.j * kTileKeys + 8 * wave, last_key) >> ps_log);
        ++pg.j;
    };
    auto fetch = [&](int asked) __attribute__((always_inline)) {     // the rows of the tile whose page was asked for
        const int key = at.j * kTileKeys + 8 * wave;
        const bool there = (unsigned)asked < (unsigned)n_pages;
        const unsigned id = there ? (unsigned)asked : 0u;
        const size_t off = (size_t)id * (page_bytes / 2) + ((head << ps_log) + (unsigned)(key & ((1 << ps_log) - 1))) * HD;
        const int bytes = __builtin_amdgcn_readfirstlane(there ? max(min(seen - key, 8), 0) * HD : 0);
        // (a page that is not there has no scale, and any number does for its zeros, but not an infinity or NaN, which page 0 may have:
        // the call's own scale is one)
        const float __attribute__((address_space(4))) *number = &rare()->scale;
        const size_t scale_at = (size_t)id * Hkv + head;
        k_sc = *(there ? (const float __attribute__((address_space(4))) *)(uintptr_t)k_scales + scale_at : number);
        v_sc = *(there ? (const float __attribute__((address_space(4))) *)(uintptr_t)v_scales + scale_at : number);
        auto kb = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)k_pages + off), 0, bytes, 0x00020000);
        auto vb = __builtin_amdgcn_make_buffer_rsrc((void *)((const char *)v_pages + off), 0, bytes, 0x00020000);
        const int at_lane = lane_now() * (HD / 8);
        if constexpr (HD == 128) {
            const u32x4 kw = __builtin_amdgcn_raw_buffer_load_b128(kb, at_lane, 0, 0), vw = __builtin_amdgcn_raw_buffer_load_b128(vb, at_lane, 0, 0);
#pragma unroll
            for (int i = 0; i < CW; ++i) { kc[i] = kw[i]; vc[i] = vw[i]; }
        } else {
            const u32x2 kw = __builtin_amdgcn_raw_buffer_load_b64(kb, at_lane, 0, 0), vw = __builtin_amdgcn_raw_buffer_load_b64(vb, at_lane, 0, 0);
#pragma unroll
            for (int i = 0; i < CW; ++i) { kc[i] = kw[i]; vc[i] = vw[i]; }
        }
        ++at.j;
    };
    auto widen4 = [](unsigned lo, unsigned hi, float s) {
        return u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true))};
    };
    auto commit = [&](unsigned char *st, int i) __attribute__((always_inline)) {
        const int l = lane_now(), r = 8 * wave + (l >> 3);
        *(u32x4 *)(st + k_off<HD>(r, (l & 7) * (CW / 2) + i)) = widen4(kc[2 * i], kc[2 * i + 1], k_sc);
        *(u32x4 *)(st + VRING + v_off<HD>(r, (l & 7) * (CW / 2) + i)) = widen4(vc[2 * i], vc[2 * i + 1], v_sc);
    };

    // ---- a tile in two phases ----
    // M(j): the products, V^T P^T of tile j - 1 and K Q^T of tile j;  S(j): the softmax of tile j.  The two waves of a SIMD (wave
    // and wave + 4) are one phase apart, so that one's matrix instructions run under the other's exponentials; a barrier ends
    // every phase: the early waves' M(j) is phase 2 j, the late ones' phase 2 j + 1.  What is asked for ahead is M's, between the products: in
    // M(j) a wave asks for its part of tile j + 2, in the stage of tile j - 2, whose values the late waves read for the last time in
    // phase 2 j - 1.  Tile j has to be there in phase 2 j: before the barrier ahead of it an early wave (at the end of S(j - 1)) and a
    // late one (at the end of M(j - 1)) waits for all but the tile asked for last.
    f32x16 s[2];
    bf16x8 pf[4];
    u32x4 vf[NDB][4];
    const bool late = wave >= 4;
    auto phase_end = [&](auto M, bool wait = true) __attribute__((always_inline)) {
        if (KIND != PAGED_BF16) {
            if (decltype(M)::value) PD_TILE_LGKM0();     // codes written in M(j) are needed in M(j + 2)
        } else if (!decltype(M)::value || (late && wait)) {
            PD_TILE_VMCNT(2 * LPW);
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (decltype(M)::value) __builtin_amdgcn_s_setprio(0);
        else __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
    };
    int ring;                                        // offset of the stage of the products' tile
    auto stage = [&](int i) __attribute__((always_inline)) { return smem + ((ring + i * TILE) & (NST * TILE - 1)); };
    auto ahead = [&](unsigned char *st, int quarter) __attribute__((always_inline)) {      // in M(j): tile j + 2, into st
        if (KIND == PAGED_BF16) {
            if (quarter < LPW) issue(st, quarter, ids);
            if (quarter == 3) ask(ids);
        } else {
            if (quarter < CW / 2) commit(st, quarter);
            if (quarter == 3) {
                fetch(ids[0]);
                ask_codes(ids[0]);
            }
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
            // (by the sign of a difference: 32 conditions at once would take the scalar registers of the whole loop)
            const int seen = limit - k0 - 4 * (lane_now() >> 5);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    int out = (seen - 1 - (32 * kb + 8 * (r >> 2) + (r & 3))) >> 31;
                    asm volatile("" : "+v"(out));
                    s[kb][r] = __builtin_bit_cast(float, (out & (int)0xff800000) | (~out & __builtin_bit_cast(int, (float)s[kb][r])));
                }
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
            large |= __any(fabsf(m_cand) > kExactScores && m_cand != kNoScore);
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < NDB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
        }
        float sum = 0.f, factor = sl2e;
        if (large) {
            factor = 1.f;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] *= sl2e;
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = pexp2(fmaf(s[kb][r], factor, -m_run));
                sum += s[kb][r];
            }
        l_run += sum;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int r = 8 * (ks & 1);              // (rounded to bf16 for the matrix pipe: 2^-8 of each weight at most, see Step16::operand)
            u32x4 w = {pack2bf(s[ks >> 1][r], s[ks >> 1][r + 1]), pack2bf(s[ks >> 1][r + 2], s[ks >> 1][r + 3]),
                       pack2bf(s[ks >> 1][r + 4], s[ks >> 1][r + 5]), pack2bf(s[ks >> 1][r + 6], s[ks >> 1][r + 7])};
            asm volatile("" : "+v"(w));              // formed in this phase, not where it is used
            pf[ks] = __builtin_bit_cast(bf16x8, w);
        }
        asm volatile("" : "+v"(l_run));
        __builtin_amdgcn_sched_barrier(0);
        load_v(st, 0);
        load_v(st, 1);
        load_v(st, 2);
        load_v(st, 3);
        __builtin_amdgcn_sched_barrier(0);
    };
    // V^T P^T out of st and, unless this was the unit's last tile, K Q^T out of st_k, requested ahead; between the products what
    // is asked for into st_next
    auto products = [&](unsigned char *st_k, unsigned char *st_next, auto NEXT) __attribute__((always_inline)) {
        mul_v(0);
        __builtin_amdgcn_sched_barrier(0);
        ahead(st_next, 0);
        mul_v(1);
        __builtin_amdgcn_sched_barrier(0);
        if (decltype(NEXT)::value) load_k(st_k, 0);
        __builtin_amdgcn_sched_barrier(0);
        ahead(st_next, 1);
        mul_v(2);
        __builtin_amdgcn_sched_barrier(0);
        ahead(st_next, 2);
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
        ahead(st_next, 3);                           // (scalar loads under way would have the products wait for all of their operands)
    };
    // A weight of 0 times a value that is infinite or NaN is NaN: such a value would reach rows that do not see it.  The results
    // tell: where one is not finite, the tiles are gone through again with the values in question taken out in LDS, and these
    // are then looked for in the pages and added to the rows that see them.
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
    // ---- a unit ends: a lane holds one row's channels 32 db + 8 (r / 4) + 4 h + r % 4 ----
    struct Ending {
        Unit u;
        int slot, Hq;
        uint16_t *out;
        float *ml, *o;
    };
    auto ending_of = [&](int i) __attribute__((always_inline)) {
        const auto args = rare();
        Ending e = {unit_of(i, args->G), PD_ITEM(i, slot), args->Hq, (uint16_t *)args->out, args->parts.ml, args->parts.o};
        e.out += ((size_t)(e.u.start + e.u.tok) * e.Hq + e.u.head + e.u.rest) * HD;
        return e;
    };
    auto finish = [&](const Ending &e) __attribute__((always_inline)) {
        const Unit &u = e.u;
        const bool ok = w0 + n < u.rows - u.r0;
        if (!clean) {
            float zero = 0.f;                        // (infinity or NaN) * 0 is NaN, and no sum removes it
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) zero = fmaf(o[db][r], 0.f, zero);
            if (__any(ok && zero != 0.f) && lane == 0) atomicOr(&bad, 1u << item);
        } else {
            const auto args = rare();
            const int g = PD_ITEM(item, g);
            const int32_t *table = args->p.table + (size_t)PD_ITEM(item, seq) * args->p.width;
            const int last = min(t_hi * kTileKeys, PD_ITEM(item, seen));
            const int32_t pages_end = args->p.n_pages, log = args->p.ps_log;
            constexpr int E = KIND == PAGED_E4M3 ? 1 : 2, STEP = 16;     // keys that share a page at every page size
            auto rows_at = [&](int id, int key) __attribute__((always_inline)) {
                return (((size_t)id * args->p.Hkv + g) << log) + (key & ((1 << log) - 1));
            };
#pragma unroll 1
            for (int tile = PD_ITEM(item, t_lo); tile < t_hi; ++tile) {
                unsigned found = 0;                  // steps of the tile with such values (or, in unused slots, numbers that look like one)
#pragma unroll
                for (int i = 0; i < kTileKeys / STEP; ++i) {
                    const int key = tile * kTileKeys + STEP * i, id = key < last ? load_const(table, key >> log) : -1;
                    if (id < 0 || id >= pages_end) continue;
                    const u32x4 *rows = (const u32x4 *)((const char *)args->p.v + rows_at(id, key) * (HD * E));
                    unsigned odd = KIND == PAGED_E4M3 && !(load_const(args->p.v_scales, (size_t)id * args->p.Hkv + g) < 0x1p120f);    // (256 * 2^120 is infinite)
#pragma unroll
                    for (int k = 0; k < STEP * HD * E / 1024; ++k) {
                        const u32x4 w = rows[64 * k + lane];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (KIND == PAGED_E4M3) odd |= ((w[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;       // a byte of 0x7f or 0xff
                            else odd |= (((w[e] & 0x7f807f80u) >> 7) + 0x00010001u) & 0x01000100u;                    // an exponent of ones
                        }
                    }
                    if (__any(odd != 0)) found |= 1u << i;
                }
                for (; found; found &= found - 1) {
                    const int first = tile * kTileKeys + STEP * (__ffs(found) - 1);
                    const int id = load_const(table, first >> log);
                    const float v_scale = KIND == PAGED_E4M3 ? load_const(args->p.v_scales, (size_t)id * args->p.Hkv + g) : 1.f;
#pragma unroll 1
                    for (int key = first; key < min(first + STEP, last); ++key) {
                        const size_t at_v = rows_at(id, key) * HD;
#pragma unroll
                        for (int db = 0; db < NDB; ++db)
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                const size_t i = at_v + 32 * db + 8 * (r >> 2) + 4 * h + (r & 3);
                                const float x = KIND == PAGED_E4M3 ? e4m3_decode(((const uint8_t *)args->p.v)[i]) * v_scale : bfbits2f(((const uint16_t *)args->p.v)[i]);
                                if (!(fabsf(x) < INFINITY) && key < limit) o[db][r] += x;
                            }
                    }
                }
            }
        }
        const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
        if (e.slot < 0) {
            // halves of the wave trade registers, so that a lane has eight consecutive channels
            const float inv = limit <= 0 ? 0.f : 1.f / l_tot;
            u32x4 x[2 * NDB];
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
                    x[2 * db + q4 / 2] = u32x4{lo[0], hi[0], lo[1], hi[1]};
                }
            rows_swap16(x);
            rows_swap8(x);
            const int piece = 8 * rows_piece(lane_now());
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int w = row_of(i), tok = u.token(w);
                uint16_t *at = e.out + ((tok * e.Hq + w - tok * u.G) * HD + piece);      // (a unit's rows are not far apart)
#pragma unroll
                for (int k = 0; k < NDB / 2; ++k)
                    if (w < u.rows - u.r0) *(u32x4 *)(at + 64 * k) = x[4 * k + i];
            }
        } else {
            const size_t to = (size_t)e.slot * kTileRows;
            if (h == 0 && ok) *(float2 *)(e.ml + (to + w0 + n) * 2) = make_float2(m_run, l_tot);
            float *op = e.o + to * HD + 4 * rows_piece(lane_now());
#pragma unroll
            for (int db = 0; db < NDB; db += NDB / 2) {
                u32x4 x[2 * NDB];
#pragma unroll
                for (int i = 0; i < 2 * NDB; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[i][c] = __builtin_bit_cast(unsigned, (float)o[db + i / 4][4 * (i & 3) + c]);
                rows_swap16(x);
                rows_swap8(x);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int w = row_of(i);
#pragma unroll
                    for (int k = 0; k < NDB / 2; ++k)
                        if (w < u.rows - u.r0) *(u32x4 *)(op + w * HD + 32 * (db + k)) = x[4 * k + i];
                }
            }
        }
    };
    auto first_scores = [&]() __attribute__((always_inline)) {       // M's second product alone
        if (clean) clean_v(stage(0));
        load_k(stage(0), 0);
        load_k(stage(0), 1);
        clear_s();
        mul_k(0);
        mul_k(1);
        __builtin_amdgcn_sched_barrier(0);
    };
    // The scalar registers' values are spilled and brought back all over a range that they live through: theirs end before and
    // behind the loop over a unit's tiles, inside of which then nothing is spilled.
    auto anew = [](auto &...x) __attribute__((always_inline)) {
        auto one = [](auto &v) __attribute__((always_inline)) {
            if constexpr (sizeof(v) == 4) v = __builtin_bit_cast(std::remove_reference_t<decltype(v)>, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
            asm volatile("" : "+s"(v));
        };
        (one(x), ...);
    };
    auto renew = [&]() __attribute__((always_inline)) {
        anew(k_pages, v_pages, n_pages, ps_log, page_bytes, wave, ring, j, t_hi);
        anew(at.item, at.j, at.t_hi, pg.item, pg.j, pg.t_hi, pages, last_key, seen, head, n_listed);
#pragma unroll
        for (int i = 0; i < (KIND == PAGED_BF16 ? LPW : 1); ++i) anew(ids[i]);
        if (KIND != PAGED_BF16) anew(k_scales, v_scales, Hkv, k_sc, v_sc);
    };
    for (int first = part.from; first < part.to;) {
        if (!clean) {
            paged_tiles_list<kTileRows, kTileKeys>(a, sh, part, first);
            n_listed = min(part.to - first, kListed);
        }
        asm volatile("" : "+v"(n), "+v"(h));         // addresses are formed here, not kept from before a loop that rarely runs twice
        page_of(0);
        rows_of(0);
        ring = 0;
        load_q(0);
        // all page numbers are asked for before the first is waited for
        if (KIND == PAGED_BF16) {
            int early[3][LPW];
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                ask(early[i]);
                settle(pg, page_of);
            }
            ask(ids);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
#pragma unroll
                for (int x = 0; x < LPW; ++x) issue(smem + i * TILE, x, early[i]);
                settle(at, rows_of);
            }
        } else {
            int early[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ask_codes(early[i]);
                settle(pg, page_of);
            }
            ask_codes(ids[0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fetch(early[i]);
#pragma unroll
                for (int x = 0; x < CW / 2; ++x)
                    if (i < 3) commit(smem + i * TILE, x);
                settle(at, rows_of);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        begin(0, bounds_of(0));
        turn_q();
        if (tid == 0) bad = 0;
        if (KIND == PAGED_BF16) PD_TILE_VMCNT(4 * LPW);
        PD_TILE_LGKM0();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (late) phase_end(std::false_type{});
        first_scores();                              // M of the first tile
        phase_end(std::true_type{});
        while (true) {
            settle_all();
            renew();
            for (int left = min(t_hi - 1 - j, min(at.t_hi - at.j, pg.t_hi - pg.j)); left > 0; --left) {       // S(j), M(j + 1)
                softmax(j, stage(0));
                phase_end(std::false_type{});
                if (clean) clean_v(stage(1));
                products(stage(1), stage(3), std::true_type{});
                phase_end(std::true_type{});
                ring = (ring + TILE) & (NST * TILE - 1);
                ++j;
            }
            renew();
            if (j < t_hi - 1) continue;
            settle_all();
            // the unit's last tile: between its two products the next unit's rows take the place of these
            const bool more = item + 1 < n_listed;
            const int next = min(item + 1, n_listed - 1);
            load_q(next);
            softmax(j, stage(0));
            const Ending e = ending_of(item);
            const Bounds x = bounds_of(next);
            if (more || !late) phase_end(std::false_type{});
            products(nullptr, stage(3), std::false_type{});
            if (KIND == PAGED_BF16 && late) PD_TILE_VMCNT(2 * LPW);        // here, not for the stores
            finish(e);
            if (!more) break;
            begin(next, x);
            turn_q();
            ring = (ring + TILE) & (NST * TILE - 1);
            first_scores();
            phase_end(std::true_type{}, false);
        }
        // requests behind the last tile: none may land in another round's tiles or outlive the workgroup's LDS
        if (KIND == PAGED_BF16) PD_TILE_VMCNT(0);
        __syncthreads();
        const unsigned redo = clean ? 0u : __builtin_amdgcn_readfirstlane(bad);
        clean = redo != 0;
        if (clean) {
            if (lane == 0)
                for (int i = 0, to = 0; i < n_listed; ++i)
                    if (redo >> i & 1) sh.item[wave][to++] = sh.item[wave][i];
            n_listed = __popc(redo);
            __syncthreads();                         // bad is read
        } else {
            first += kListed;
        }
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
