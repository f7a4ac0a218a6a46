// Appending rows to a paged key/value cache, with the rotary embedding of keys and queries on the way.
//
//   y[c] = x[c] cos - x[c + hd/2] sin,  y[c + hd/2] = x[c] sin + x[c + hd/2] cos,  angle = position * base^(-2c / hd)
//
// Nothing is used twice, so the floor is the rows read once and the pages and rotated queries written once.  The angle is
// formed in double as turns (position * base^(-2c/hd) / 2 pi) and reduced to half a turn before it becomes fp32, at three
// double-precision instructions instead of a double-precision sine: the rest is within 3e-9 rad at positions up to 2^24 and 2e-7
// rad at 2^30, and fp32 rounds it by 9e-8.  Measured, heads of 128: 24 chunks of up to 700 rows, 40 heads on 8, bf16, 57 us or 4.3 TB/s (a large copy
// reaches 4.9); four prompts of 2048, 32 heads on 8, to E4M3 pages 47 us or 4.0 TB/s; one row 3.4 us, which is a launch.
#include "paged.h"

namespace pd {

// Largest index i < n with key(i) <= x for non-decreasing keys (0 if there is none), by one wave: 64 probes, then the 64
// (n <= 4096) between the two that enclose x.
template <typename KEY>
__device__ __forceinline__ int wave_last_le(int n, int x, KEY key)
{
    const int lane = threadIdx.x & 63;
    const int stride = (n + 63) >> 6;
    int i = lane * stride;
    const int blk = max(__popcll(__ballot(i < n && key(min(i, n - 1)) <= x)) - 1, 0) * stride;
    i = blk + lane;
    return blk + max(__popcll(__ballot(lane < stride && i < n && key(min(i, n - 1)) <= x)) - 1, 0);
}

// (cos, sin) of a position's angle.  Sine and cosine of x, |x| <= pi/4, by their power series up to x^9 and x^8: the first
// terms left out are 2e-9 and 2e-8, and with fp32's roundings both are within 1e-7 (the library's functions take twice the
// instructions, and every head forms the factors again).
__device__ __forceinline__ float2 rope_turn(double turns, int pos)
{
    double t = (double)pos * turns;
    t -= rint(t);
    const float f = (float)t, q = rintf(4.f * f);
    const float x = fmaf(4.f, f, -q) * 1.57079637f, x2 = x * x;
    const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
    const float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const int i = (int)q;                            // quarter turns
    const float a = i & 1 ? s : c, b = i & 1 ? c : s;
    return make_float2((i + 1) & 2 ? -a : a, i & 2 ? -b : b);
}

__device__ __forceinline__ void load8(const uint16_t *p, float (&x)[8])
{
    const uint4 w = *(const uint4 *)p;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = bfbits2f(u[j] & 0xffffu);
        x[2 * j + 1] = bfbits2f(u[j] >> 16);
    }
}
__device__ __forceinline__ void store8(uint16_t *p, const float (&x)[8])
{
    *(uint4 *)p = make_uint4(pack2bf(x[0], x[1]), pack2bf(x[2], x[3]), pack2bf(x[4], x[5]), pack2bf(x[6], x[7]));
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8])
{
    const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    ((float4 *)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4 *)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

constexpr int kRowsPerGroup = 4;

// The rows row0 .. row0 + n - 1 (n <= kRowsPerGroup) by a workgroup of 256: their queries, and (KV) keys and values into
// pages of the rows' type.  A thread takes 8 channels and their partners half a head away, 16 bytes (bf16) each.
template <typename T, int HD, bool KV>
__device__ __forceinline__ void append_rows(const PagedAppendArgs &a, int row0, int n, float2 (*cs)[HD / 2], int (*at)[3])
{
    constexpr int HALF = HD / 2, NV = HALF / 8;      // 8-channel vectors of half a head
    const PagedView &p = a.p;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    if (wave < n) {                                  // a wave finds the sequence, position and page of one row
        const int row = row0 + wave;
        const int b = p.starts ? wave_last_le(p.n_seqs, row, [&](int i) { return load_const(p.starts, i); }) : min(row, p.n_seqs - 1);
        const int start = paged_start(p, b), rows = paged_rows(p, b, start);
        const int i = row - start, pos = paged_len(p, b) - rows + i;
        int page = -1;
        const bool held = i >= 0 && i < rows && pos >= 0;
        if (KV && held) {
            page = load_const(p.table, (size_t)b * p.width + (pos >> p.ps_log));
            if (page >= p.n_pages) page = -1;        // such a position has no page: nothing is stored for it
        }
        if (lane == 0) {
            at[wave][0] = held ? pos : -1;
            at[wave][1] = page;
        }
        if (a.rope && held)
            for (int c = lane; c < HALF; c += 64) cs[wave][c] = rope_turn(a.turns[c], pos);
    }
    __syncthreads();
    const int heads = (a.q ? a.Hq : 0) + (KV ? p.Hkv : 0), per_row = heads * NV + (KV ? p.Hkv * NV * 2 : 0);
    for (int e = tid; e < n * per_row; e += 256) {
        const int r = e / per_row, j = e - r * per_row, row = row0 + r, pos = at[r][0];
        if (pos < 0) continue;
        const int slot = pos & ((1 << p.ps_log) - 1);
        float lo[8], hi[8];
        if (j < heads * NV) {
            const int h = j / NV, c = (j & (NV - 1)) * 8;
            const bool isq = h < heads - (KV ? p.Hkv : 0);
            const int g = isq ? 0 : h - (heads - p.Hkv);
            if (!isq && at[r][1] < 0) continue;
            const T *src = isq ? (const T *)a.q + row * a.q_stride + h * HD : (const T *)a.k + row * a.k_stride + g * HD;
            load8(src + c, lo);
            load8(src + c + HALF, hi);
            if (a.rope)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 f = cs[r][c + i];
                    rope_pair(lo[i], hi[i], f.x, f.y, lo[i], hi[i]);
                }
            T *dst = isq ? (T *)a.q_out + row * a.q_out_stride + h * HD
                         : (T *)p.k + ((((size_t)at[r][1] * p.Hkv + g) << p.ps_log) + slot) * HD;
            store8(dst + c, lo);
            store8(dst + c + HALF, hi);
        } else if (at[r][1] >= 0) {
            const int g = (j - heads * NV) / (2 * NV), c = ((j - heads * NV) & (2 * NV - 1)) * 8;
            load8((const T *)a.v + row * a.v_stride + g * HD + c, lo);
            store8((T *)p.v + ((((size_t)at[r][1] * p.Hkv + g) << p.ps_log) + slot) * HD + c, lo);
        }
    }
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_append_rows_kernel(PagedAppendArgs a, int per_group)
{
    __shared__ float2 cs[kRowsPerGroup][HD / 2];
    __shared__ int at[kRowsPerGroup][3];
    const int row0 = blockIdx.x * per_group;
    append_rows<T, HD, true>(a, row0, min(per_group, a.p.n_rows - row0), cs, at);
}

// the smallest power of two s with most <= 448 s (448 = 1.75 * 2^8), at least kPagedMinScale; most finite, >= 0
__device__ __forceinline__ float scale_for(float most)
{
    const uint32_t u = __float_as_uint(most);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < 67 ? kPagedMinScale : __uint_as_float((uint32_t)e << 23);      // 67: the exponent field of 2^-60
}

__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv)
{
    uint2 r;
    r.x = e4m3_cvt2(x[0] * inv, x[1] * inv) | (e4m3_cvt2(x[2] * inv, x[3] * inv) << 16);
    r.y = e4m3_cvt2(x[4] * inv, x[5] * inv) | (e4m3_cvt2(x[6] * inv, x[7] * inv) << 16);
    return r;
}

// The codes of the slots before the call's first one, read at the page's old scale, at its new one: value * ratio with
// ratio = old / new, a power of two below 1, so that only values that become subnormal codes are rounded again.
template <int HD>
__device__ __forceinline__ void recode(uint8_t *page, int slots, float ratio, int first, int step)
{
    for (int i = first; i < slots * (HD / 16); i += step) {
        uint4 w = ((uint4 *)page)[i];
        uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[j], true);
            u[j] = e4m3_cvt2(a[0] * ratio, a[1] * ratio) | (e4m3_cvt2(b[0] * ratio, b[1] * ratio) << 16);
        }
        ((uint4 *)page)[i] = make_uint4(u[0], u[1], u[2], u[3]);
    }
}

// E4M3 pages: a workgroup owns the positions that the call brings to one (page, kv head), so that the page's scale is
// found, and its older codes are brought to it, without atomics.  The rows stay in registers between the search for the
// largest value and their encoding (NI rounds of 256 / (HD / 16) rows), so they are read once.
//
// Which page a workgroup has follows from device data.  Sequence b touches at most rows / ps + 2 pages (rounded down), so
// with first(b) = start(b) / ps + 2 b the workgroups first(b) .. first(b + 1) - 1 suffice for it, and a workgroup
// finds its sequence by a search over starts alone.  Behind them come workgroups for every few rows' queries.  `first` is the
// launch's first workgroup of the call's.
template <int HD, int NI>
__global__ __launch_bounds__(256) void paged_append_codes_kernel(PagedAppendArgs a, int page_groups, int per_group, int first)
{
    constexpr int HALF = HD / 2, TPR = HD / 16, RPR = 256 / TPR;   // threads of a row, rows of a round
    __shared__ float2 cs[kRowsPerGroup][HALF];
    __shared__ int at[kRowsPerGroup][3];
    __shared__ float red[2][4];
    const PagedView &p = a.p;
    const int tid = threadIdx.x;
    const int block = first + (int)blockIdx.x, pgs = page_groups * p.Hkv;
    if (block >= pgs) {
        const int row0 = (block - pgs) * per_group;
        append_rows<uint16_t, HD, false>(a, row0, min(per_group, p.n_rows - row0), cs, at);
        return;
    }
    const int pj = block / p.Hkv, g = block - pj * p.Hkv;
    const int ps_log = p.ps_log;
    const int b = wave_last_le(p.n_seqs, pj, [&](int i) { return (paged_start(p, i) >> ps_log) + 2 * i; });
    const int start = paged_start(p, b), rows = paged_rows(p, b, start), len = paged_len(p, b);
    const int p0 = max(len - rows, 0);
    const int t = (p0 >> ps_log) + pj - ((start >> ps_log) + 2 * b);
    const int lo = max(p0, t << ps_log), hi = min(len, (t + 1) << ps_log);
    if (rows == 0 || t < 0 || lo >= hi) return;
    const int page = load_const(p.table, (size_t)b * p.width + t);
    if (page < 0 || page >= p.n_pages) return;
    const int slot0 = lo & ((1 << ps_log) - 1), n = hi - lo;
    const int row0 = start + lo - (len - rows);
    const size_t unit = (size_t)page * p.Hkv + g;
    const float k_old = p.k_scales[unit], v_old = p.v_scales[unit];
    const int c = (tid & (TPR - 1)) * 8, tr = tid / TPR;
    float k[NI][2][8], v[NI][2][8], k_most = 0.f, v_most = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int r = i * RPR + tr;
        if (r < n) {
            const uint16_t *ks = (const uint16_t *)a.k + (row0 + r) * a.k_stride + g * HD + c;
            const uint16_t *vs = (const uint16_t *)a.v + (row0 + r) * a.v_stride + g * HD + c;
            load8(ks, k[i][0]);
            load8(ks + HALF, k[i][1]);
            load8(vs, v[i][0]);
            load8(vs + HALF, v[i][1]);
        }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int r = i * RPR + tr;
        if (r < n) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (a.rope) {
                    const float2 f = rope_turn(a.turns[c + j], lo + r);
                    rope_pair(k[i][0][j], k[i][1][j], f.x, f.y, k[i][0][j], k[i][1][j]);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {        // an infinity says nothing about the others' scale (a NaN fails every comparison)
                    if (fabsf(k[i][h][j]) < INFINITY) k_most = fmaxf(k_most, fabsf(k[i][h][j]));
                    if (fabsf(v[i][h][j]) < INFINITY) v_most = fmaxf(v_most, fabsf(v[i][h][j]));
                }
            }
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        k_most = fmaxf(k_most, __shfl_xor(k_most, off, 64));
        v_most = fmaxf(v_most, __shfl_xor(v_most, off, 64));
    }
    if ((tid & 63) == 0) {
        red[0][tid >> 6] = k_most;
        red[1][tid >> 6] = v_most;
    }
    __syncthreads();
    float k_new = scale_for(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])));
    float v_new = scale_for(fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3])));
    uint8_t *kp = (uint8_t *)p.k + ((unit << ps_log) * HD), *vp = (uint8_t *)p.v + ((unit << ps_log) * HD);
    if (slot0 > 0) {
        if (k_new > k_old) recode<HD>(kp, slot0, k_old / k_new, tid, 256); else k_new = fmaxf(k_new, k_old);
        if (v_new > v_old) recode<HD>(vp, slot0, v_old / v_new, tid, 256); else v_new = fmaxf(v_new, v_old);
    }
    if (tid == 0) {
        p.k_scales[unit] = k_new;
        p.v_scales[unit] = v_new;
    }
    const float k_inv = 1.f / k_new, v_inv = 1.f / v_new;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int r = i * RPR + tr;
        if (r < n) {
            const size_t off = (size_t)(slot0 + r) * HD + c;
            *(uint2 *)(kp + off) = codes8(k[i][0], k_inv);
            *(uint2 *)(kp + off + HALF) = codes8(k[i][1], k_inv);
            *(uint2 *)(vp + off) = codes8(v[i][0], v_inv);
            *(uint2 *)(vp + off + HALF) = codes8(v[i][1], v_inv);
        }
    }
}

// E4M3 pages, one row per sequence: HD / 16 lanes have a head of a row - a query head, or a kv head's key and value - and with it
// all that the call brings to its page, so that nothing has to be exchanged beyond those lanes.  256 sequences: 5.8 us where no scale
// grows.  Where one does, its lanes recode the page slot by slot, keys before values, and the launch takes as long as the fullest of
// such pages: 21 us with 15 slots, 64 with up to 63, 127 with 127.
template <int HD>
__global__ __launch_bounds__(256) void paged_append_one_kernel(PagedAppendArgs a)
{
    constexpr int HALF = HD / 2, TPR = HD / 16;
    const PagedView &p = a.p;
    const int hq = a.q ? a.Hq : 0, heads = hq + p.Hkv;
    const int64_t group = ((int64_t)blockIdx.x * 256 + threadIdx.x) / TPR;
    const int row = (int)(group / heads), h = (int)(group - (int64_t)row * heads), c = (threadIdx.x & (TPR - 1)) * 8;
    if (row >= p.n_seqs) return;
    const bool isq = h < hq;
    const int g = isq ? 0 : h - hq;
    float k[2][8], v[2][8];
    {
        const uint16_t *ks = isq ? (const uint16_t *)a.q + row * a.q_stride + h * HD + c : (const uint16_t *)a.k + row * a.k_stride + g * HD + c;
        load8(ks, k[0]);
        load8(ks + HALF, k[1]);
        if (!isq) {
            const uint16_t *vs = (const uint16_t *)a.v + row * a.v_stride + g * HD + c;
            load8(vs, v[0]);
            load8(vs + HALF, v[1]);
        }
    }
    const int pos = paged_len(p, row) - 1;
    if (pos < 0) return;
    if (a.rope)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 f = rope_turn(a.turns[c + j], pos);
            rope_pair(k[0][j], k[1][j], f.x, f.y, k[0][j], k[1][j]);
        }
    if (isq) {
        uint16_t *dst = (uint16_t *)a.q_out + row * a.q_out_stride + h * HD + c;
        store8(dst, k[0]);
        store8(dst + HALF, k[1]);
        return;
    }
    const int page = load_const(p.table, (size_t)row * p.width + (pos >> p.ps_log)), slot = pos & ((1 << p.ps_log) - 1);
    if (page < 0 || page >= p.n_pages) return;
    const size_t unit = (size_t)page * p.Hkv + g;
    const float k_old = p.k_scales[unit], v_old = p.v_scales[unit];
    float k_most = 0.f, v_most = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (fabsf(k[i][j]) < INFINITY) k_most = fmaxf(k_most, fabsf(k[i][j]));
            if (fabsf(v[i][j]) < INFINITY) v_most = fmaxf(v_most, fabsf(v[i][j]));
        }
#pragma unroll
    for (int off = TPR / 2; off > 0; off >>= 1) {
        k_most = fmaxf(k_most, __shfl_xor(k_most, off, 64));
        v_most = fmaxf(v_most, __shfl_xor(v_most, off, 64));
    }
    float k_new = scale_for(k_most), v_new = scale_for(v_most);
    uint8_t *kp = (uint8_t *)p.k + ((unit << p.ps_log) * HD), *vp = (uint8_t *)p.v + ((unit << p.ps_log) * HD);
    if (slot > 0) {
        if (k_new > k_old) recode<HD>(kp, slot, k_old / k_new, threadIdx.x & (TPR - 1), TPR); else k_new = fmaxf(k_new, k_old);
        if (v_new > v_old) recode<HD>(vp, slot, v_old / v_new, threadIdx.x & (TPR - 1), TPR); else v_new = fmaxf(v_new, v_old);
    }
    if (c == 0) {
        p.k_scales[unit] = k_new;
        p.v_scales[unit] = v_new;
    }
    const size_t off = (size_t)slot * HD + c;
    *(uint2 *)(kp + off) = codes8(k[0], 1.f / k_new);
    *(uint2 *)(kp + off + HALF) = codes8(k[1], 1.f / k_new);
    *(uint2 *)(vp + off) = codes8(v[0], 1.f / v_new);
    *(uint2 *)(vp + off + HALF) = codes8(v[1], 1.f / v_new);
}

// Workgroups of a launch: 2^32 threads are more than a grid can have, and a call of 2^24 rows has up to 2^30 workgroups.
constexpr int kAppendGroups = 1 << 23;

template <int HD>
static hipError_t launch_codes(const PagedAppendArgs &a, int page_groups, int per_group, int groups, hipStream_t s)
{
    for (int first = 0; first < groups; first += kAppendGroups) {
        const unsigned grid = (unsigned)(groups - first < kAppendGroups ? groups - first : kAppendGroups);
        switch ((HD << a.p.ps_log) / 4096) {         // rounds that a full page takes
        case 0: case 1: paged_append_codes_kernel<HD, 1><<<grid, 256, 0, s>>>(a, page_groups, per_group, first); break;
        case 2: paged_append_codes_kernel<HD, 2><<<grid, 256, 0, s>>>(a, page_groups, per_group, first); break;
        default: paged_append_codes_kernel<HD, 4><<<grid, 256, 0, s>>>(a, page_groups, per_group, first); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_paged_append(int kind, int hd, const PagedAppendArgs &a, hipStream_t s)
{
    // a workgroup per row while that leaves CUs idle, then four: one search and one set of angles per wave
    const int per_group = a.p.n_rows <= 1024 ? 1 : kRowsPerGroup;
    const unsigned row_groups = (unsigned)((a.p.n_rows + per_group - 1) / per_group);
    if (kind == PAGED_E4M3 && !a.p.starts) {
        const int64_t threads = (int64_t)a.p.n_seqs * ((a.q ? a.Hq : 0) + a.p.Hkv) * (hd / 16);
        const unsigned grid = (unsigned)((threads + 255) / 256);
        if (hd == 128) paged_append_one_kernel<128><<<grid, 256, 0, s>>>(a);
        else paged_append_one_kernel<64><<<grid, 256, 0, s>>>(a);
    } else if (kind == PAGED_E4M3) {
        const int page_groups = (a.p.n_rows >> a.p.ps_log) + 2 * a.p.n_seqs;
        const int groups = page_groups * a.p.Hkv + (a.q ? (int)row_groups : 0);
        return hd == 128 ? launch_codes<128>(a, page_groups, per_group, groups, s) : launch_codes<64>(a, page_groups, per_group, groups, s);
    } else if (kind == PAGED_BF16) {
        if (hd == 128) paged_append_rows_kernel<uint16_t, 128><<<row_groups, 256, 0, s>>>(a, per_group);
        else paged_append_rows_kernel<uint16_t, 64><<<row_groups, 256, 0, s>>>(a, per_group);
    } else {
        if (hd == 128) paged_append_rows_kernel<float, 128><<<row_groups, 256, 0, s>>>(a, per_group);
        else paged_append_rows_kernel<float, 64><<<row_groups, 256, 0, s>>>(a, per_group);
    }
    return hipGetLastError();
}

}  // namespace pd
