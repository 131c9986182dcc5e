// Attention of one (token, query head) row over pages with fp32 FMAs, by one warp or several: any storage and head width. Keys are taken 32 at a time:
// a lane computes one logit, then all lanes add up their columns of the weighted values. Masked keys are never touched, so nothing that
// lies in them matters.
#pragma once

#include <math.h>

#include "page_attention.cuh"

namespace reflex {

// COLS consecutive elements of storage (T, or bytes of an 8-bit format without their exponent), as floats
template <typename T, int FMT, int COLS>
__device__ __forceinline__ void load_columns(const void *pool, size_t at, float (&v)[8])
{
    constexpr int BYTES = COLS * (FMT == REFLEX_PAGE_SAME ? (int)sizeof(T) : 1);
    const uint8_t *src = (const uint8_t *)pool + at * (FMT == REFLEX_PAGE_SAME ? sizeof(T) : 1);
    uint32_t w[BYTES < 4 ? 1 : BYTES / 4];
    if constexpr (BYTES == 1) w[0] = *src;
    else if constexpr (BYTES == 2) w[0] = *reinterpret_cast<const uint16_t *>(src);
    else if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t *>(src);
    else if constexpr (BYTES == 8) { const uint2 x = *reinterpret_cast<const uint2 *>(src); w[0] = x.x; w[1] = x.y; }
    else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const uint4 x = reinterpret_cast<const uint4 *>(src)[i];
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
    }
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
        if constexpr (FMT != REFLEX_PAGE_SAME) {
            const uint32_t byte = (w[i >> 2] >> (8 * (i & 3))) & 0xffu;
            v[i] = __uint_as_float(expand2<FMT, 0, 0>(biased<FMT>(byte)) << 16);
        } else if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
        else v[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
}

// This lane's COLS columns of eight rows, those of lanes k0 .. k0 + 7: coalesced, and all on their way together. (Rows that are not to be read have `at` 0,
// the first row there is.)
template <typename T, int FMT, int COLS>
__device__ __forceinline__ void load_rows8(const void *pool, size_t at, int k0, float (&v)[8][8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) load_columns<T, FMT, COLS>(pool, (__shfl_sync(0xffffffffu, (unsigned long long)at, k0 + k) * 32 + (threadIdx.x & 31)) * COLS, v[k]);
}

// of a row: d / 32 consecutive columns of the weighted values, this lane's share of the weights, the row's maximum
struct PlainSum { float acc[8], m, l; bool bad; };

// Blocks first, first + step, .. of 32 keys of a row. (With a key's row to each lane and values one by one, 273 keys of 64 columns took 142 us.)
template <typename T, int FMT, int COLS>
__device__ __forceinline__ void page_plain_sum(const PageAttention &p, int b, int row, int64_t pos, int len, int hq, int first, int step, PlainSum &a)
{
    const PageGeom &g = p.g;
    constexpr float kShare = 0x1p-24f;
    static_assert(kWeightShift == 24.f, "2^-kWeightShift");
    const int lane = threadIdx.x & 31, h = hq / (g.Hq / g.Hkv);
    const int64_t cap = (int64_t)p.q.max_pages << g.log_p;          // (of positions past the table the first one is looked at)
    const int64_t hi = min(p.causal ? min((int64_t)len, pos + 1) : (int64_t)len, cap + 1);
    const int64_t lo = min(p.window > 0 ? max((int64_t)0, pos - p.window + 1) : (int64_t)0, cap);
    float q[8];
    load_columns<T, REFLEX_PAGE_SAME, COLS>(p.qry, (((size_t)row * g.Hq + hq) * 32 + lane) * COLS, q);
    a.m = -INFINITY; a.l = 0.f;
    a.bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) a.acc[i] = 0.f;
    for (int64_t j0 = (lo & ~31ll) + 32 * first; j0 < hi; j0 += 32 * step) {
        const int64_t j = j0 + lane;
        const bool seen = j >= lo && j < hi;
        const int page = seen ? page_at(p.q, g.n_pages, b, (int)(j >> g.log_p)) : -1;
        a.bad |= seen && page < 0;
        const size_t at = page < 0 ? 0 : page_row(g, page, h) + (size_t)(j & (g.P - 1));
        const uint32_t live = __ballot_sync(0xffffffffu, page >= 0);
        float s = 0.f, vs = 1.f, v[8][8];
#pragma unroll 1
        for (int k0 = 0; k0 < 32; k0 += 8) {
            if (((live >> k0) & 0xffu) == 0u) continue;
            load_rows8<T, FMT, COLS>(g.k, at, k0, v);
            // eight sums over the lanes, halved among them: key k0 + lane / 4 is left
            float sum[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sum[k] = 0.f;
#pragma unroll
                for (int i = 0; i < COLS; ++i) sum[k] = fmaf(v[k][i], q[i], sum[k]);
            }
#pragma unroll
            for (int n = 4; n > 0; n >>= 1) {
                const bool upper = (lane & (4 * n)) != 0;
#pragma unroll
                for (int c = 0; c < n; ++c) {
                    const float other = __shfl_xor_sync(0xffffffffu, upper ? sum[c] : sum[c + n], 4 * n);
                    sum[c] = (upper ? sum[c + n] : sum[c]) + other;
                }
            }
            sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], 2);
            sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], 1);
            const float mine = __shfl_sync(0xffffffffu, sum[0], (lane & 7) * 4);
            if ((lane & 24) == k0) s = mine;
        }
        if (page >= 0) {
            if constexpr (FMT != REFLEX_PAGE_SAME) { s *= exponent_f32<FMT>(g.ke[at]); vs = exponent_f32<FMT>(g.ve[at]); }
            s *= p.scale;
        } else s = -INFINITY;
        float top = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float x = __shfl_xor_sync(0xffffffffu, top, o);
            top = !(x <= top) ? x : top;         // (a NaN stays, or shows in the sum)
        }
        const float m_new = !(top <= a.m) ? top : a.m;
        const float mr = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = expf(a.m - mr), w = page >= 0 ? expf(s - mr) * kShare : 0.f, wv = w * vs;
        a.m = m_new;
        a.l = a.l * alpha + w;
#pragma unroll
        for (int i = 0; i < COLS; ++i) a.acc[i] *= alpha;
#pragma unroll 1
        for (int k0 = 0; k0 < 32; k0 += 8) {
            if (((live >> k0) & 0xffu) == 0u) continue;
            load_rows8<T, FMT, COLS>(g.v, at, k0, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float wj = __shfl_sync(0xffffffffu, wv, k0 + k);
                const bool there = (live >> (k0 + k)) & 1u;
#pragma unroll
                for (int i = 0; i < COLS; ++i) a.acc[i] = fmaf(wj, there ? v[k][i] : 0.f, a.acc[i]);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a.l += __shfl_xor_sync(0xffffffffu, a.l, o);
    a.bad = __any_sync(0xffffffffu, a.bad);
}
template <typename T, int FMT>
__device__ __forceinline__ void page_plain_sum(const PageAttention &p, int b, int row, int64_t pos, int len, int hq, int first, int step, PlainSum &a)
{
    if (p.g.d == 32) page_plain_sum<T, FMT, 1>(p, b, row, pos, len, hq, first, step, a);
    else if (p.g.d == 64) page_plain_sum<T, FMT, 2>(p, b, row, pos, len, hq, first, step, a);
    else if (p.g.d == 128) page_plain_sum<T, FMT, 4>(p, b, row, pos, len, hq, first, step, a);
    else page_plain_sum<T, FMT, 8>(p, b, row, pos, len, hq, first, step, a);
}

// the whole warp
template <typename T>
__device__ __forceinline__ void page_plain_write(const PageAttention &p, int b, int row, int hq, PlainSum &a)
{
    const int lane = threadIdx.x & 31, cols = p.g.d >> 5;
    if (a.bad) {
        if (lane == 0) report_bad_page(p.g.status, b);
        a.l = __int_as_float(0x7fc00000);
    }
    // (nothing seen, or every logit -inf: 0)
    const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
    T *o = (T *)p.out + ((size_t)row * p.g.Hq + hq) * p.g.d;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < cols) {
            const float f = a.acc[i] * inv;
            if constexpr (sizeof(T) == 4) o[lane * cols + i] = f; else o[lane * cols + i] = __float2bfloat16_rn(f);
        }
}

// by one warp
template <typename T, int FMT>
__device__ __forceinline__ void page_plain_row(const PageAttention &p, int b, int row, int64_t pos, int len, int hq)
{
    PlainSum a;
    page_plain_sum<T, FMT>(p, b, row, pos, len, hq, 0, 1, a);
    page_plain_write<T>(p, b, row, hq, a);
}

}  // namespace reflex
