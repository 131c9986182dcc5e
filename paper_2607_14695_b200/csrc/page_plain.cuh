// Attention of one (token, query head) row over pages with fp32 FMAs, by one warp: any storage and head width. Keys are taken 32 at a time:
// a lane computes one logit, then all lanes add up their columns of the weighted values. Masked keys are never touched, so nothing that
// lies in them matters.
#pragma once

#include <math.h>

#include "page_attention.cuh"

namespace reflex {

template <typename T, int FMT>
__device__ __forceinline__ void load8_page(const void *pool, size_t at, float *f)
{
    if constexpr (FMT == REFLEX_PAGE_SAME) load8((const T *)pool + at, f);
    else {
        const uint2 w = *reinterpret_cast<const uint2 *>((const uint8_t *)pool + at);
        const uint32_t o[4] = {expand2<FMT, 0, 1>(biased<FMT>(w.x)), expand2<FMT, 2, 3>(biased<FMT>(w.x)), expand2<FMT, 0, 1>(biased<FMT>(w.y)), expand2<FMT, 2, 3>(biased<FMT>(w.y))};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(o[i] << 16); f[2 * i + 1] = __uint_as_float(o[i] & 0xffff0000u); }
    }
}

// q_s: 256 floats of shared memory of this warp's own
template <typename T, int FMT>
__device__ __forceinline__ void page_plain_row(const PageAttention &p, int b, int row, int64_t pos, int len, int hq, float *q_s)
{
    const PageGeom &g = p.g;
    const int lane = threadIdx.x & 31, h = hq / (g.Hq / g.Hkv);
    const T *qr = (const T *)p.qry + ((size_t)row * g.Hq + hq) * g.d;
    __syncwarp();
    for (int i = lane; i < g.d; i += 32) q_s[i] = (float)qr[i];
    __syncwarp();
    const int64_t hi = p.causal ? min((int64_t)len, pos + 1) : len;
    const int64_t lo = p.window > 0 ? max((int64_t)0, pos - p.window + 1) : 0;
    const int cols = g.d >> 5;                  // columns lane, lane + 32, ...
    float acc[8], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    bool bad = false;
    for (int64_t j0 = lo & ~31ll; j0 < hi; j0 += 32) {
        const int64_t j = j0 + lane;
        const bool seen = j >= lo && j < hi;
        const int page = seen ? page_at(p.q, g.n_pages, b, (int)(j >> g.log_p)) : -1;
        bad |= seen && page < 0;
        const size_t at = page < 0 ? 0 : page_row(g, page, h) + (size_t)(j & (g.P - 1));
        float s = -INFINITY, vs = 1.f;
        if (page >= 0) {
            s = 0.f;
            for (int i = 0; i < g.d; i += 8) {
                float k8[8];
                load8_page<T, FMT>(g.k, at * g.d + i, k8);
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fmaf(k8[e], q_s[i + e], s);
            }
            if constexpr (FMT != REFLEX_PAGE_SAME) { s *= exponent_f32<FMT>(g.ke[at]); vs = exponent_f32<FMT>(g.ve[at]); }
            s *= p.scale;
        }
        float top = s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float x = __shfl_xor_sync(0xffffffffu, top, o);
            top = !(x <= top) ? x : top;         // (a NaN stays, or shows in the sum)
        }
        const float m_new = !(top <= m) ? top : m;
        const float mr = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = expf(m - mr), w = page >= 0 ? expf(s - mr) : 0.f;
        m = m_new;
        l = l * alpha + w;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] *= alpha;
        for (uint32_t todo = __ballot_sync(0xffffffffu, page >= 0); todo; todo &= todo - 1) {
            const int src = __ffs(todo) - 1;
            const float wj = __shfl_sync(0xffffffffu, w, src) * __shfl_sync(0xffffffffu, vs, src);
            const size_t vat = __shfl_sync(0xffffffffu, (unsigned long long)at, src) * g.d;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= cols) break;
                float v;
                if constexpr (FMT == REFLEX_PAGE_SAME) v = (float)((const T *)g.v)[vat + lane + 32 * i];
                else {
                    const uint32_t w8 = ((const uint8_t *)g.v)[vat + lane + 32 * i];
                    v = __uint_as_float(expand2<FMT, 0, 0>(biased<FMT>(w8)) << 16);
                }
                acc[i] = fmaf(wj, v, acc[i]);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (__any_sync(0xffffffffu, bad)) {
        if (lane == 0) report_bad_page(g.status, b);
        l = __int_as_float(0x7fc00000);
    }
    // (nothing seen, or every logit -inf: 0)
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *o = (T *)p.out + ((size_t)row * g.Hq + hq) * g.d;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < cols) {
            const float f = acc[i] * inv;
            if constexpr (sizeof(T) == 4) o[lane + 32 * i] = f; else o[lane + 32 * i] = __float2bfloat16_rn(f);
        }
}

}  // namespace reflex
