// Joining the partial results of a unit: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, in the order of the keys.
#pragma once

#include "page_attention.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

struct PageSum { float m, l, o[8]; };

// partials first, first + step .. of the n of a unit that CTA (or pair) `cta` began, of 8 columns of a row
__device__ __forceinline__ void page_sum(const PagePartials &part, int d, int cta, int n, int r, int c0, int first, int step, PageSum &a)
{
    auto slot = [&](int i) -> size_t { return i == 0 ? 2 * (size_t)cta + 1 : 2 * (size_t)(cta + i); };
    a.m = -INFINITY; a.l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) a.o[e] = 0.f;
    for (int i0 = first; i0 < n; i0 += 8 * step) {
        float v[8][8];
        float2 ml[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * step;
            if (i < n) {
                ml[j] = part.ml[slot(i) * part.rows + r];
                ptx::ld_global_v8(partial8(part, slot(i), d, r, c0), v[j]);
            } else ml[j] = make_float2(-INFINITY, 0.f);
        }
        float top = a.m;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, ml[j].x);
        // (a weight may underflow to 0: what was finite then counts nothing, and an infinity makes NaN, as it does inside a part)
        const float old = a.m == -INFINITY ? 1.f : ptx::ex2(a.m - top);
        a.l *= old;                                      // (0, or the NaN of a part that went wrong)
#pragma unroll
        for (int e = 0; e < 8; ++e) a.o[e] *= old;
        a.m = top;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float w = ml[j].x == -INFINITY ? 0.f : ptx::ex2(ml[j].x - top);
            a.l += ml[j].y * w;
            if (ml[j].x == -INFINITY) continue;         // (what a part that has seen nothing left there is not looked at)
#pragma unroll
            for (int e = 0; e < 8; ++e) a.o[e] = fmaf(v[j][e], w, a.o[e]);
        }
    }
}

}  // namespace reflex
