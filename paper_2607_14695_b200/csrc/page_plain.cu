// Attention over pages, plain form: fp32 FMAs, one warp per (token, query head), any storage and head width. Keys are taken 32 at a time:
// a lane computes one logit, then all lanes add up their columns of the weighted values. Masked keys are never touched, so nothing that
// lies in them matters.
#include <math.h>

#include "pages.cuh"

namespace reflex {

constexpr int kPlainWarps = 4;

template <typename T, int FMT>
__device__ __forceinline__ void load8_page(const void *pool, size_t at, float *f)
{
    if constexpr (FMT == REFLEX_PAGE_SAME) load8((const T *)pool + at, f);
    else {
        const uint2 w = *reinterpret_cast<const uint2 *>((const uint8_t *)pool + at);
        const uint32_t o[4] = {bytes_to_bf16x2<FMT, 0, 1>(w.x, w.x), bytes_to_bf16x2<FMT, 2, 3>(w.x, w.x), bytes_to_bf16x2<FMT, 0, 1>(w.y, w.y), bytes_to_bf16x2<FMT, 2, 3>(w.y, w.y)};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(o[i] << 16); f[2 * i + 1] = __uint_as_float(o[i] & 0xffff0000u); }
    }
}

template <typename T, int FMT>
__global__ void __launch_bounds__(32 * kPlainWarps)
page_plain_kernel(const PageAttention p)
{
    extern __shared__ int cu_s[];
    __shared__ __align__(16) float q_s[kPlainWarps][256];
    load_cu(p.q, cu_s);
    __syncthreads();
    const PageGeom &g = p.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * kPlainWarps + warp;
    const int64_t row = item / g.Hq;
    const int hq = (int)(item % g.Hq);
    if (row >= p.n_rows || row >= cu_s[p.q.B] || row < cu_s[0]) return;
    const int b = find_seq(cu_s, p.q.B, (int)row), h = hq / (g.Hq / g.Hkv);
    const int len = p.q.len[b];
    const int64_t pos = (int64_t)len - cu_s[b + 1] + row;
    const T *qr = (const T *)p.qry + ((size_t)row * g.Hq + hq) * g.d;
    for (int i = lane; i < g.d; i += 32) q_s[warp][i] = (float)qr[i];
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
                for (int e = 0; e < 8; ++e) s = fmaf(k8[e], q_s[warp][i + e], s);
            }
            if constexpr (FMT != REFLEX_PAGE_SAME) { s *= exponent_f32(g.ke[at]); vs = exponent_f32(g.ve[at]); }
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
                    v = __uint_as_float(bytes_to_bf16x2<FMT, 0, 0>(w8, w8) << 16);
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

cudaError_t launch_page_plain(const PageAttention &a, int dtype, int format, cudaStream_t st)
{
    const int64_t items = (int64_t)a.n_rows * a.g.Hq;
    const unsigned grid = (unsigned)((items + kPlainWarps - 1) / kPlainWarps);
    const size_t smem = (size_t)(a.q.B + 1) * 4;
    count_launch();
    auto go = [&](auto zero, auto f) { page_plain_kernel<decltype(zero), decltype(f)::value><<<grid, 32 * kPlainWarps, smem, st>>>(a); };
    auto fmt = [&](auto zero) {
        if (format == REFLEX_PAGE_SAME) go(zero, std::integral_constant<int, REFLEX_PAGE_SAME>{});
        else if (format == REFLEX_PAGE_E4M3) go(zero, std::integral_constant<int, REFLEX_PAGE_E4M3>{});
        else go(zero, std::integral_constant<int, REFLEX_PAGE_INT8>{});
    };
    if (dtype == REFLEX_DTYPE_F32) fmt(float{}); else fmt(__nv_bfloat16{});
    return cudaGetLastError();
}

}  // namespace reflex
