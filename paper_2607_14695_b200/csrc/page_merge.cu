// Joins the partial results of units that several CTAs have worked on: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, in the order of the keys.
// A warp per row and 64 columns: the (m, l) pairs of up to 32 partials at a time, one a lane, then their O with eight loads in flight.
#include <math.h>

#include "page_attention.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

constexpr int kMergeWarps = 8;

__global__ void __launch_bounds__(32 * kMergeWarps)
page_merge_kernel(const PageAttention p, const PagePartials part)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 meta = part.meta[blockIdx.x];
    if (meta.x < 0) return;
    const int cta = blockIdx.x, rows = meta.z & 0xffff, h = (int)((uint32_t)meta.z >> 16), n = meta.w - cta + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int d = p.g.d, groups = d >> 6, G = p.g.Hq / p.g.Hkv;
    const int item = blockIdx.y * kMergeWarps + warp;
    const int r = item / groups, c0 = item % groups * 64 + 2 * lane;
    if (r >= rows) return;
    auto slot = [&](int i) -> size_t { return ((size_t)(i == 0 ? 2 * cta + 1 : 2 * (cta + i))) * part.rows + r; };
    float m = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int mine = i0 + lane;
        const float2 ml = mine < n ? part.ml[slot(mine)] : make_float2(-INFINITY, 0.f);
        float top = ml.x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        top = fmaxf(top, m);
        const float old = m == -INFINITY ? 0.f : ptx::ex2(m - top);
        float w = ml.x == -INFINITY ? 0.f : ptx::ex2(ml.x - top);
        float sum = ml.y * w;                                       // (a NaN sum stays one)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        l = l * old + sum;
        a0 *= old; a1 *= old;
        m = top;
        const int count = min(32, n - i0);
        for (int j0 = 0; j0 < count; j0 += 8) {
            float2 v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j0 + j < count) v[j] = *reinterpret_cast<const float2 *>(part.o + slot(i0 + j0 + j) * d + c0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float wj = __shfl_sync(0xffffffffu, w, (j0 + j) & 31);
                if (j0 + j < count && wj != 0.f) { a0 = fmaf(v[j].x, wj, a0); a1 = fmaf(v[j].y, wj, a1); }
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int rr = meta.y + r;
    __nv_bfloat16 *out = (__nv_bfloat16 *)p.out + ((size_t)(meta.x + rr / G) * p.g.Hq + h * G + rr % G) * d + c0;
    *reinterpret_cast<uint32_t *>(out) = pack_bf16(a0 * inv, a1 * inv);
}

cudaError_t launch_page_merge(const PageAttention &a, const PagePartials &part, int ctas, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas, (unsigned)((part.rows * (a.g.d / 64) + kMergeWarps - 1) / kMergeWarps));
    cfg.blockDim = dim3(32 * kMergeWarps);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, page_merge_kernel, a, part);
}

}  // namespace reflex
