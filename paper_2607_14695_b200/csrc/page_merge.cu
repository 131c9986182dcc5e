// Joins the partial results of units that several CTAs have worked on: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, in an order that the
// units alone decide. A thread takes 8 columns of a row (partials lie as [column group][row][8], so a warp reads a contiguous kilobyte) and has
// the loads of 4 partials in flight; long lists (one sequence over the whole device) are cut in 8 among the warps of a block, which then add up.
//
// It also computes again, row by row, the sequences that the tensor-core kernel has marked (see PagePartials::careful).
#include "page_plain.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

constexpr int kMergeThreads = 256;
constexpr int kMergeMost = kMostCtas;
constexpr int kMergeLong = 16;            // partials of a unit from which on its list is cut

struct MergeSum { float m, l, o[8]; };

__device__ __forceinline__ void merge_list(const PagePartials &part, int d, int cta, int n, int r, int c0, int first, int step, MergeSum &a)
{
    auto slot = [&](int i) -> size_t { return i == 0 ? 2 * (size_t)cta + 1 : 2 * (size_t)(cta + i); };
    a.m = -INFINITY; a.l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) a.o[e] = 0.f;
    for (int i0 = first; i0 < n; i0 += 4 * step) {
        float4 v[4][2];
        float2 ml[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * step;
            if (i < n) {
                ml[j] = part.ml[slot(i) * part.rows + r];
                const float4 *src = reinterpret_cast<const float4 *>(partial8(part, slot(i), d, r, c0));
                v[j][0] = src[0]; v[j][1] = src[1];
            } else ml[j] = make_float2(-INFINITY, 0.f);
        }
        float top = a.m;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, ml[j].x);
        const float old = a.m == -INFINITY ? 0.f : ptx::ex2(a.m - top);
        a.l *= a.m == -INFINITY ? 1.f : old;             // (0, or the NaN of a part that went wrong)
#pragma unroll
        for (int e = 0; e < 8; ++e) a.o[e] *= old;
        a.m = top;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float w = ml[j].x == -INFINITY ? 0.f : ptx::ex2(ml[j].x - top);
            a.l += ml[j].y * w;
            if (w == 0.f) continue;                     // (what a part that has seen nothing left there is not looked at)
            const float f[8] = {v[j][0].x, v[j][0].y, v[j][0].z, v[j][0].w, v[j][1].x, v[j][1].y, v[j][1].z, v[j][1].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) a.o[e] = fmaf(f[e], w, a.o[e]);
        }
    }
}

template <int FMT>
__global__ void __launch_bounds__(kMergeThreads, 4)
page_merge_kernel(const PageAttention p, const PagePartials part, int ctas)
{
    __shared__ int first_s[kMergeMost + 1];        // first piece of work of each unit that was split (by the CTA that began it)
    __shared__ __align__(16) uint8_t scratch[kMergeThreads * 44];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int d = p.g.d, groups = d >> 3, G = p.g.Hq / p.g.Hkv;
    // pieces: 256 (row, column group) items of a unit; 32 where its list of partials is cut
    // (sequences are marked before this kernel, and the marks go when its last block is done: all blocks see the same)
    bool marked = false;
    for (int b = tid; b < p.q.B; b += kMergeThreads) marked |= part.careful[b] != 0;
    int pieces[2], of[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = 2 * tid + k;
        pieces[k] = 0;
        of[k] = -1;
        if (c < ctas) {
            const PageSplit m = part.meta[c];
            of[k] = m.b;
            const int per = m.last - c + 1 > kMergeLong ? 32 : 256;
            if (m.b >= 0) pieces[k] = (m.rows * groups + per - 1) / per;
        }
    }
    const bool any_marked = __syncthreads_or(marked);
    if (any_marked) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (of[k] >= 0 && part.careful[of[k]]) pieces[k] = 0;
    }
    {
        const int mine = pieces[0] + pieces[1];
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        int *sum_s = reinterpret_cast<int *>(scratch);
        if (lane == 31) sum_s[warp] = incl;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int q = 0; q < kMergeThreads / 32; ++q) {
            if (q < warp) before += sum_s[q];
            all += sum_s[q];
        }
        static_assert(kMergeMost == 2 * kMergeThreads, "two entries a thread");
        first_s[2 * tid] = before + incl - mine;
        first_s[2 * tid + 1] = before + incl - mine + pieces[0];
        if (tid == 0) first_s[kMergeMost] = all;
        if (ctas < kMergeMost && tid == 0) first_s[ctas] = all;
        __syncthreads();
    }
    for (int w = blockIdx.x; w < first_s[ctas]; w += gridDim.x) {
        int lo = 0, hi = ctas;                      // first_s[lo] <= w < first_s[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_s[mid] <= w) lo = mid; else hi = mid;
        }
        const PageSplit m = part.meta[lo];
        const int n = m.last - lo + 1;
        const bool cut = n > kMergeLong;
        const int item = (w - first_s[lo]) * (cut ? 32 : 256) + (cut ? lane : tid);
        const int r = item % m.rows, c0 = item / m.rows * 8, at = r < m.half ? r : 128 + r - m.half;
        const bool live = c0 < d;
        MergeSum a;
        if (live) merge_list(part, d, lo, n, at, c0, cut ? warp : 0, cut ? 8 : 1, a);
        if (cut) {
            MergeSum *all = reinterpret_cast<MergeSum *>(scratch);
            __syncthreads();
            if (live) all[tid] = a;
            __syncthreads();
            if (warp > 0 || !live) continue;
            for (int q = 1; q < 8; ++q) {
                const MergeSum b = all[q * 32 + lane];
                const float top = fmaxf(a.m, b.m), fa = a.m == -INFINITY ? 0.f : ptx::ex2(a.m - top), fb = b.m == -INFINITY ? 0.f : ptx::ex2(b.m - top);
                a.l = (a.m == -INFINITY ? a.l : a.l * fa) + (b.m == -INFINITY ? b.l : b.l * fb);
#pragma unroll
                for (int e = 0; e < 8; ++e) a.o[e] = a.o[e] * fa + b.o[e] * fb;
                a.m = top;
            }
        }
        if (!live) continue;
        const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
#pragma unroll
        for (int e = 0; e < 8; ++e) a.o[e] *= inv;
        const int rr = m.first + r;
        store8((__nv_bfloat16 *)p.out + ((size_t)(m.row0 + rr / G) * p.g.Hq + m.h * G + rr % G) * d + c0, a.o);
    }
    if (!any_marked) return;
    // ---- marked sequences ----
    __syncthreads();
    float *q_s = reinterpret_cast<float *>(scratch) + warp * 256;
    for (int b = 0; b < p.q.B; ++b) {
        if (!part.careful[b]) continue;
        const PageSeq s = page_seq(p, b);
        const long long items = (long long)s.n * p.g.Hq, warps = (long long)gridDim.x * (kMergeThreads / 32);
        for (long long i = (long long)blockIdx.x * (kMergeThreads / 32) + warp; i < items; i += warps) {
            const int t = (int)(i / p.g.Hq);
            page_plain_row<__nv_bfloat16, FMT>(p, b, s.row0 + t, (int64_t)s.len - s.n + t, s.len, (int)(i % p.g.Hq), q_s);
        }
    }
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        if (atomicAdd(part.careful_done, 1u) == gridDim.x - 1u) {
            for (int b = 0; b < p.q.B; ++b) part.careful[b] = 0;
            *part.careful_done = 0u;
        }
    }
}

cudaError_t launch_page_merge(const PageAttention &a, const PagePartials &part, int ctas, int format, int sm_count, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(4 * sm_count));
    cfg.blockDim = dim3(kMergeThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    count_launch();
    if (format == REFLEX_PAGE_SAME) return cudaLaunchKernelEx(&cfg, page_merge_kernel<REFLEX_PAGE_SAME>, a, part, ctas);
    if (format == REFLEX_PAGE_E4M3) return cudaLaunchKernelEx(&cfg, page_merge_kernel<REFLEX_PAGE_E4M3>, a, part, ctas);
    return cudaLaunchKernelEx(&cfg, page_merge_kernel<REFLEX_PAGE_INT8>, a, part, ctas);
}

}  // namespace reflex
