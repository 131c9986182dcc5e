// Joins the partial results of units that several CTAs have worked on: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, in an order that the units
// alone decide. A thread takes 8 columns of a row (partials lie as [column group][row][8], so a warp reads a contiguous kilobyte) and has the loads of 8
// partials in flight (which is why there are two blocks per SM and not four: a frame of 256 tokens over 3376 keys in 23.9 us, not 27.0); long lists (one
// sequence over the whole device) are cut among the warps of a block, which then add up.
//
// It also computes again, row by row, the sequences that the tensor-core kernel has marked (see PagePartials::careful). That is the plain kernel's work,
// one row at a time: with one value of one sequence not finite at a key that some rows of a unit see and others do not, a causal frame of 256 tokens over
// 3376 keys takes 0.76 ms and not 0.024, 16 such frames 1.6 and not 0.115, a causal prefill of 4160 tokens (16 heads of 128) 10.2 and not 0.30.
#include "page_join.cuh"
#include "page_plain.cuh"

namespace reflex {

constexpr int kMergeThreads = 256;
constexpr int kMergeMost = kMostPairs;
constexpr int kMergeLong = 16;            // partials of a unit from which on its list is cut
constexpr int kMergeCut = 4;              // ... in so many

__device__ __forceinline__ void page_add(PageSum &a, const PageSum &b)
{
    const float top = fmaxf(a.m, b.m), fa = a.m == -INFINITY ? 0.f : ptx::ex2(a.m - top), fb = b.m == -INFINITY ? 0.f : ptx::ex2(b.m - top);
    a.l = (a.m == -INFINITY ? a.l : a.l * fa) + (b.m == -INFINITY ? b.l : b.l * fb);
#pragma unroll
    for (int e = 0; e < 8; ++e) a.o[e] = a.o[e] * fa + b.o[e] * fb;
    a.m = top;
}

template <int FMT>
__global__ void __launch_bounds__(kMergeThreads, 2)
page_merge_kernel(const PageAttention p, const PagePartials part, int pairs)
{
    __shared__ int first_s[kMergeMost + 1];        // first piece of work of each unit that was split (by the CTA that began it)
    __shared__ __align__(16) uint8_t scratch[kMergeThreads * 44];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int d = p.g.d, groups = d >> 3, G = p.g.Hq / p.g.Hkv;
    // pieces: 256 (row, column group) items of a unit; fewer where its list of partials is cut
    constexpr int kItems = kMergeThreads / kMergeCut;
    // (sequences are marked before this kernel, and the marks go when its last block is done: all blocks see the same)
    bool marked = false;
    for (int b = tid; b < p.q.B; b += kMergeThreads) marked |= part.careful[b] != 0;
    int pieces = 0, of = -1;
    if (tid < pairs) {
        const PageSplit s = part.meta[tid];
        of = s.b;
        const int per = s.last - tid + 1 > kMergeLong ? kItems : kMergeThreads;
        if (s.b >= 0) pieces = (s.rows * groups + per - 1) / per;
    }
    const bool any_marked = __syncthreads_or(marked);
    if (any_marked && of >= 0 && part.careful[of]) pieces = 0;
    {
        int incl = pieces;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        int *sum_s = reinterpret_cast<int *>(scratch);
        if (lane == 31) sum_s[warp] = incl;
        __syncthreads();
        int before = 0;
        for (int q = 0; q < warp; ++q) before += sum_s[q];
        static_assert(kMergeMost < kMergeThreads, "an entry a thread, and the end");
        if (tid <= pairs) first_s[tid] = before + incl - pieces;
        __syncthreads();
    }
    for (int w = blockIdx.x; w < first_s[pairs]; w += gridDim.x) {
        int lo = 0, hi = pairs;                      // first_s[lo] <= w < first_s[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_s[mid] <= w) lo = mid; else hi = mid;
        }
        const PageSplit m = part.meta[lo];
        const int n = m.last - lo + 1;
        const bool cut = n > kMergeLong;
        const int item = (w - first_s[lo]) * (cut ? kItems : kMergeThreads) + (cut ? tid % kItems : tid);
        const int r = item % m.rows, c0 = item / m.rows * 8, at = r < m.half ? r : 128 + r - m.half;
        const bool live = c0 < d;
        PageSum a;
        if (live) page_sum(part, d, lo, n, at, c0, cut ? tid / kItems : 0, cut ? kMergeCut : 1, a);
        if (cut) {
            PageSum *all = reinterpret_cast<PageSum *>(scratch);
            __syncthreads();
            if (live) all[tid] = a;
            __syncthreads();
            if (tid >= kItems || !live) continue;
            for (int q = 1; q < kMergeCut; ++q) page_add(a, all[q * kItems + tid]);
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
    for (int b = 0; b < p.q.B; ++b) {
        if (!part.careful[b]) continue;
        const PageSeq s = page_seq(p, b);
        const long long items = (long long)s.n * p.g.Hq, warps = (long long)gridDim.x * (kMergeThreads / 32);
        for (long long i = (long long)blockIdx.x * (kMergeThreads / 32) + warp; i < items; i += warps) {
            const int t = (int)(i / p.g.Hq);
            page_plain_row<__nv_bfloat16, FMT>(p, b, s.row0 + t, (int64_t)s.len - s.n + t, s.len, (int)(i % p.g.Hq));
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

cudaError_t launch_page_merge(const PageAttention &a, const PagePartials &part, int pairs, int format, int sm_count, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * sm_count));
    cfg.blockDim = dim3(kMergeThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    count_launch();
    if (format == REFLEX_PAGE_SAME) return cudaLaunchKernelEx(&cfg, page_merge_kernel<REFLEX_PAGE_SAME>, a, part, pairs);
    if (format == REFLEX_PAGE_E4M3) return cudaLaunchKernelEx(&cfg, page_merge_kernel<REFLEX_PAGE_E4M3>, a, part, pairs);
    return cudaLaunchKernelEx(&cfg, page_merge_kernel<REFLEX_PAGE_INT8>, a, part, pairs);
}

}  // namespace reflex
