// Attention over pages, plain form (page_plain.cuh): a warp per (token, query head), or a block where there are few. Serves fp32, heads of 32 and,
// from some rows on, groups of more than 128 heads. Bound by instructions and latency: every row reads its keys by itself, from L2.
#include "page_plain.cuh"

namespace reflex {

constexpr int kPlainWarps = 4, kSplitWarps = 16;
// Below this many (token, head) rows per SM the warps of a block share a row's keys: else a few warps alone wait for one load after the other. fp32, a warp
// and sixteen: 254 and 26 us for 8 rows of 817 keys, 2192 and 167 for 128 of 3300 (256 columns); 124 and 59 for 640 of 1000, but 11 and 29 for
// 640 of 60 (64 columns; how long sequences are is not known to the host); 177 and 252 for 3200 of 1000.
constexpr int kSplitRows = 4;

// SPLIT: the warps of a block share the keys of one row
template <typename T, int FMT, bool SPLIT>
__global__ void __launch_bounds__(32 * (SPLIT ? kSplitWarps : kPlainWarps))
page_plain_kernel(const PageAttention p)
{
    extern __shared__ int cu_s[];
    load_cu(p.q, cu_s);
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t item = SPLIT ? blockIdx.x : (int64_t)blockIdx.x * kPlainWarps + warp;
    const int64_t row = item / p.g.Hq;
    if (row >= p.n_rows || row >= cu_s[p.q.B] || row < cu_s[0]) return;
    const int b = find_seq(cu_s, p.q.B, (int)row), len = p.q.len[b], hq = (int)(item % p.g.Hq);
    const int64_t pos = (int64_t)len - cu_s[b + 1] + row;
    if constexpr (!SPLIT) page_plain_row<T, FMT>(p, b, (int)row, pos, len, hq);
    else {
        __shared__ float acc_s[kSplitWarps][256], m_s[kSplitWarps], l_s[kSplitWarps];
        __shared__ int bad_s[kSplitWarps];
        PlainSum a;
        page_plain_sum<T, FMT>(p, b, (int)row, pos, len, hq, warp, kSplitWarps, a);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc_s[warp][lane + 32 * i] = a.acc[i];
        if (lane == 0) { m_s[warp] = a.m; l_s[warp] = a.l; bad_s[warp] = a.bad; }
        __syncthreads();
        if (warp > 0) return;
        float top = -INFINITY;
        for (int q = 0; q < kSplitWarps; ++q) top = !(m_s[q] <= top) ? m_s[q] : top;
        const float mr = top == -INFINITY ? 0.f : top;
        PlainSum all;
        all.l = 0.f;
        all.bad = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) all.acc[i] = 0.f;
#pragma unroll 4
        for (int q = 0; q < kSplitWarps; ++q) {
            const float f = expf(m_s[q] - mr);
            all.l = fmaf(l_s[q], f, all.l);
            all.bad |= bad_s[q] != 0;
            if (m_s[q] == -INFINITY) continue;       // (nothing was seen: nothing there is looked at)
#pragma unroll
            for (int i = 0; i < 8; ++i) all.acc[i] = fmaf(acc_s[q][lane + 32 * i], f, all.acc[i]);
        }
        page_plain_write<T>(p, b, (int)row, hq, all);
    }
}

cudaError_t launch_page_plain(const PageAttention &a, int dtype, int format, int sm_count, cudaStream_t st)
{
    const int64_t items = (int64_t)a.n_rows * a.g.Hq;
    const bool split = items < kSplitRows * (int64_t)sm_count;
    const unsigned grid = (unsigned)(split ? items : (items + kPlainWarps - 1) / kPlainWarps);
    const size_t smem = (size_t)(a.q.B + 1) * 4;
    count_launch();
    auto go = [&](auto zero, auto f) {
        if (split) page_plain_kernel<decltype(zero), decltype(f)::value, true><<<grid, 32 * kSplitWarps, smem, st>>>(a);
        else page_plain_kernel<decltype(zero), decltype(f)::value, false><<<grid, 32 * kPlainWarps, smem, st>>>(a);
    };
    auto fmt = [&](auto zero) {
        if (format == REFLEX_PAGE_SAME) go(zero, std::integral_constant<int, REFLEX_PAGE_SAME>{});
        else if (format == REFLEX_PAGE_E4M3) go(zero, std::integral_constant<int, REFLEX_PAGE_E4M3>{});
        else go(zero, std::integral_constant<int, REFLEX_PAGE_INT8>{});
    };
    if (dtype == REFLEX_DTYPE_F32) fmt(float{}); else fmt(__nv_bfloat16{});
    return cudaGetLastError();
}

}  // namespace reflex
