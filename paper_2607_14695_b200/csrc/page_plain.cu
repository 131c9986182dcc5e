// Attention over pages, plain form (page_plain.cuh): a warp per (token, query head). Serves fp32, heads of 32 and groups of more than 128 heads.
#include "page_plain.cuh"

namespace reflex {

constexpr int kPlainWarps = 4;

template <typename T, int FMT>
__global__ void __launch_bounds__(32 * kPlainWarps)
page_plain_kernel(const PageAttention p)
{
    extern __shared__ int cu_s[];
    __shared__ __align__(16) float q_s[kPlainWarps][256];
    load_cu(p.q, cu_s);
    __syncthreads();
    const int warp = threadIdx.x >> 5;
    const int64_t item = (int64_t)blockIdx.x * kPlainWarps + warp;
    const int64_t row = item / p.g.Hq;
    if (row >= p.n_rows || row >= cu_s[p.q.B] || row < cu_s[0]) return;
    const int b = find_seq(cu_s, p.q.B, (int)row), len = p.q.len[b];
    page_plain_row<T, FMT>(p, b, (int)row, (int64_t)len - cu_s[b + 1] + row, len, (int)(item % p.g.Hq), q_s[warp]);
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
