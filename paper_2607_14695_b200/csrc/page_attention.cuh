// Shared by the attention kernels over pages: sequences and their masks, the line of work that CTAs share, partial results.
#pragma once

#include "pages.cuh"

namespace reflex {

struct PageSeq { int b, row0, n, len; };      // first row of its new tokens, how many, tokens in all

// (whatever the device arrays hold, rows stay inside [0, n_rows))
__device__ __forceinline__ PageSeq page_seq(const PageAttention &p, int b)
{
    PageSeq s;
    s.b = b;
    const int c0 = p.q.cu[b], c1 = p.q.cu[b + 1];
    s.row0 = min(max(c0, 0), p.n_rows);
    s.n = max(0, min(c1, p.n_rows) - s.row0);
    s.len = max(0, p.q.len[b]);
    return s;
}

// positions that new tokens [t0, t1] of a sequence see between them
struct PageRange { int lo, hi; };
__device__ __forceinline__ PageRange page_range(const PageSeq &s, const PageAttention &p, int t0, int t1)
{
    const int p0 = s.len - s.n + t0, p1 = s.len - s.n + t1;
    PageRange r;
    r.hi = p.causal ? max(0, min(s.len, p1 + 1)) : s.len;
    r.lo = p.window > 0 ? max(0, p0 - p.window + 1) : 0;      // (p0 >= -n: no underflow)
    return r;
}

// CTA c of nc works on [page_share(c), page_share(c + 1)) of a line of `total` blocks
__host__ __device__ inline long long page_share(long long c, long long total, int nc) { return c * total / nc; }

// Partial results. A CTA (or pair) leaves at most two: slot 2c of the unit that it entered in the middle, slot 2c + 1 of the unit that it
// began and did not finish. meta[c] of the latter: {first row of the sequence, first (token, head) row of the tile, rows | KV head << 16, last CTA on the unit},
// -1 first where there is none.
struct PagePartials {
    float *o;              // [2 CTAs][rows][d]
    float2 *ml;            // [2 CTAs][rows]: maximum in log2 units, sum
    int4 *meta;            // [CTAs]
    int rows;              // rows of a slot
    float scale_log2;
};

int page_token_ctas(int sm_count);
int page_token_rows(int dtype, int format, int d, int rows);
cudaError_t launch_page_token(const PageAttention &a, const PagePartials &part, int format, int rows, int ctas, cudaStream_t st);
cudaError_t launch_page_merge(const PageAttention &a, const PagePartials &part, int ctas, cudaStream_t st);

}  // namespace reflex
