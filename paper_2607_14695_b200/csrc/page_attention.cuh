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

// ---- the line of work ----
// A unit is a tile of consecutive (token, head of the group) rows of a sequence and a KV head; it costs what SPAN says of its tile, in blocks of
// keys, and one at least (rows that see nothing have to be written too). Units stand in a line by sequence, tile and KV head, and
// CTA c of nc works on blocks [of(c), of(c + 1)) of it, whatever the lengths are. (32 bits: the host refuses calls whose line could be longer.)
struct PageShares {
    int each, more;          // `more` CTAs have each + 1 blocks, the others `each`
    __device__ __forceinline__ PageShares(int total, int nc) : each(total / nc), more(total % nc) {}
    __device__ __forceinline__ int of(int c) const { return c * each + min(c, more); }
    // the CTA that works on block x
    __device__ __forceinline__ int owner(int x) const
    {
        const int longer = more * (each + 1);
        return x < longer ? x / (each + 1) : more + (x - longer) / each;
    }
};

// SPAN: tiles(s) of a sequence; (s, tile) gives a struct with .count (blocks). Functions that take `lane`: whole warps, all lanes get the same.
template <typename SPAN>
struct PageLine {
    const PageAttention &p;
    const SPAN span;

    // With few sequences several lanes share one: width() of them.
    __device__ __forceinline__ int width() const
    {
        int w = 32;
        while (w > 1 && p.q.B * w > 32) w >>= 1;
        return w;
    }
    // the blocks of sequence b0 + lane / w (0 behind the last one), in all its w lanes
    __device__ __forceinline__ int seq_cost(int b0, int w, int lane, int &longest) const
    {
        int cost = 0;
        if (b0 + lane / w < p.q.B) {
            const PageSeq s = page_seq(p, b0 + lane / w);
            const int n = span.tiles(s);
            for (int t = lane & (w - 1); t < n; t += w) {
                const int c = max(1, span(s, t).count);
                cost += c;
                longest = max(longest, c);
            }
        }
        for (int o = 1; o < w; o <<= 1) cost += __shfl_xor_sync(0xffffffffu, cost, o);
        return cost * p.g.Hkv;
    }
    __device__ __forceinline__ int total(int lane, int &longest) const
    {
        const int w = width();
        int sum = 0;
        longest = 1;
        for (int b0 = 0; b0 < p.q.B; b0 += 32 / w) {
            const int c = seq_cost(b0, w, lane, longest);
            sum += (lane & (w - 1)) == 0 ? c : 0;
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
        return __reduce_add_sync(0xffffffffu, sum);
    }

    // ---- a place in the line: unit (s, tile, h) begins at block `at` ----
    struct Place {
        PageSeq s;
        int tiles, tile, h, cost, at;
        decltype(span(PageSeq(), 0)) sp;
    };
    static __device__ __forceinline__ int scan(int c, int lane)
    {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, c, o);
            if (lane >= o) c += y;
        }
        return c;
    }
    // the unit that block x (< total) belongs to
    __device__ __forceinline__ Place find(int x, int lane) const
    {
        Place u;
        const int w = width();
        int unused = 0, b = 0;
        u.at = 0;
        for (int b0 = 0; b0 < p.q.B; b0 += 32 / w) {
            const int c = (lane & (w - 1)) == 0 || w == 1 ? 1 : 0, cost = seq_cost(b0, w, lane, unused) * c;
            const int incl = scan(cost, lane);
            const uint32_t past = __ballot_sync(0xffffffffu, u.at + incl > x);
            if (past) {
                const int src = __ffs(past) - 1;          // (the first lane of its sequence's)
                b = b0 + src / w;
                u.at += __shfl_sync(0xffffffffu, incl - cost, src);
                break;
            }
            u.at += __shfl_sync(0xffffffffu, incl, 31);
        }
        u.s = page_seq(p, b);
        u.tiles = span.tiles(u.s);
        u.tile = 0;
        for (int t0 = 0; t0 < u.tiles; t0 += 32) {
            const int c = t0 + lane < u.tiles ? max(1, span(u.s, t0 + lane).count) * p.g.Hkv : 0;
            const int incl = scan(c, lane);
            const uint32_t past = __ballot_sync(0xffffffffu, u.at + incl > x);
            if (past) {
                const int src = __ffs(past) - 1;
                u.tile = t0 + src;
                u.at += __shfl_sync(0xffffffffu, incl - c, src);
                break;
            }
            u.at += __shfl_sync(0xffffffffu, incl, 31);
        }
        u.sp = span(u.s, u.tile);
        u.cost = max(1, u.sp.count);
        u.h = p.g.Hkv == 1 ? 0 : (x - u.at) / u.cost;
        u.at += u.h * u.cost;
        return u;
    }
    // the unit behind u (callable by single lanes); behind the last one u.s.b is B
    __device__ __forceinline__ void next(Place &u) const
    {
        u.at += u.cost;
        if (++u.h < p.g.Hkv) return;
        u.h = 0;
        if (++u.tile >= u.tiles) {
            u.tile = 0;
            do {
                if (++u.s.b >= p.q.B) return;
                u.s = page_seq(p, u.s.b);
            } while (u.s.n == 0);
            u.tiles = span.tiles(u.s);
        }
        u.sp = span(u.s, u.tile);
        u.cost = max(1, u.sp.count);
    }
};

// ---- partial results ----
// A CTA (or pair) leaves at most two: slot 2c of the unit that it entered in the middle, slot 2c + 1 of the unit that it began and did not
// finish; the latter's entry in `meta` says what the unit is and which CTA is the last on it.
// (first: first (token, head) row of the tile, which lies in row 0 of the slot; rows from `half` on lie from row 128 on; b = -1: none)
struct PageSplit { int b, row0, first, rows, h, last, half, unused; };
struct PagePartials {
    float *o;              // [2 CTAs][d / 8][rows][8], unnormalised
    float2 *ml;            // [2 CTAs][rows]: maximum in log2 units, sum
    PageSplit *meta;       // [CTAs]
    // Sequences (a byte each) whose rows page_merge_kernel computes again one by one, since what lies at a key that some rows of a
    // tile see and others do not was not finite, and 0 times it is NaN on the tensor cores; and the blocks of that kernel that are done with them.
    uint8_t *careful;
    uint32_t *careful_done;
    int rows;              // rows of a slot
    float scale_log2;
};
__device__ __forceinline__ float *partial8(const PagePartials &part, size_t slot, int d, int r, int c0) { return part.o + ((slot * (size_t)(d >> 3) + (size_t)(c0 >> 3)) * part.rows + r) * 8; }
int page_token_ctas(int sm_count);
int page_token_rows(int dtype, int format, int d, int G, int rows);
cudaError_t launch_page_token(const PageAttention &a, const PagePartials &part, int format, int rows, int ctas, cudaStream_t st);
bool page_chunk_takes(int dtype, int G, int d);
cudaError_t launch_page_widen(const PageAttention &a, void *k_wide, void *v_wide, int format, int sm_count, cudaStream_t st);
// k, v: one layer's pages in bf16
cudaError_t launch_page_chunk(const PageAttention &a, const PagePartials &part, const void *k, const void *v, int pairs, cudaStream_t st);
cudaError_t launch_page_merge(const PageAttention &a, const PagePartials &part, int ctas, int format, int sm_count, cudaStream_t st);

}  // namespace reflex
