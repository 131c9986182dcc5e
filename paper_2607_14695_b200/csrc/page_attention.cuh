// Shared by the attention kernels over pages: sequences and their masks, the line of work that CTAs share, partial results.
#pragma once

#include "pages.cuh"

namespace reflex {

__device__ __forceinline__ void report_page_wait(uint32_t *status, uint32_t site) { atomicCAS(status, 0u, status_word(site)); }

// Weights are 2^-24 of what the softmax has them, in sums and in products alike, so that it goes with the division: O is a sum over the keys of weights,
// which reach 2^8 between two changes of the reference, times values, which reach 2^127 and more, and is not to pass fp32 ahead of the division (nor a
// weight times a value's 2^e bf16). That holds for 2^15 such keys. Down below, values of 2^-100 are still normal numbers as products. (The tensor-core
// kernels round them to bf16 for the product with V, the one form that its operands have there; the sum takes them as they are. Against 64 bits the
// result's error goes from 0.0017 of its size, which is its own rounding to bf16, to 0.0023.)
constexpr float kWeightShift = 24.f;

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
    r.lo = p.window > 0 && p0 >= p.window ? p0 - p.window + 1 : 0;      // (p0 may be negative, and the window as large as there is)
    // (of positions past the table the first one is looked at, and reported, however far a length goes)
    const int cap = p.q.max_pages << p.g.log_p;
    r.hi = min(r.hi, cap + 1);
    r.lo = min(r.lo, cap);
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
// A warp works on 32 sequences at a time; with fewer, `width` lanes share one. The first 32 (or all) are kept in registers.
template <typename SPAN>
struct PageLine {
    const PageAttention &p;
    SPAN span;
    int width, longest;              // lanes of a sequence; the longest unit
    PageSeq mine;                    // sequence lane / width
    int mine_cost;                   // its blocks, in the first of its lanes (0 in the others)

    // blocks of the sequence that `width` lanes hold, in the first of them
    __device__ __forceinline__ int seq_cost(const PageSeq &s, int lane, int &longest_) const
    {
        int cost = 0;
        const int n = span.tiles(s);
        for (int t = lane & (width - 1); t < n; t += width) {
            const int c = max(1, span(s, t).count);
            cost += c;
            longest_ = max(longest_, c);
        }
        for (int o = 1; o < width; o <<= 1) cost += __shfl_xor_sync(0xffffffffu, cost, o);
        return (lane & (width - 1)) == 0 ? cost * p.g.Hkv : 0;
    }
    __device__ __forceinline__ PageSeq seq_of(int b) const
    {
        PageSeq s = {b, 0, 0, 0};
        if (b < p.q.B) s = page_seq(p, b);
        return s;
    }
    // the length of the line
    __device__ __forceinline__ int begin(int lane)
    {
        width = 32;
        while (width > 1 && p.q.B * width > 32) width >>= 1;
        mine = seq_of(lane / width);
        return count(lane);
    }
    // (again, when `span` counts otherwise)
    __device__ __forceinline__ int count(int lane)
    {
        longest = 1;
        mine_cost = seq_cost(mine, lane, longest);
        int sum = mine_cost;
        for (int b0 = 32; b0 < p.q.B; b0 += 32) sum += seq_cost(seq_of(b0 + lane), lane, longest);
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
    // the unit that block x (< the line's length) belongs to
    __device__ __forceinline__ Place find(int x, int lane) const
    {
        Place u;
        u.at = 0;
        PageSeq s = mine;
        int cost = mine_cost, unused = 0;
        if (p.q.B == 1) u.s = {0, __shfl_sync(0xffffffffu, s.row0, 0), __shfl_sync(0xffffffffu, s.n, 0), __shfl_sync(0xffffffffu, s.len, 0)};
        else for (int b0 = 0;;) {
            const int incl = scan(cost, lane);
            const uint32_t past = __ballot_sync(0xffffffffu, u.at + incl > x);
            if (past || b0 + 32 >= p.q.B) {
                const int src = past ? __ffs(past) - 1 : 0;          // (the first lane of its sequence's)
                u.at += __shfl_sync(0xffffffffu, incl - cost, src);
                u.s.b = __shfl_sync(0xffffffffu, s.b, src);
                u.s.row0 = __shfl_sync(0xffffffffu, s.row0, src);
                u.s.n = __shfl_sync(0xffffffffu, s.n, src);
                u.s.len = __shfl_sync(0xffffffffu, s.len, src);
                break;
            }
            u.at += __shfl_sync(0xffffffffu, incl, 31);
            b0 += 32;
            s = seq_of(b0 + lane);
            cost = seq_cost(s, lane, unused);
        }
        u.tiles = span.tiles(u.s);
        u.tile = 0;
        for (int t0 = 0; u.tiles > 1 && t0 < u.tiles; t0 += 32) {
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
    uint32_t *arrived;     // [CTAs]: how many CTAs have left their partial of the unit that this one began (page_token_kernel; zero between launches)
    int rows;              // rows of a slot
    float scale_log2;
};
__device__ __forceinline__ float *partial8(const PagePartials &part, size_t slot, int d, int r, int c0) { return part.o + ((slot * (size_t)(d >> 3) + (size_t)(c0 >> 3)) * part.rows + r) * 8; }
constexpr int kTokenCtas = 160, kMostPairs = 128;      // of page_token_kernel's CTAs, of page_chunk_kernel's pairs
int page_token_rows(int dtype, int format, int d, int G, int rows);
cudaError_t launch_page_token(const PageAttention &a, const PagePartials &part, int format, int rows, int sm_count, cudaStream_t st);
bool page_chunk_takes(int dtype, int G, int d);
cudaError_t launch_page_widen(const PageAttention &a, void *k_wide, void *v_wide, int format, int sm_count, cudaStream_t st);
// k, v: one layer's pages in bf16
cudaError_t launch_page_chunk(const PageAttention &a, const PagePartials &part, const void *k, const void *v, int pairs, cudaStream_t st);
cudaError_t launch_page_merge(const PageAttention &a, const PagePartials &part, int pairs, int format, int sm_count, cudaStream_t st);

}  // namespace reflex
