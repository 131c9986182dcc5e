// Attention of few new tokens per sequence over pages (reflex_pages_attention): one token of each stream, or a handful.
//
// Bound by memory: the keys and values of a (sequence, KV head) are read once for its G query heads and a tile of 8 or 16 rows (token, head).
// Nothing is staged in shared memory: a thread asks for 16-byte pieces of the rows in the pages, and what it gets are its operands of
// mma.m16n8k16 as they lie there, because the order of the contraction is free. With g = lane / 4 and t = lane % 4:
//   S^T = K Q^T, 16 keys by 8 query rows: thread (g, t) takes pieces of keys g and g + 8; four consecutive elements of the pieces of t = 0 .. 3 are the
//     16 of one step over head_dim (two of a thread's for the lower half of the step, two for the upper), and Q is put down in that order;
//   O^T = V^T P^T: thread (g, t) takes the same columns, chosen by g, of keys 2t, 2t + 1, 2t + 8, 2t + 9; a pair of keys in a register is one byte
//     permutation, and in 8-bit formats the one that unpacks them anyway. P^T comes out of S^T's accumulators by movmatrix.
// 8-bit rows stay unscaled in the products (they are exact in bf16): 2^e of a key scales its logits, 2^e of a value the key's weight, in fp32.
// A warp walks every fourth block of 16 keys with a running maximum; K of the next block is asked for as soon as this one's logits exist, V
// as soon as its products are issued, so that 6 KB or more per warp are on their way all the time.
//
// The keys of all (sequence, row tile, KV head) units form one line that the CTAs share evenly, whatever the lengths; a unit that more than one
// CTA works on leaves fp32 partials, which page_merge_kernel joins in the order of the keys (results do not depend on timing).
#include <math.h>

#include "page_attention.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

using namespace ptx;

constexpr int kTokWarps = 4;
constexpr int kTokBlock = 16 * kTokWarps;      // keys of a block: what the line of work is counted in

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint4 load_piece(const uint8_t *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 load_half_piece(const uint8_t *p)
{
    uint2 v;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}

template <int FMT, int HD, int NT> struct Tok {
    static constexpr bool BYTES = FMT != REFLEX_PAGE_SAME;
    static constexpr int ROW = HD * (BYTES ? 1 : 2);               // bytes of a row
    static constexpr int STEPS = HD / 16;                          // steps over head_dim
    static constexpr int KP = ROW / 64;                            // 16-byte pieces of a key per thread
    static constexpr int KEPP = BYTES ? 16 : 8;                    // elements of a piece of K
    static constexpr int VB = ROW / 8;                             // bytes of a value row per thread: 8, 16, 32, 64
    static constexpr int VW = VB / 4;                              // ... in words
    static constexpr int VCOLS = VB < 16 ? 8 : BYTES ? 16 : 8;     // consecutive columns of a thread
    static constexpr int VPIECES = HD / 8 / VCOLS;
    static constexpr int ROWS = 8 * NT;
    static constexpr int OSTRIDE = HD + 4;                         // floats of a row of O in shared memory
    static constexpr uint32_t OFF_O = 0;                           // [warps][ROWS][OSTRIDE]
    static constexpr uint32_t OFF_Q = OFF_O + kTokWarps * ROWS * OSTRIDE * 4;      // [step][NT][lane] of two registers
    static constexpr uint32_t OFF_ML = OFF_Q + STEPS * NT * 256;   // [warps][ROWS] of (maximum, sum)
    static constexpr uint32_t SMEM = OFF_ML + kTokWarps * ROWS * 8;
};

// the blocks of keys that a tile of ROWS rows needs
struct TokSpan { int lo, hi, count; };
template <int ROWS>
struct TokSpanOf {
    const PageAttention &p;
    int G;
    __device__ __forceinline__ int tiles(const PageSeq &s) const { return (s.n * G + ROWS - 1) / ROWS; }
    __device__ __forceinline__ TokSpan operator()(const PageSeq &s, int tile) const
    {
        const PageRange r = page_range(s, p, tile * ROWS / G, (min(s.n * G, (tile + 1) * ROWS) - 1) / G);
        TokSpan t;
        t.lo = r.lo & ~15;
        t.hi = r.hi;
        t.count = t.hi > t.lo ? (t.hi - t.lo + kTokBlock - 1) / kTokBlock : 0;
        return t;
    }
};

template <int FMT, int HD, int NT>
__global__ void __launch_bounds__(32 * kTokWarps, 2)
page_token_kernel(const PageAttention p, const PagePartials part)
{
    using C = Tok<FMT, HD, NT>;
    constexpr int ROWS = C::ROWS;
    extern __shared__ __align__(16) uint8_t smem[];
    float *o_s = reinterpret_cast<float *>(smem + C::OFF_O);
    uint2 *q_s = reinterpret_cast<uint2 *>(smem + C::OFF_Q);
    float2 *ml_s = reinterpret_cast<float2 *>(smem + C::OFF_ML);
    const PageGeom &g = p.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, t4 = lane & 3;
    const int G = g.Hq / g.Hkv;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    PageLine<TokSpanOf<ROWS>> line{p, {p, G}};
    const int total = line.begin(lane);
    // No more CTAs than leave each the square root of a tenth of the longest unit: a partial costs the merge a tenth of what a block costs here.
    const int least = max(1, (int)sqrtf((float)line.longest * 0.1f));
    const int nc = min((int)gridDim.x, (total + least - 1) / least);
    const int cta = blockIdx.x;
    if (threadIdx.x == 0) part.meta[cta].b = -1;
    if (cta >= nc) return;
    const PageShares shares(total, nc);
    const int x0 = shares.of(cta), x1 = shares.of(cta + 1);
    auto u = line.find(x0, lane);

    for (int x = x0; x < x1;) {
        const PageSeq s = u.s;
        const TokSpan span = u.sp;
        const int rt = u.tile, h = u.h, b = s.b;
        const int k0 = x - u.at, k1 = min(u.cost, x1 - u.at);
        const int kend = min(k1, span.count);
        // ---- Q of the unit's rows, in the order of K's pieces ----
        __syncthreads();             // (the last unit's results and Q have been read)
        for (int i = threadIdx.x; i < C::STEPS * NT * 32; i += 32 * kTokWarps) {
            const int ln = i & 31, nt = (i >> 5) % NT, step = (i >> 5) / NT;
            const int r = rt * ROWS + nt * 8 + (ln >> 2);
            const int d0 = (C::BYTES ? 64 * (step >> 2) + 16 * (ln & 3) + 4 * (step & 3) : 32 * (step >> 1) + 8 * (ln & 3) + 4 * (step & 1));
            uint2 v = make_uint2(0u, 0u);
            if (r < s.n * G) v = *reinterpret_cast<const uint2 *>((const __nv_bfloat16 *)p.qry + ((size_t)(s.row0 + r / G) * g.Hq + h * G + r % G) * HD + d0);
            q_s[i] = v;
        }
        __syncthreads();

        // ---- this thread's query rows: 2t, 2t + 1 of every group of 8 ----
        int lo_r[2 * NT], hi_r[2 * NT], lo_min, lo_max, hi_min, hi_max;      // (the limits of all the tile's rows)
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            const int r = min(rt * ROWS + (i >> 1) * 8 + 2 * t4 + (i & 1), s.n * G - 1);
            const PageRange v = page_range(s, p, r / G, r / G);
            lo_r[i] = v.lo; hi_r[i] = v.hi;
        }
        {
            const int t_last = (min((rt + 1) * ROWS, s.n * G) - 1) / G;
            const PageRange first = page_range(s, p, rt * ROWS / G, rt * ROWS / G), last = page_range(s, p, t_last, t_last);
            lo_min = first.lo; hi_min = first.hi; lo_max = last.lo; hi_max = last.hi;
        }

        float o[HD / 16][NT][4];
        float m[2 * NT], l[2 * NT];
#pragma unroll
        for (int i = 0; i < HD / 16; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
        bool bad = false;

        const int key0 = span.lo + warp * 16;        // keys of block i: key0 + 64 i ..
        uint4 kr[2][C::KP];
        uint32_t vr[4][C::VW];
        int ke[2] = {127, 127}, ve[2] = {127, 127};
        int page_ids = -1, ids_from = k0;
        auto page_of_block = [&](int i) -> int {      // (the pages of 32 blocks are looked up together)
            if (i == k0 || i - ids_from >= 32) {
                ids_from = i;
                const int mine = i + lane;
                page_ids = mine < kend ? page_at(p.q, g.n_pages, b, (key0 + mine * kTokBlock) >> g.log_p) : -1;
            }
            return __shfl_sync(0xffffffffu, page_ids, i - ids_from);
        };
        auto row_of = [&](int page, int key) -> size_t { return page_row(g, page, h) + (size_t)(key & (g.P - 1)); };
        auto load_k = [&](size_t row) {
            const uint8_t *base = (const uint8_t *)g.k + row * C::ROW + t4 * 16;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int j = 0; j < C::KP; ++j) kr[e][j] = load_piece(base + (size_t)(gq + 8 * e) * C::ROW + j * 64);
            if constexpr (C::BYTES) { ke[0] = g.ke[row + gq]; ke[1] = g.ke[row + gq + 8]; }
        };
        auto load_v = [&](size_t row) {
            const uint8_t *base = (const uint8_t *)g.v + row * C::ROW + gq * (C::VB < 16 ? 8 : 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint8_t *r = base + (size_t)(2 * t4 + (e & 1) + 8 * (e >> 1)) * C::ROW;
                if constexpr (C::VB < 16) {
                    const uint2 v = load_half_piece(r);
                    vr[e][0] = v.x; vr[e][1] = v.y;
                } else {
#pragma unroll
                    for (int j = 0; j < C::VB / 16; ++j) {
                        const uint4 v = load_piece(r + j * 128);
                        vr[e][4 * j] = v.x; vr[e][4 * j + 1] = v.y; vr[e][4 * j + 2] = v.z; vr[e][4 * j + 3] = v.w;
                    }
                }
            }
            if constexpr (C::BYTES) { ve[0] = g.ve[row + gq]; ve[1] = g.ve[row + gq + 8]; }
        };
        // O^T += V^T P^T of the loaded block; keep: which of this thread's four keys are live (the others count as zeros)
        auto times_v = [&](const uint32_t (&pt)[NT][2], uint32_t keep) {
#pragma unroll
            for (int i = 0; i < C::VW; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (keep >> e) & 1u ? vr[e][i] : 0u;
                if constexpr (C::BYTES) {
                    // four columns of four keys: two tiles of 16 (column, column + 1) pairs
                    const uint32_t a[8] = {bytes_to_bf16x2<FMT, 0, 0>(w[0], w[1]), bytes_to_bf16x2<FMT, 1, 1>(w[0], w[1]), bytes_to_bf16x2<FMT, 0, 0>(w[2], w[3]), bytes_to_bf16x2<FMT, 1, 1>(w[2], w[3]),
                                           bytes_to_bf16x2<FMT, 2, 2>(w[0], w[1]), bytes_to_bf16x2<FMT, 3, 3>(w[0], w[1]), bytes_to_bf16x2<FMT, 2, 2>(w[2], w[3]), bytes_to_bf16x2<FMT, 3, 3>(w[2], w[3])};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_bf16(o[2 * i][nt], a[0], a[1], a[2], a[3], pt[nt][0], pt[nt][1]);
                        mma_bf16(o[2 * i + 1][nt], a[4], a[5], a[6], a[7], pt[nt][0], pt[nt][1]);
                    }
                } else {
                    const uint32_t a0 = __byte_perm(w[0], w[1], 0x5410), a1 = __byte_perm(w[0], w[1], 0x7632), a2 = __byte_perm(w[2], w[3], 0x5410), a3 = __byte_perm(w[2], w[3], 0x7632);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_bf16(o[i][nt], a0, a1, a2, a3, pt[nt][0], pt[nt][1]);
                }
            }
        };

        size_t row = 0;
        int page = -1;
        if (k0 < kend) {
            page = page_of_block(k0);
            bad |= page < 0 && key0 + k0 * kTokBlock < span.hi;
            row = row_of(max(page, 0), key0 + k0 * kTokBlock);
            load_k(row);
            load_v(row);
        }
        for (int i = k0; i < kend; ++i) {
            const int key = key0 + i * kTokBlock;
            const bool more = i + 1 < kend;
            const int page_next = more ? page_of_block(i + 1) : -1;
            const size_t row_next = more ? row_of(max(page_next, 0), key + kTokBlock) : 0;
            // ---- logits ----
            float c[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[nt][0][e] = c[nt][1][e] = 0.f;
#pragma unroll
            for (int step = 0; step < C::STEPS; ++step) {
                uint32_t a0, a1, a2, a3;
                if constexpr (C::BYTES) {
                    const uint32_t w0 = (&kr[0][step >> 2].x)[step & 3], w1 = (&kr[1][step >> 2].x)[step & 3];
                    a0 = bytes_to_bf16x2<FMT, 0, 1>(w0, w0); a1 = bytes_to_bf16x2<FMT, 0, 1>(w1, w1);
                    a2 = bytes_to_bf16x2<FMT, 2, 3>(w0, w0); a3 = bytes_to_bf16x2<FMT, 2, 3>(w1, w1);
                } else {
                    a0 = (&kr[0][step >> 1].x)[2 * (step & 1)]; a1 = (&kr[1][step >> 1].x)[2 * (step & 1)];
                    a2 = (&kr[0][step >> 1].x)[2 * (step & 1) + 1]; a3 = (&kr[1][step >> 1].x)[2 * (step & 1) + 1];
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint2 q = q_s[(step * NT + nt) * 32 + lane];
                    mma_bf16(c[nt][step & 1], a0, a1, a2, a3, q.x, q.y);
                }
            }
            const float ks0 = C::BYTES ? exponent_f32(ke[0]) * part.scale_log2 : part.scale_log2, ks1 = C::BYTES ? exponent_f32(ke[1]) * part.scale_log2 : part.scale_log2;
            if (more) load_k(row_next);
            // ---- masks, running maximum, weights ----
            const bool whole = key >= lo_max && key + 16 <= hi_min && page >= 0;
            float w[NT][4];            // (key g, row 2t), (g, 2t + 1), (g + 8, 2t), (g + 8, 2t + 1)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[nt][e] = (c[nt][0][e] + c[nt][1][e]) * (e < 2 ? ks0 : ks1);
                    if (!whole) {
                        const int j = key + gq + (e < 2 ? 0 : 8);
                        if (j < lo_r[2 * nt + (e & 1)] || j >= hi_r[2 * nt + (e & 1)] || page < 0) w[nt][e] = -INFINITY;
                    }
                }
            bool grows = false;
            float top[2 * NT];
#pragma unroll
            for (int r = 0; r < 2 * NT; ++r) {
                top[r] = fmaxf(w[r >> 1][r & 1], w[r >> 1][2 + (r & 1)]);
#pragma unroll
                for (int x2 = 4; x2 < 32; x2 <<= 1) top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], x2));
                grows |= top[r] > m[r] + 8.f || (m[r] == -INFINITY && top[r] > -INFINITY);
            }
            if (__any_sync(0xffffffffu, grows)) {
                // O and the sums are brought to a new reference only where a maximum has grown by more than 2^8 (all lanes of a row alike)
#pragma unroll
                for (int r = 0; r < 2 * NT; ++r) {
                    const float to = fmaxf(m[r], top[r]);
                    const float f = m[r] == -INFINITY ? 0.f : ex2(m[r] - to);
                    m[r] = to;
                    l[r] *= f;
#pragma unroll
                    for (int q = 0; q < HD / 16; ++q) { o[q][r >> 1][r & 1] *= f; o[q][r >> 1][2 + (r & 1)] *= f; }
                }
            }
            uint32_t pt[NT][2];
            const float vs0 = C::BYTES ? exponent_f32(ve[0]) : 1.f, vs1 = C::BYTES ? exponent_f32(ve[1]) : 1.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x2 = w[nt][e], mr = m[2 * nt + (e & 1)];
                    const float pe = ex2(x2 - (mr == -INFINITY ? 0.f : mr));
                    l[2 * nt + (e & 1)] += pe;
                    v[e] = !whole && x2 == -INFINITY ? 0.f : C::BYTES ? pe * (e < 2 ? vs0 : vs1) : pe;
                }
                pt[nt][0] = transpose8x8(pack_bf16(v[0], v[1]));
                pt[nt][1] = transpose8x8(pack_bf16(v[2], v[3]));
            }
            // ---- values ----
            if (whole || C::BYTES) times_v(pt, 15u);
            else {
                // A masked key has weight 0, but 0 times what lies there may be NaN: keys that no row sees count as zeros. A key that some
                // rows see is multiplied for all of them, which does no harm while it is finite.
                uint32_t live = 0;
                bool odd = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = key + 2 * t4 + (e & 1) + 8 * (e >> 1);
                    if (j >= lo_min && j < hi_max && page >= 0) {
                        live |= 1u << e;
#pragma unroll
                        for (int q = 0; q < C::VW; ++q) odd |= (vr[e][q] & 0x7f80u) == 0x7f80u || (vr[e][q] & 0x7f800000u) == 0x7f800000u;
                    }
                }
                if (__any_sync(0xffffffffu, odd)) {
                    // what is not finite goes, as it is, to the rows that see it (whatever their weight), and counts as zero in the products
#pragma unroll 1
                    for (int from = 0; from < 4; ++from) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int j = key + 2 * from + (e & 1) + 8 * (e >> 1);
#pragma unroll
                            for (int i2 = 0; i2 < C::VW; ++i2) {
                                const uint32_t v = __shfl_sync(0xffffffffu, vr[e][i2], (lane & ~3) | from);
#pragma unroll
                                for (int half = 0; half < 2; ++half) {
                                    const uint32_t bits = half ? v & 0xffff0000u : v << 16;
                                    if ((bits & 0x7f800000u) != 0x7f800000u) continue;
#pragma unroll
                                    for (int r = 0; r < 2 * NT; ++r)
                                        if (j >= lo_r[r] && j < hi_r[r]) o[i2 < HD / 16 ? i2 : 0][r >> 1][2 * half + (r & 1)] += __uint_as_float(bits);
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int q = 0; q < C::VW; ++q) {
                            if ((vr[e][q] & 0x7f80u) == 0x7f80u) vr[e][q] &= 0xffff0000u;
                            if ((vr[e][q] & 0x7f800000u) == 0x7f800000u) vr[e][q] &= 0x0000ffffu;
                        }
                }
                times_v(pt, live);
            }
            if (more) {
                load_v(row_next);
                bad |= page_next < 0 && key + kTokBlock < span.hi;
            }
            page = page_next;
        }
        // ---- the warps' shares meet ----
        const bool any_bad = __any_sync(0xffffffffu, bad);
        if (any_bad && lane == 0) report_bad_page(g.status, b);
#pragma unroll
        for (int r = 0; r < 2 * NT; ++r) {
#pragma unroll
            for (int x2 = 4; x2 < 32; x2 <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x2);
            if (any_bad) l[r] = __int_as_float(0x7fc00000);
            if (gq == 0) ml_s[warp * ROWS + (r >> 1) * 8 + 2 * t4 + (r & 1)] = make_float2(m[r], l[r]);
        }
        __syncthreads();
        float f[2 * NT];
#pragma unroll
        for (int r = 0; r < 2 * NT; ++r) {
            const int rr = (r >> 1) * 8 + 2 * t4 + (r & 1);
            float all = -INFINITY;
#pragma unroll
            for (int q = 0; q < kTokWarps; ++q) all = fmaxf(all, ml_s[q * ROWS + rr].x);
            f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - all);
            // column c of piece j: 8 VCOLS j + VCOLS g + c; register (tile, 0 / 2) holds an even / odd column of an even row's pair
            float *dst = o_s + (warp * ROWS + rr) * C::OSTRIDE + gq * C::VCOLS;
#pragma unroll
            for (int j = 0; j < C::VPIECES; ++j)
#pragma unroll
                for (int x2 = 0; x2 < C::VCOLS; x2 += 4) {
                    const int tile = (j * C::VCOLS + x2) / 2;
                    *reinterpret_cast<float4 *>(dst + j * 8 * C::VCOLS + x2) = make_float4(o[tile][r >> 1][r & 1] * f[r], o[tile][r >> 1][2 + (r & 1)] * f[r],
                                                                                         o[tile + 1][r >> 1][r & 1] * f[r], o[tile + 1][r >> 1][2 + (r & 1)] * f[r]);
                }
        }
        __syncthreads();
        const bool starts = k0 == 0, ends = k1 == u.cost;
        const int slot = 2 * cta + (starts ? 1 : 0);
        for (int i = threadIdx.x; i < ROWS * (HD / 8); i += 32 * kTokWarps) {
            const int r = i / (HD / 8), c0 = i % (HD / 8) * 8;
            const int rr = rt * ROWS + r;
            if (rr >= s.n * G) continue;
            float all = -INFINITY, sum = 0.f, acc[8];
#pragma unroll
            for (int q = 0; q < kTokWarps; ++q) all = fmaxf(all, ml_s[q * ROWS + r].x);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
            for (int q = 0; q < kTokWarps; ++q) {
                const float2 v = ml_s[q * ROWS + r];
                // (a maximum of -inf carries no weight, a sum that is NaN is kept)
                sum += v.x == -INFINITY ? v.y * 0.f : v.y * ex2(v.x - all);
                const float4 *src = reinterpret_cast<const float4 *>(o_s + (q * ROWS + r) * C::OSTRIDE + c0);
                const float4 y0 = src[0], y1 = src[1];
                acc[0] += y0.x; acc[1] += y0.y; acc[2] += y0.z; acc[3] += y0.w;
                acc[4] += y1.x; acc[5] += y1.y; acc[6] += y1.z; acc[7] += y1.w;
            }
            if (starts && ends) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] *= inv;
                store8((__nv_bfloat16 *)p.out + ((size_t)(s.row0 + rr / G) * g.Hq + h * G + rr % G) * HD + c0, acc);
            } else {
                store8(partial8(part, slot, HD, r, c0), acc);
                if (c0 == 0) part.ml[(size_t)slot * part.rows + r] = make_float2(all, sum);
            }
        }
        if (starts && !ends && threadIdx.x == 0) {
            PageSplit m2 = {b, s.row0, rt * ROWS, min(ROWS, s.n * G - rt * ROWS), h, shares.owner(u.at + u.cost - 1), ROWS, 0};
            part.meta[cta] = m2;
        }
        x = u.at + k1;
        if (ends) line.next(u);
    }
}

template <int FMT, int HD, int NT>
static cudaError_t launch_token(const PageAttention &a, const PagePartials &part, int ctas, cudaStream_t st)
{
    using C = Tok<FMT, HD, NT>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = once_per_device(done, [] { return cudaFuncSetAttribute(page_token_kernel<FMT, HD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM); });
    if (e != cudaSuccess) return e;
    count_launch();
    page_token_kernel<FMT, HD, NT><<<ctas, 32 * kTokWarps, C::SMEM, st>>>(a, part);
    return cudaGetLastError();
}

int page_token_ctas(int sm_count) { return 2 * sm_count; }

// Rows of a tile for `rows` (token, head) rows per sequence and KV head on average; 0: not for this kernel.
int page_token_rows(int dtype, int format, int d, int G, int rows)
{
    if (dtype != REFLEX_DTYPE_BF16 || d < 64) return 0;
    const bool wide = format == REFLEX_PAGE_SAME && d == 256;         // (16 rows of bf16 rows of 256 do not fit the registers)
    if (rows > (format == REFLEX_PAGE_SAME ? 16 : 64) && page_chunk_takes(dtype, G, d)) return 0;
    return rows <= 8 || wide ? 8 : 16;
}

cudaError_t launch_page_token(const PageAttention &a, const PagePartials &part, int format, int rows, int ctas, cudaStream_t st)
{
    auto go = [&](auto f, auto hd) -> cudaError_t {
        constexpr int FMT = decltype(f)::value, HD = decltype(hd)::value;
        if constexpr (!(FMT == REFLEX_PAGE_SAME && HD == 256))
            if (rows == 16) return launch_token<FMT, HD, 2>(a, part, ctas, st);
        return launch_token<FMT, HD, 1>(a, part, ctas, st);
    };
    auto by_d = [&](auto f) -> cudaError_t {
        if (a.g.d == 64) return go(f, std::integral_constant<int, 64>{});
        if (a.g.d == 128) return go(f, std::integral_constant<int, 128>{});
        return go(f, std::integral_constant<int, 256>{});
    };
    return format == REFLEX_PAGE_SAME ? by_d(std::integral_constant<int, REFLEX_PAGE_SAME>{})
           : format == REFLEX_PAGE_E4M3 ? by_d(std::integral_constant<int, REFLEX_PAGE_E4M3>{}) : by_d(std::integral_constant<int, REFLEX_PAGE_INT8>{});
}

}  // namespace reflex
