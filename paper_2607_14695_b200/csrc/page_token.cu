// Attention of few new tokens per sequence over pages (reflex_pages_attention): one token of each stream, or a handful.
//
// The keys and values of a (sequence, KV head) are read once for its G query heads and a tile of 8 or 16 rows (token, head).
// TMA brings 16 rows of keys and 16 of values in swizzled boxes, and a thread's 16-byte pieces of them are its operands of mma.m16n8k16 as they lie
// there, because the order of the contraction is free: no transposition, no bank conflict. With g = lane / 4 and t = lane % 4:
//   S^T = K Q^T, 16 keys by 8 query rows: thread (g, t) takes pieces of keys g and g + 8; four consecutive elements of the pieces of t = 0 .. 3 are the
//     16 of one step over head_dim (two of a thread's for the lower half of the step, two for the upper), and Q is put down in that order;
//   O^T = V^T P^T: thread (g, t) takes the same columns, chosen by g, of keys 2t, 2t + 1, 2t + 8, 2t + 9; a pair of keys in a register is one byte
//     permutation, and in 8-bit formats the one that unpacks them anyway. P^T comes out of S^T's accumulators by movmatrix.
// 8-bit rows stay unscaled in the products (they are exact in bf16): 2^e of a key scales its logits, 2^e of a value the key's weight, in fp32.
// A warp walks every WARPS-th block of 16 keys with a running maximum, fetches for itself, and has one or two blocks on their way while it works on one:
// 100 KB or more per SM. (64 streams of 3300 keys in 8 bits, 112 MB: 46.7 us with one block at a time in registers, 49.5 with rows by cp.async, whose
// 17 instructions a block kept the load pipe busy, 33.6 by TMA and with all that follows. That is twice the 17 that the bytes take: the schedulers issue 0.41
// instructions a cycle, and the largest stall is the block's barriers, three at the end of a unit, where all warps of the SM's one CTA stand.)
//
// The keys of all (sequence, row tile, KV head) units form one line that the CTAs share evenly, whatever the lengths; a unit that more than one
// CTA works on leaves fp32 partials, which the last of them to finish joins in the order of the keys (results do not depend on timing).
#include <math.h>

#include <algorithm>

#include "page_join.cuh"

namespace reflex {

using namespace ptx;

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
constexpr unsigned long long kTokenWaitNs = 1000000000ull;

// Adds 1 and returns what was there. What the block has written before its last barrier is seen by whoever sees the sum, and the other way round
__device__ __forceinline__ uint32_t arrive_gpu(uint32_t *at)
{
    uint32_t old;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(at) : "memory");
    return old;
}

template <int FMT, int HD, int NT> struct Tok {
    static constexpr bool BYTES = FMT != REFLEX_PAGE_SAME;
    static constexpr int ROW = HD * (BYTES ? 1 : 2);               // bytes of a row
    static constexpr int STEPS = HD / 16;                          // steps over head_dim
    static constexpr int KP = ROW / 64;                            // 16-byte pieces of a key per thread
    static constexpr int KEPP = BYTES ? 16 : 8;                    // elements of a piece of K
    static constexpr int VB = ROW / 8;                             // bytes of a value row per thread: 8, 16, 32, 64
    static constexpr int VPB = VB < 16 ? 8 : 16;                   // ... in pieces of so many
    static constexpr int VW = VB / 4;                              // ... in words
    static constexpr int VCOLS = VB < 16 ? 8 : BYTES ? 16 : 8;     // consecutive columns of a thread
    static constexpr int VPIECES = HD / 8 / VCOLS;
    static constexpr int ROWS = 8 * NT;
    // a warp's blocks of keys: 16 rows of K, 16 of V, in boxes of 128 bytes (or 64) as TMA swizzles them; the exponents lie behind all stages
    static constexpr int BOX = ROW < 128 ? ROW : 128;
    static constexpr uint32_t K_BYTES = 16 * ROW, STAGE = 2 * K_BYTES;
    static constexpr int STAGES = STAGE > 4 * 1024 ? 2 : 3;
    // One CTA per SM, with as many warps as registers (some 64 of O per 8 rows of head_dim 256, and 100 others) and stages leave room for: what a
    // CTA does per unit (its place, Q, joining its warps, a partial) is then shared by all keys that the SM takes of it.
    static constexpr int WARPS = HD * NT <= 64 ? 16 : BYTES ? (HD * NT > 256 ? 8 : 12) : HD == 256 ? 6 : HD * NT > 128 ? 8 : 12;
    static constexpr int BLOCK = 16 * WARPS;                       // keys of a block: what the line of work is counted in
    // a warp's share of O takes the place of its keys in the end: of the last ones, while the first ones of the next unit come, if it is no larger
    static constexpr uint32_t O_BYTES = ROWS * HD * 4;
    static constexpr bool EARLY = O_BYTES <= STAGE;
    static constexpr uint32_t WARP = ((STAGES * STAGE > O_BYTES ? STAGES * STAGE : O_BYTES) + 1023u) & ~1023u;
    static constexpr uint32_t OFF_Q = WARPS * WARP;            // [step][NT][lane] of two registers
    static constexpr uint32_t OFF_ML = OFF_Q + STEPS * NT * 256;   // [warps][ROWS] of (maximum, sum)
    static constexpr uint32_t OFF_PLACE = OFF_ML + WARPS * ROWS * 8;
    static constexpr uint32_t OFF_EXP = OFF_PLACE + 128;           // [warps][STAGES] of 16 + 16 exponents
    static constexpr uint32_t OFF_BAR = OFF_EXP + (BYTES ? WARPS * STAGES * 32 : 0);      // [warps][STAGES]
    static constexpr uint32_t NEED = OFF_BAR + WARPS * STAGES * 8, SMEM = NEED + 1008;    // (room to begin at a multiple of 1024)
    static_assert(SMEM <= 232448, "shared memory");
};

// the blocks of keys that a tile of ROWS rows needs, and the pieces of `per` blocks that they make
struct TokSpan { int lo, hi, blocks, count; };
template <int ROWS, int BLOCK>
struct TokSpanOf {
    const PageAttention &p;
    int G, per;
    __device__ __forceinline__ int tiles(const PageSeq &s) const { return (s.n * G + ROWS - 1) / ROWS; }
    __device__ __forceinline__ TokSpan operator()(const PageSeq &s, int tile) const
    {
        const PageRange r = page_range(s, p, p.token_of(tile * ROWS, G), p.token_of(min(s.n * G, (tile + 1) * ROWS) - 1, G));
        TokSpan t;
        t.lo = r.lo & ~15;
        t.hi = r.hi;
        t.blocks = t.hi > t.lo ? (t.hi - t.lo + BLOCK - 1) / BLOCK : 0;
        t.count = per == 1 ? t.blocks : (t.blocks + per - 1) / per;
        return t;
    }
};

template <int FMT, int HD, int NT>
__global__ void __launch_bounds__((32 * Tok<FMT, HD, NT>::WARPS), 1)
page_token_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const PageAttention p, const PagePartials part)
{
    using C = Tok<FMT, HD, NT>;
    constexpr int ROWS = C::ROWS, WARPS = C::WARPS, BLOCK = C::BLOCK;
    extern __shared__ __align__(16) uint8_t raw_smem[];
    uint8_t *smem = raw_smem + (-smem_u32(raw_smem) & 1023u);
    uint2 *q_s = reinterpret_cast<uint2 *>(smem + C::OFF_Q);
    float2 *ml_s = reinterpret_cast<float2 *>(smem + C::OFF_ML);
    const PageGeom &g = p.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, t4 = lane & 3;
    const int G = g.Hq / g.Hkv;
    uint8_t *keys = smem + warp * C::WARP;             // this warp's stages
    const uint32_t keys_at = smem_u32(keys), exps_at = smem_u32(smem + C::OFF_EXP) + warp * C::STAGES * 32, bars = smem_u32(smem + C::OFF_BAR) + warp * C::STAGES * 8;

    // Warp 0 walks the line for all. Where there are fewer blocks than keep all CTAs busy, the line is counted in pieces of several blocks, a CTA takes one, and
    // none has parts of two units: the square root of a fifth of the longest unit, since joining a partial costs about a fifth of a block.
    // (8 streams of 3300 keys, bf16: 27.0 us in blocks, 35 a stream and two a CTA, 18.6 in pieces of two.)
    using Line = PageLine<TokSpanOf<ROWS, BLOCK>>;
    Line line{p, {p, G, 1}};
    struct Join { int parts, from, row, head, m, rows; };           // a split unit that this CTA has to join (parts: 0 if it has not)
    struct Shared { typename Line::Place u; int total, nc, per; Join join[2]; };      // (u: the first unit, and later the next)
    static_assert(sizeof(Shared) <= 128, "place in shared memory");
    Shared *sh = reinterpret_cast<Shared *>(smem + C::OFF_PLACE);
    const int cta = blockIdx.x;
    if (lane < C::STAGES) mbar_init(bars + lane * 8, 1);
    fence_mbar_init();
    if (warp == 1 && lane < 2) prefetch_tmap(lane ? &tm_v : &tm_k);
    if (warp == 0) {
        int total = line.begin(lane);
        const int per = (int)sqrtf((float)line.longest * 0.2f);
        if (per > 1 && total <= per * (int)gridDim.x) {
            line.span.per = per;
            total = line.count(lane);
        }
        const int nc = min((int)gridDim.x, total);
        if (cta < nc) {
            const typename Line::Place first = line.find(PageShares(total, nc).of(cta), lane);
            if (lane == 0) sh->u = first;
        }
        if (lane == 0) { sh->total = total; sh->nc = nc; sh->per = line.span.per; sh->join[0].parts = sh->join[1].parts = 0; }
    }
    __syncthreads();
    const int nc = sh->nc;
    if (cta >= nc) return;
    const PageShares shares(sh->total, nc);
    const int x0 = shares.of(cta), x1 = shares.of(cta + 1), per = sh->per;
    line.span.per = per;

    int put = 0, got = 0;                              // the stage that is filled next, that is read next
    uint32_t got_phase = 0;
    int pending = 0;                                   // asked for and not yet waited for
    bool dead = false;                                 // a wait has run out: nothing more is asked for
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        if (mbar_try_wait(bar, parity)) return true;
        const unsigned long long t0 = globaltimer_ns();
        for (uint32_t n = 1;; ++n) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((n & 255u) == 0u && globaltimer_ns() - t0 > kTokenWaitNs) return false;
        }
    };
    // where this thread's pieces lie in a stage
    const uint32_t k_piece = C::ROW < 128 ? gq * 64 + ((t4 ^ (gq >> 1)) << 4) : gq * 128 + (((2 * t4) ^ gq) << 4);
    const uint32_t v_piece = C::K_BYTES + (C::ROW < 128 ? t4 * 128 + (((gq >> 1) ^ t4) << 4) + (gq & 1) * 8 : t4 * 256 + (((2 * t4) ^ gq) << 4));
    auto key_at = [&](int e, int j) -> uint32_t {      // piece j of key g + 8 e
        return C::ROW < 128 ? k_piece + e * 512 : (k_piece ^ ((j & 1) << 4)) + (j >> 1) * 2048 + e * 1024;
    };
    auto value_at = [&](int e, int j) -> uint32_t {    // piece j of key 2 t + (e & 1) + 8 (e >> 1)
        return C::ROW < 128 ? v_piece + (e & 1) * 64 + (e >> 1) * 512 : (v_piece ^ ((e & 1) << 4)) + (e & 1) * 128 + (e >> 1) * 1024 + j * 2048;
    };
    // ---- the unit at hand ----
    typename Line::Place u = sh->u;
    int t_first, m_first, rows_here, k0, kend, key0, ids_from, page_ids;
    uint32_t bad_pages;                                // of the blocks on their way, the first in bit 0
    auto token_of = [&](int r) -> int { return G == 1 ? r : (int)__umulhi((uint32_t)(m_first + r), p.g_magic); };        // of the tile's row r, from t_first on
    // (the pages of 32 of this warp's blocks are looked up together)
    auto look_up = [&](int i) {
        ids_from = i;
        page_ids = i + lane < kend ? page_at(p.q, g.n_pages, u.s.b, (key0 + (i + lane) * BLOCK) >> g.log_p) : -1;
    };
    auto enter = [&](int x) {
        u = sh->u;
        t_first = p.token_of(u.tile * ROWS, G);
        m_first = u.tile * ROWS - t_first * G;
        rows_here = min(ROWS, u.s.n * G - u.tile * ROWS);
        k0 = (x - u.at) * per;
        kend = min(min(u.cost, x1 - u.at) * per, u.sp.blocks);
        key0 = u.sp.lo + warp * 16;                    // keys of block i: key0 + BLOCK i ..
        bad_pages = 0;
        look_up(k0);
    };
    auto fetch = [&](int i) {
        if (i >= kend || dead) return;
        if (i - ids_from >= 32) look_up(i);
        const int key = key0 + i * BLOCK, page = __shfl_sync(0xffffffffu, page_ids, i - ids_from);
        if (page < 0) bad_pages |= 1u << (i - k0 & 31);
        else bad_pages &= ~(1u << (i - k0 & 31));
        const size_t row = page_row(g, max(page, 0), u.h) + (size_t)(key & (g.P - 1));
        const uint32_t dst = keys_at + put * C::STAGE, bar = bars + put * 8;
        mbar_expect_tx_elect(bar, C::STAGE + (C::BYTES ? 32 : 0));
        tma_load_3d_elect(dst, &tm_k, bar, 0, (int)row, 0);
        if constexpr (C::BYTES) {
            bulk_load_elect(exps_at + put * 32, g.ke + row, bar, 16);
            bulk_load_elect(exps_at + put * 32 + 16, g.ve + row, bar, 16);
        }
        tma_load_3d_elect(dst + C::K_BYTES, &tm_v, bar, 0, (int)row, 0);
        put = put + 1 == C::STAGES ? 0 : put + 1;
        ++pending;
    };
    auto fetch_first = [&] {
#pragma unroll
        for (int i = 0; i < C::STAGES - 1; ++i) fetch(k0 + i);
    };
    auto stage_q = [&] {                               // Q of the unit's rows, in the order of K's pieces
        for (int i = threadIdx.x; i < C::STEPS * NT * 32; i += 32 * WARPS) {
            const int ln = i & 31, nt = (i >> 5) % NT, step = (i >> 5) / NT;
            const int r = nt * 8 + (ln >> 2), t = token_of(r);
            const int j = C::BYTES ? step >> 2 : step >> 1;
            const int d0 = (C::ROW < 128 ? 16 * (ln & 3) : (j >> 1) * (C::BYTES ? 128 : 64) + (2 * (ln & 3) + (j & 1)) * C::KEPP) + 4 * (C::BYTES ? step & 3 : step & 1);
            uint2 v = make_uint2(0u, 0u);
            if (r < rows_here) v = *reinterpret_cast<const uint2 *>((const __nv_bfloat16 *)p.qry + ((size_t)(u.s.row0 + t_first + t) * g.Hq + u.h * G + m_first + r - t * G) * HD + d0);
            q_s[i] = v;
        }
    };
    enter(x0);
    fetch_first();
    stage_q();
    __syncthreads();

    for (;;) {
        const PageSeq s = u.s;
        const TokSpan span = u.sp;
        const int x = min(u.at + u.cost, x1);          // the next unit begins there
        if (x < x1 && warp == WARPS - 1 && lane == 0) {
            typename Line::Place next = u;
            line.next(next);
            sh->u = next;
        }
        // ---- this thread's query rows: 2t, 2t + 1 of every group of 8 ----
        int lo_r[2 * NT], hi_r[2 * NT], lo_min, lo_max, hi_min, hi_max;      // (the limits of all the tile's rows)
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            const int t = t_first + token_of(min((i >> 1) * 8 + 2 * t4 + (i & 1), rows_here - 1));
            const PageRange v = page_range(s, p, t, t);
            lo_r[i] = v.lo; hi_r[i] = v.hi;
        }
        {
            const int t_last = t_first + token_of(rows_here - 1);
            const PageRange first = page_range(s, p, t_first, t_first), last = page_range(s, p, t_last, t_last);
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

        // O^T += V^T P^T of the loaded block
        auto value_word = [&](const uint8_t *stage, int e, int i) -> uint32_t {       // word i of this thread's part of the e-th of its keys
            return *reinterpret_cast<const uint32_t *>(stage + value_at(e, i / (C::VPB / 4)) + i % (C::VPB / 4) * 4);
        };
        auto times_v = [&](const uint8_t *stage, const uint32_t (&pt)[NT][2]) {
            uint32_t v[4][C::VPB / 4];
#pragma unroll
            for (int i = 0; i < C::VW; ++i) {
                if (i % (C::VPB / 4) == 0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint8_t *src = stage + value_at(e, i / (C::VPB / 4));
                        if constexpr (C::VPB == 16) *reinterpret_cast<uint4 *>(v[e]) = *reinterpret_cast<const uint4 *>(src);
                        else *reinterpret_cast<uint2 *>(v[e]) = *reinterpret_cast<const uint2 *>(src);
                    }
                }
                const uint32_t w[4] = {v[0][i % (C::VPB / 4)], v[1][i % (C::VPB / 4)], v[2][i % (C::VPB / 4)], v[3][i % (C::VPB / 4)]};
                if constexpr (C::BYTES) {
                    // four columns of four keys: two tiles of 16 (column, column + 1) pairs. Pairs of keys are put side by side first.
                    const uint32_t lo01 = biased<FMT>(__byte_perm(w[0], w[1], 0x5140)), hi01 = biased<FMT>(__byte_perm(w[0], w[1], 0x7362));
                    const uint32_t lo23 = biased<FMT>(__byte_perm(w[2], w[3], 0x5140)), hi23 = biased<FMT>(__byte_perm(w[2], w[3], 0x7362));
                    const uint32_t a[8] = {expand2<FMT, 0, 1>(lo01), expand2<FMT, 2, 3>(lo01), expand2<FMT, 0, 1>(lo23), expand2<FMT, 2, 3>(lo23),
                                           expand2<FMT, 0, 1>(hi01), expand2<FMT, 2, 3>(hi01), expand2<FMT, 0, 1>(hi23), expand2<FMT, 2, 3>(hi23)};
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

#pragma unroll 1
        for (int i = k0; i < kend; ++i) {
            const int key = key0 + i * BLOCK;
            __syncwarp();                             // (the stage that is filled next has been read by all lanes)
            fetch(i + C::STAGES - 1);
            const int st = got;
            if (pending > 0) {
                --pending;
                if (!__all_sync(0xffffffffu, wait(bars + st * 8, got_phase)) && !dead) {
                    dead = true;
                    if (lane == 0) report_page_wait(g.status, kSitePageToken + 1u);
                }
                got = got + 1 == C::STAGES ? 0 : got + 1;
                got_phase ^= got == 0 ? 1u : 0u;
            }
            const uint8_t *stage = keys + st * C::STAGE;
            const bool lost = (bad_pages >> (i - k0 & 31)) & 1u;             // no page to read these keys from
            bad |= dead || (lost && key < span.hi);
            // ---- logits ----
            float c[NT][2][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[nt][0][e] = c[nt][1][e] = 0.f;
#pragma unroll
            for (int j = 0; j < C::KP; ++j) {
                uint4 k4[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) k4[e] = *reinterpret_cast<const uint4 *>(stage + key_at(e, j));
                const uint32_t w0[4] = {k4[0].x, k4[0].y, k4[0].z, k4[0].w}, w1[4] = {k4[1].x, k4[1].y, k4[1].z, k4[1].w};
#pragma unroll
                for (int u2 = 0; u2 < (C::BYTES ? 4 : 2); ++u2) {
                    const int step = j * (C::BYTES ? 4 : 2) + u2;
                    uint32_t a0, a1, a2, a3;
                    if constexpr (C::BYTES) {
                        const uint32_t x0 = biased<FMT>(w0[u2]), x1 = biased<FMT>(w1[u2]);
                        a0 = expand2<FMT, 0, 1>(x0); a1 = expand2<FMT, 0, 1>(x1);
                        a2 = expand2<FMT, 2, 3>(x0); a3 = expand2<FMT, 2, 3>(x1);
                    } else {
                        a0 = w0[2 * u2]; a1 = w1[2 * u2]; a2 = w0[2 * u2 + 1]; a3 = w1[2 * u2 + 1];
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint2 q = q_s[(step * NT + nt) * 32 + lane];
                        mma_bf16(c[nt][step & 1], a0, a1, a2, a3, q.x, q.y);
                    }
                }
            }
            int ke[2] = {127, 127}, ve[2] = {127, 127};
            if constexpr (C::BYTES) {
                const uint8_t *ex = smem + C::OFF_EXP + (warp * C::STAGES + st) * 32;
                ke[0] = ex[gq]; ke[1] = ex[gq + 8]; ve[0] = ex[16 + gq]; ve[1] = ex[16 + gq + 8];
            }
            const float ks0 = C::BYTES ? exponent_f32<FMT>(ke[0]) * part.scale_log2 : part.scale_log2, ks1 = C::BYTES ? exponent_f32<FMT>(ke[1]) * part.scale_log2 : part.scale_log2;
            // ---- masks, running maximum, weights ----
            const bool whole = key >= lo_max && key + 16 <= hi_min && !lost;
            float w[NT][4];            // (key g, row 2t), (g, 2t + 1), (g + 8, 2t), (g + 8, 2t + 1)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[nt][e] = (c[nt][0][e] + c[nt][1][e]) * (e < 2 ? ks0 : ks1);
                    if (!whole) {
                        const int j = key + gq + (e < 2 ? 0 : 8);
                        if (j < lo_r[2 * nt + (e & 1)] || j >= hi_r[2 * nt + (e & 1)] || lost) w[nt][e] = -INFINITY;
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
            const float vs0 = C::BYTES ? exponent_f32<FMT>(ve[0]) : 1.f, vs1 = C::BYTES ? exponent_f32<FMT>(ve[1]) : 1.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x2 = w[nt][e], mr = m[2 * nt + (e & 1)];
                    const float pe = ex2(x2 - (mr == -INFINITY ? 0.f : mr + kWeightShift));
                    l[2 * nt + (e & 1)] += pe;
                    v[e] = !whole && x2 == -INFINITY ? 0.f : C::BYTES ? pe * (e < 2 ? vs0 : vs1) : pe;
                }
                pt[nt][0] = transpose8x8(pack_bf16(v[0], v[1]));
                pt[nt][1] = transpose8x8(pack_bf16(v[2], v[3]));
            }
            // ---- values ----
            if (!C::BYTES && !whole) {
                // A masked key has weight 0, but 0 times what lies there may be NaN: keys that no row sees become zeros. A key that some
                // rows see is multiplied for all of them, which does no harm while it is finite. (In place and in short loops: as a second
                // form of the products this was 1000 instructions, and 7 us of the one block at the end of a sequence, most of them to fetch the code.)
                auto each_piece = [&](auto change) -> bool {          // change(key, uint32_t &pair of elements) -> bool
                    bool any = false;
#pragma unroll 1
                    for (uint32_t at = lane * 16; at < C::K_BYTES; at += 512) {
                        uint4 *piece = reinterpret_cast<uint4 *>(const_cast<uint8_t *>(stage) + C::K_BYTES + at);
                        uint4 v = *piece;
                        const int j = key + (int)((at / C::BOX) & 15);
                        any |= change(j, v.x); any |= change(j, v.y); any |= change(j, v.z); any |= change(j, v.w);
                        *piece = v;
                    }
                    fence_proxy_async_smem();         // (TMA writes there next)
                    __syncwarp();
                    return __any_sync(0xffffffffu, any);
                };
                auto odd_low = [](uint32_t w) -> bool { return (w & 0x7f80u) == 0x7f80u; };
                auto odd_high = [](uint32_t w) -> bool { return (w & 0x7f800000u) == 0x7f800000u; };
                const bool any_odd = each_piece([&](int j, uint32_t &w) -> bool {
                    if (j < lo_min || j >= hi_max || lost) w = 0u;
                    return odd_low(w) || odd_high(w);
                });
                if (any_odd) {
                    // what is not finite goes, as it is, to the rows that see it (whatever their weight), and counts as zero in the products
#pragma unroll 1
                    for (int from = 0; from < 4; ++from) {
#pragma unroll 1
                        for (int e = 0; e < 4; ++e) {
                            const int j = key + 2 * from + (e & 1) + 8 * (e >> 1);
#pragma unroll
                            for (int i2 = 0; i2 < C::VW; ++i2) {
                                const uint32_t v = __shfl_sync(0xffffffffu, value_word(stage, e, i2), (lane & ~3) | from);
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
                    each_piece([&](int, uint32_t &w) -> bool {
                        if (odd_low(w)) w &= 0xffff0000u;
                        if (odd_high(w)) w &= 0x0000ffffu;
                        return false;
                    });
                }
            }
            times_v(stage, pt);
        }
        __syncwarp();                                 // (the stages may be written over)
        // ---- the warps' shares meet ----
        const uint32_t o_at = C::EARLY ? (put == 0 ? C::STAGES - 1 : put - 1) * C::STAGE : 0;      // (the same for all warps)
        const bool any_bad = __any_sync(0xffffffffu, bad);
        if (any_bad && lane == 0) report_bad_page(g.status, s.b);
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
            for (int q = 0; q < WARPS; ++q) all = fmaxf(all, ml_s[q * ROWS + rr].x);
            f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - all);
            // column c of piece j: 8 VCOLS j + VCOLS g + c; register (tile, 0 / 2) holds an even / odd column of an even row's pair. Four columns lie
            // where 16-byte pieces of a row are swapped by its bits 1 and 2: neither these writes nor the reads below meet in a bank more often than they must.
            float *dst = reinterpret_cast<float *>(keys + o_at) + rr * HD;
#pragma unroll
            for (int j = 0; j < C::VPIECES; ++j)
#pragma unroll
                for (int x2 = 0; x2 < C::VCOLS; x2 += 4) {
                    const int tile = (j * C::VCOLS + x2) / 2, piece = (j * 8 + gq) * (C::VCOLS / 4) + x2 / 4;
                    *reinterpret_cast<float4 *>(dst + 4 * (piece ^ t4)) = make_float4(o[tile][r >> 1][r & 1] * f[r], o[tile][r >> 1][2 + (r & 1)] * f[r],
                                                                                      o[tile + 1][r >> 1][r & 1] * f[r], o[tile + 1][r >> 1][2 + (r & 1)] * f[r]);
                }
        }
        // ---- the next unit is on its way while this one's results are written ----
        const bool starts = k0 == 0, ends = u.at + u.cost <= x1;
        const int slot = 2 * cta + (starts ? 1 : 0), h = u.h, rows_done = rows_here, t_done = t_first, m_done = m_first;
        const int from = starts ? cta : shares.owner(u.at), parts = (ends ? cta : shares.owner(u.at + u.cost - 1)) - from + 1;     // the CTAs on this unit
        if (x < x1) {
            enter(x);
            if (C::EARLY) fetch_first();
            stage_q();
        }
        __syncthreads();
        for (int i = threadIdx.x; i < ROWS * (HD / 8); i += 32 * WARPS) {
            const int r = i / (HD / 8), c0 = i % (HD / 8) * 8;
            if (r >= rows_done) continue;
            const int t = G == 1 ? r : (int)__umulhi((uint32_t)(m_done + r), p.g_magic);
            float all = -INFINITY, sum = 0.f, acc[8];
            if (parts == 1 || c0 == 0) {
#pragma unroll
                for (int q = 0; q < WARPS; ++q) all = fmaxf(all, ml_s[q * ROWS + r].x);
#pragma unroll
                for (int q = 0; q < WARPS; ++q) {
                    const float2 v = ml_s[q * ROWS + r];
                    // (a maximum of -inf carries no weight, a sum that is NaN is kept)
                    sum += v.x == -INFINITY ? v.y * 0.f : v.y * ex2(v.x - all);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
            for (int q = 0; q < WARPS; ++q) {
                const float *src = reinterpret_cast<const float *>(smem + q * C::WARP + o_at) + r * HD;
                const float4 y0 = *reinterpret_cast<const float4 *>(src + 4 * ((c0 >> 2) ^ ((r >> 1) & 3))), y1 = *reinterpret_cast<const float4 *>(src + 4 * ((c0 >> 2) + 1 ^ ((r >> 1) & 3)));
                acc[0] += y0.x; acc[1] += y0.y; acc[2] += y0.z; acc[3] += y0.w;
                acc[4] += y1.x; acc[5] += y1.y; acc[6] += y1.z; acc[7] += y1.w;
            }
            if (parts == 1) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] *= inv;
                store8((__nv_bfloat16 *)p.out + ((size_t)(s.row0 + t_done + t) * g.Hq + h * G + m_done + r - t * G) * HD + c0, acc);
            } else {
                const uint32_t bits[8] = {__float_as_uint(acc[0]), __float_as_uint(acc[1]), __float_as_uint(acc[2]), __float_as_uint(acc[3]),
                                          __float_as_uint(acc[4]), __float_as_uint(acc[5]), __float_as_uint(acc[6]), __float_as_uint(acc[7])};
                st_global_v8(partial8(part, slot, HD, r, c0), bits);
                if (c0 == 0) part.ml[(size_t)slot * part.rows + r] = make_float2(all, sum);
            }
        }
        fence_proxy_async_smem();    // (blocks come over what the warps put down)
        __syncthreads();             // (this unit's results have been read, the next one's Q is there)
        if (parts > 1 && threadIdx.x == 0) {
            Join &jn = sh->join[starts ? 1 : 0];
            jn.parts = arrive_gpu(part.arrived + from) == (uint32_t)parts - 1u ? parts : 0;
            jn.from = from; jn.row = s.row0 + t_done; jn.head = h * G; jn.m = m_done; jn.rows = rows_done;
        }
        if (x >= x1) break;
        if (!C::EARLY) fetch_first();
    }

    // ---- the last CTA on a split unit to come by joins the partials of all, behind its own units ----
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        const Join jn = sh->join[which];
        const int n = jn.parts;
        if (n == 0) continue;
        if (threadIdx.x == 0) part.arrived[jn.from] = 0u;
        // (short code: what runs once costs what it takes to fetch it; with the partials in shared memory, or the weights worked out first, it was no faster)
        for (int i = threadIdx.x; i < ROWS * (HD / 8); i += 32 * WARPS) {
            const int r = i % ROWS, c0 = i / ROWS * 8, t = G == 1 ? r : (int)__umulhi((uint32_t)(jn.m + r), p.g_magic);
            PageSum a;
            page_sum(part, HD, jn.from, n, r, c0, 0, 1, a);
            if (r >= jn.rows) continue;
            const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
#pragma unroll
            for (int e = 0; e < 8; ++e) a.o[e] *= inv;
            store8((__nv_bfloat16 *)p.out + ((size_t)(jn.row + t) * g.Hq + jn.head + jn.m + r - t * G) * HD + c0, a.o);
        }
    }
}

template <int FMT, int HD, int NT>
static cudaError_t launch_token(const PageAttention &a, const PagePartials &part, int sm_count, cudaStream_t st)
{
    using C = Tok<FMT, HD, NT>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = once_per_device(done, [] { return cudaFuncSetAttribute(page_token_kernel<FMT, HD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM); });
    if (e != cudaSuccess) return e;
    CUtensorMap tk, tv;
    if (!encode_map_rows(&tk, a.g.k, C::ROW, a.g.n_pages * a.g.Hkv * a.g.P, 16) || !encode_map_rows(&tv, a.g.v, C::ROW, a.g.n_pages * a.g.Hkv * a.g.P, 16)) return cudaErrorInvalidValue;
    count_launch();
    page_token_kernel<FMT, HD, NT><<<std::min(sm_count, kTokenCtas), 32 * C::WARPS, C::SMEM, st>>>(tk, tv, a, part);
    return cudaGetLastError();
}

// Rows of a tile for `rows` (token, head) rows per sequence and KV head on average; 0: not for this kernel. Every tile reads the keys again (from L2) and has
// them expanded again, so page_chunk_kernel is ahead from some number of rows on; later in 8-bit formats, whose pages have to be widened for it.
// bf16, 64 streams: 53 us here and 57 there at 16 rows of 256 (3300 keys), 124 and 57 at 32; 95 and 79 at 32 rows of 128 (2000 keys, 4 KV heads).
// int8: 63 and 115 at 32 rows of 256, 111 and 117 at 64; 96 and 145, 174 and 145 at 32 and 64 rows of 128; 134 and 202 at 32 rows of 64.
// (What is known of a batch is its average: lengths are on the device. A chunk of hundreds of rows among many sequences of one token comes here as well, where
// each of its tiles reads the keys again; the figures are those of even batches.)
int page_token_rows(int dtype, int format, int d, int G, int rows)
{
    if (dtype != REFLEX_DTYPE_BF16 || d < 64 || G > 4096) return 0;
    const bool wide = format == REFLEX_PAGE_SAME && d == 256;         // (16 rows of bf16 rows of 256 do not fit the registers)
    if (rows > (format == REFLEX_PAGE_SAME ? 16 : 64) && page_chunk_takes(dtype, G, d)) return 0;
    return rows <= 8 || wide ? 8 : 16;
}

cudaError_t launch_page_token(const PageAttention &a, const PagePartials &part, int format, int rows, int sm_count, cudaStream_t st)
{
    auto go = [&](auto f, auto hd) -> cudaError_t {
        constexpr int FMT = decltype(f)::value, HD = decltype(hd)::value;
        if constexpr (!(FMT == REFLEX_PAGE_SAME && HD == 256))
            if (rows == 16) return launch_token<FMT, HD, 2>(a, part, sm_count, st);
        return launch_token<FMT, HD, 1>(a, part, sm_count, st);
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
