// Attention of a chunk of new tokens over pages (reflex_pages_attention) on the tensor cores: tcgen05.mma.cta_group::2, M = 256.
//
// A pair of CTAs takes 256 (token, head) rows of a sequence and KV head, 128 each, and walks the keys in tiles of 128. Of every tile a CTA holds half:
// 64 keys of K, and half of the columns of V; TMA brings them from the pages, one box per page (or per 64 tokens of a larger page), to
// where the swizzled tile has them. S = Q K^T and O = P V accumulate in tensor memory; P (bf16) is written over the logits it came from and is
// the A operand of P V from there. Per CTA:
//   warp 0       TMA producer (its Q tile, its half of K, its columns of V)
//   warp 1       MMA issuer (leader CTA): Q K^T of the next tile before P V of this one
//   warps 2..9   softmax: two threads per row, 64 keys each; maxima through shared memory, lazy rescale of O
// What bounds it: at head_dim 256 the tensor pipe (2048 cycles a tile; operand reads then take two thirds of the shared memory's bandwidth), at 128 and
// 64 the softmax (16 K exponentials a tile and SM). Heads of 64 run as heads of 128 whose upper chunk is left out of Q K^T and whose upper columns of O
// are never read: P V costs twice, underneath the softmax.
//
// The grid is one pair per SM pair; the tiles of all units form one line that the pairs share evenly (PageLine), so uneven sequences, causal masks and single
// sequences fill the device alike. A unit that more than one pair works on leaves fp32 partials for page_merge_kernel.
// 8-bit pages are first widened to bf16, exactly, into one layer's worth of workspace (page_widen_kernel): a page is used by every row tile and by both
// CTAs of a pair, and unpacking it inside each costs more instruction slots than the softmax leaves.
//
// Every wait is bounded; one that runs out is reported in the status word and makes the results NaN.
#include <math.h>

#include <algorithm>

#include "page_attention.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

using namespace ptx;

constexpr int kChunkKeys = 128;
constexpr int kChunkThreads = 64 + 256;
constexpr int kChunkRows = 256;                // of a unit
constexpr unsigned long long kChunkWaitNs = 1000000000ull;
constexpr float kChunkGrow = 8.0f;             // log2 units: O is rescaled only where a maximum grows by more than 2^8
constexpr int kChunkPoly = 2;                  // of every 8 pairs of exponentials, how many go through the FMA pipe

__device__ __forceinline__ void report_page_wait(uint32_t *status, uint32_t code) { atomicCAS(status, 0u, status_word(kSitePages + code)); }

struct ChunkSpan { int tile0, count, hi; };    // key tiles [tile0, tile0 + count), keys below hi
struct ChunkSpanOf {
    const PageAttention &p;
    int tokens;                                // of a unit
    __device__ __forceinline__ ChunkSpan operator()(const PageSeq &s, int tile) const
    {
        const PageRange r = page_range(s, p, tile * tokens, min(s.n, (tile + 1) * tokens) - 1);
        ChunkSpan c;
        c.tile0 = r.lo / kChunkKeys;
        c.hi = r.hi;
        c.count = r.hi > r.lo ? (r.hi + kChunkKeys - 1) / kChunkKeys - c.tile0 : 0;
        return c;
    }
};

template <int HD, int D> struct Chunk {
    static constexpr int CH = D / 64;                           // 64-column chunks of Q and K
    static constexpr int VCH = HD / 128;                        // chunks of V of this CTA
    static constexpr int NST = HD == 256 ? 2 : 4;               // stages of K, and of V
    static constexpr uint32_t Q_BYTES = CH * 128 * 128;
    static constexpr uint32_t K_STAGE = CH * 64 * 128;
    static constexpr uint32_t V_STAGE = VCH * 128 * 128;
    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_K = OFF_Q + Q_BYTES;
    static constexpr uint32_t OFF_V = OFF_K + NST * K_STAGE;
    static constexpr uint32_t OFF_STAGE = OFF_V + NST * V_STAGE;      // two halves of 128 rows x 64 columns of the result
    static constexpr uint32_t OFF_BAR = OFF_STAGE + 2 * 128 * 128;
    static constexpr uint32_t OFF_XMAX = OFF_BAR + 256;               // [2][128][2] row maxima
    static constexpr uint32_t NEED = OFF_XMAX + 2 * 128 * 2 * 4;
    static constexpr uint32_t TOTAL = NEED + 1024 > 232448 ? 232448 : NEED + 1024;
    static constexpr int QFULL = 0, QEMPTY = 1, KFULL = 2, KEMPTY = KFULL + NST, VLAND = KEMPTY + NST, VEMPTY = VLAND + NST, SFULL = VEMPTY + NST, PFULL = SFULL + 2,
                         PVDONE = PFULL + 2, OFREE = PVDONE + 2, COUNT = OFREE + 1;
    static_assert(8 * COUNT + 8 + 32 <= 256, "barriers, tensor memory's address, abort flag, bad units");
};

// bits [lo, hi) of a 64-bit word, whatever lo and hi are
__device__ __forceinline__ uint64_t bits64(int lo, int hi)
{
    lo = max(lo, 0); hi = min(hi, 64);
    if (hi <= lo) return 0ull;
    return (hi >= 64 ? ~0ull : (1ull << hi) - 1ull) & ~((1ull << lo) - 1ull);
}

template <int HD, int D>
__global__ void __launch_bounds__(kChunkThreads, 1)         // clusters of two
page_chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const PageAttention p, const PagePartials part, int tile_tokens, int box)
{
    using L = Chunk<HD, D>;
    constexpr int CH = L::CH, VCH = L::VCH, NST = L::NST;
    constexpr uint32_t kColS = HD;
    static_assert(HD + 2 * kChunkKeys <= 512, "tensor memory");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw_addr);
    const uint32_t bar0 = base + L::OFF_BAR;
    auto bar = [&](int i) -> uint32_t { return bar0 + 8u * (uint32_t)i; };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::OFF_BAR + 8 * L::COUNT);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    volatile uint32_t *bad_unit = tmem_slot + 2;          // [8]: number (from 1) of the last unit of that residue which met a bad page
    if ((base - raw_addr) + L::NEED > L::TOTAL) {          // (the same for every CTA: all of them leave)
        if (threadIdx.x == 0) report_page_wait(p.g.status, 15u);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int G = p.g.Hq / p.g.Hkv;
    const ChunkSpanOf span_of{p, 2 * tile_tokens};
    const PageLine<ChunkSpanOf> line{p, span_of, 2 * tile_tokens * G, G};

    if (threadIdx.x == 0) {
        for (int i = 0; i < L::COUNT; ++i) mbar_init(bar(i), i == L::PFULL || i == L::PFULL + 1 || i == L::OFREE ? 16u : 1u);      // one arrival per softmax warp of either CTA
        *abort_flag = 0u;
        for (int i = 0; i < 8; ++i) bad_unit[i] = 0u;
        fence_mbar_init();
        prefetch_tmap(&tm_q); prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    }
    if (warp == 1) tmem_alloc2(smem_u32((const void *)tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // (the merge, which waits for this grid's end)

    auto wait = [&](int i, uint32_t parity, uint32_t code) -> bool {
        if (mbar_try_wait(bar(i), parity)) return true;
        const unsigned long long t_start = globaltimer_ns();
        for (uint32_t n = 1;; ++n) {
            if (mbar_try_wait(bar(i), parity)) return true;
            if ((n & 255u) == 0u) {
                if (*abort_flag) return false;
                if (globaltimer_ns() - t_start > kChunkWaitNs) break;
            }
        }
        *abort_flag = 1u;
        report_page_wait(p.g.status, code);
        return false;
    };

    int longest;
    const long long total = line.total(lane, longest);
    const int nc = (int)min((long long)pairs, total);
    if (threadIdx.x == 64 && rank == 0) part.meta[pair].b = -1;      // (the thread that may write the entry later)
    const bool works = pair < nc;
    const long long x0 = works ? page_share(pair, total, nc) : 0, x1 = works ? page_share(pair + 1, total, nc) : 0;
    using Place = typename PageLine<ChunkSpanOf>::Place;
    // this pair's units, one after the other: the slice [k0, k1) of the unit's blocks, of which `n` are tiles of keys from tile `t0` on
    struct Slice { Place u; long long x; int k0, k1, t0, n; };
    auto cut = [&](Slice &w) {
        w.k0 = (int)(w.x - w.u.at);
        w.k1 = (int)min((long long)w.u.cost, x1 - w.u.at);
        w.t0 = w.u.sp.tile0 + w.k0;
        w.n = max(0, min(w.k1, w.u.sp.count) - w.k0);
    };
    auto step = [&](Slice &w) -> bool {      // to the next unit of the share
        w.x = w.u.at + w.k1;
        if (w.x >= x1) return false;
        line.next(w.u);
        cut(w);
        return true;
    };
    Slice w0;
    if (works) {
        w0.u = line.find(x0, lane);
        w0.x = x0;
        cut(w0);
    }

    if (!works) {
        // (no unit: on to the end, where the pair leaves together)
    } else if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            // The MMA warp issues Q K^T(j + 1) before P V(j): K goes one tile ahead of V through the same list of tiles.
            struct Cursor { Slice w; int jj, g, ui; bool valid; };
            auto settle = [&](Cursor &c) {          // at or behind c.w: the next unit with a tile
                while (c.w.n == 0) {
                    if (!step(c.w)) { c.valid = false; return; }
                }
                c.jj = 0;
            };
            auto advance = [&](Cursor &c) {
                ++c.g;
                if (++c.jj == c.w.n) {
                    ++c.ui;
                    if (!step(c.w)) c.valid = false; else settle(c);
                }
            };
            // boxes of the 64 keys from key0 on that hold a key below hi
            auto boxes = [&](int key0, int hi) -> int { return (min(max(hi - key0, 0), 64) + box - 1) / box; };
            auto row_of = [&](const Cursor &c, int key) -> int {
                int page = page_at(p.q, p.g.n_pages, c.w.u.s.b, key >> p.g.log_p);
                if (page < 0) { page = 0; bad_unit[c.ui & 7] = (uint32_t)c.ui + 1u; }
                return (int)(page_row(p.g, page, c.w.u.h)) + (key & (p.g.P - 1));
            };
            bool ok = true;
            auto issue_k = [&](const Cursor &c) {
                const int st = c.g % NST, key0 = (c.w.t0 + c.jj) * kChunkKeys, hi = c.w.u.sp.hi;
                if (c.g >= NST) ok = wait(L::KEMPTY + st, (uint32_t)(c.g / NST - 1) & 1u, 1);
                if (!ok) return;
                if (rank == 0) mbar_expect_tx(bar(L::KFULL + st), (uint32_t)((boxes(key0, hi) + boxes(key0 + 64, hi)) * box * 128 * CH));
                const int mine = key0 + 64 * (int)rank, nb = boxes(mine, hi);
                for (int i = 0; i < nb; ++i) {
                    const int row = row_of(c, mine + i * box);
#pragma unroll
                    for (int ch = 0; ch < CH; ++ch)
                        tma2_load_2d(base + L::OFF_K + st * L::K_STAGE + ch * (64 * 128) + i * box * 128, &tm_k, bar(L::KFULL + st) & kPeerBitMask, ch * 64, row);
                }
            };
            auto issue_q = [&](const Cursor &c) {
                if (c.ui >= 1) ok = wait(L::QEMPTY, (uint32_t)(c.ui - 1) & 1u, 2);
                if (!ok) return;
                const uint32_t bytes = (uint32_t)(G * tile_tokens * 128 * CH);
                if (rank == 0) mbar_expect_tx(bar(L::QFULL), 2 * bytes);
                const int t = c.w.u.s.row0 + (2 * c.w.u.tile + (int)rank) * tile_tokens;
                for (int ch = 0; ch < CH; ++ch) tma2_load_3d(base + L::OFF_Q + ch * (128 * 128), &tm_q, bar(L::QFULL) & kPeerBitMask, ch * 64, c.w.u.h * G, t);
            };
            auto issue_v = [&](const Cursor &c) {
                const int st = c.g % NST, key0 = (c.w.t0 + c.jj) * kChunkKeys, hi = c.w.u.sp.hi;
                if (c.g >= NST) ok = wait(L::VEMPTY + st, (uint32_t)(c.g / NST - 1) & 1u, 3);
                if (!ok) return;
                const int nb[2] = {boxes(key0, hi), boxes(key0 + 64, hi)};
                int rows[2][4];
                const bool holds = D == HD || rank == 0;          // (heads of 64: the upper columns are nobody's)
                for (int hh = 0; hh < 2; ++hh)
                    for (int i = 0; i < nb[hh]; ++i) rows[hh][i] = row_of(c, key0 + 64 * hh + i * box);
                mbar_expect_tx(bar(L::VLAND + st), holds ? (uint32_t)((nb[0] + nb[1]) * box * 128 * VCH) : 0u);
                if (!holds) return;
                for (int hh = 0; hh < 2; ++hh)
                    for (int i = 0; i < nb[hh]; ++i)
#pragma unroll
                        for (int ch = 0; ch < VCH; ++ch)
                            tma_load_2d(base + L::OFF_V + st * L::V_STAGE + ch * (128 * 128) + hh * (64 * 128) + i * box * 128, &tm_v, bar(L::VLAND + st), ((int)rank * VCH + ch) * 64, rows[hh][i]);
            };
            Cursor ck;
            ck.w = w0; ck.jj = 0; ck.g = 0; ck.ui = 0; ck.valid = true;
            settle(ck);
            Cursor cv = ck;
            if (ck.valid) { issue_k(ck); if (ok) issue_q(ck); advance(ck); }
            while (cv.valid && ok) {
                const bool k_now = ck.valid;
                if (k_now) { issue_k(ck); if (!ok) break; }
                issue_v(cv);
                if (!ok) break;
                if (k_now) {
                    if (ck.jj == 0) { issue_q(ck); if (!ok) break; }
                    advance(ck);
                }
                advance(cv);
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (leader CTA; the warp stays converged, one lane issues) ----------------
        if (rank == 0) {
            constexpr uint16_t both = 3;
            constexpr uint32_t idesc_qk = umma_idesc_bf16(256, kChunkKeys, false), idesc_pv = umma_idesc_bf16(256, HD, true);
            const uint64_t qdesc0 = umma_desc_sw128(base + L::OFF_Q, 16, 1024), kdesc0 = umma_desc_sw128(base + L::OFF_K, 16, 1024);
            const uint64_t vdesc0 = umma_desc_sw128(base + L::OFF_V, 128 * 128, 1024);
            auto qk = [&](int gi, bool last) -> bool {
                const int st = gi % NST, buf = gi & 1;
                if (!wait(L::KFULL + st, (uint32_t)(gi / NST) & 1u, 4)) return false;
                tc_fence_after();
                uint64_t qd = qdesc0, kd = kdesc0;
                umma_desc_advance(kd, (uint32_t)st * L::K_STAGE);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    umma2_ss_elect(tmem_base + kColS + buf * kChunkKeys, qd, kd, idesc_qk, kk > 0 ? 1u : 0u);
                    umma_desc_advance(qd, (kk & 3) == 3 ? 128 * 128 - 96 : 32);
                    umma_desc_advance(kd, (kk & 3) == 3 ? 64 * 128 - 96 : 32);
                }
                umma2_commit_mc_elect(bar(L::KEMPTY + st), both);
                umma2_commit_mc_elect(bar(L::SFULL + buf), both);
                if (last) umma2_commit_mc_elect(bar(L::QEMPTY), both);
                return true;
            };
            bool ok = true;
            int gt = 0, ui = 0;
            Slice w = w0;
            do {
                const int n = w.n;
                if (n == 0) continue;
                ok = wait(L::QFULL, (uint32_t)ui & 1u, 5) && qk(gt, n == 1);
                for (int jj = 0; jj < n && ok; ++jj) {
                    const int gi = gt + jj, st = gi % NST, buf = gi & 1;
                    if (jj + 1 < n) { ok = qk(gi + 1, jj + 2 == n); if (!ok) break; }
                    ok = wait(L::PFULL + buf, (uint32_t)(gi >> 1) & 1u, 6);
                    if (ok && jj == 0 && ui >= 1) ok = wait(L::OFREE, (uint32_t)(ui - 1) & 1u, 7);
                    if (!ok) break;
                    tc_fence_after();
                    uint64_t vd = vdesc0;
                    umma_desc_advance(vd, (uint32_t)st * L::V_STAGE);
                    // (a second half past the last key: its P is zero and its V was never loaded)
                    const int ksteps = (w.t0 + jj) * kChunkKeys + 64 < w.u.sp.hi ? kChunkKeys / 16 : kChunkKeys / 32;
#pragma unroll 4
                    for (int kk = 0; kk < ksteps; ++kk) {
                        umma2_ts_elect(tmem_base, tmem_base + kColS + buf * kChunkKeys + kk * 8, vd, idesc_pv, jj > 0 || kk > 0 ? 1u : 0u);
                        umma_desc_advance(vd, 16 * 128);
                    }
                    umma2_commit_mc_elect(bar(L::VEMPTY + st), both);
                    umma2_commit_mc_elect(bar(L::PVDONE + buf), both);
                }
                gt += n;
                ++ui;
            } while (ok && step(w));
        }
    } else {
        // ---------------- softmax, rescaling, results ----------------
        const int sw = warp - 2, half = sw >> 2;          // which 64 keys of the tile
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t leader_pfull[2] = {mapa(bar(L::PFULL), 0), mapa(bar(L::PFULL + 1), 0)};
        const uint32_t leader_ofree = mapa(bar(L::OFREE), 0);
        float *xmax = reinterpret_cast<float *>(smem + L::OFF_XMAX);         // [2 buffers][128 rows][2 halves]
        const int rows_here = tile_tokens * G;
        const int tid = threadIdx.x - 64;
        bool ok = true;
        int gt = 0, ui = 0;
        Slice w = w0;
        do {
            const PageSeq &s = w.u.s;
            const int token0 = (2 * w.u.tile + (int)rank) * tile_tokens;         // first of this CTA's rows
            const int t_row = token0 + row / G;
            const bool row_live = row < rows_here && t_row < s.n;
            const PageRange mine = page_range(s, p, min(t_row, s.n - 1), min(t_row, s.n - 1));
            const bool whole = w.k0 == 0 && w.k1 == w.u.cost;
            // keys that every row of the pair sees (either CTA's V meets the rows of both)
            const int all_lo = page_range(s, p, min(s.n, 2 * (w.u.tile + 1) * tile_tokens) - 1, 0).lo, all_hi = page_range(s, p, 0, 2 * w.u.tile * tile_tokens).hi;
            const int slot = 2 * pair + (w.k0 == 0 ? 1 : 0);
            float m_ref = -INFINITY, l = 0.f;
            auto tile = [&](auto mode_c, const int jj) {
                constexpr bool FULL = decltype(mode_c)::value == 0;
                constexpr bool DEAD = decltype(mode_c)::value == 2;        // a half past the unit's last key: no logits to read and no P to write
                const int gi = gt + jj, buf = gi & 1, st = gi % NST;
                const uint32_t vph = (uint32_t)(gi / NST) & 1u;
                const int key0 = (w.t0 + jj) * kChunkKeys + half * 64;
                uint64_t smask = ~0ull, tmask = ~0ull;          // keys that this row sees; keys that lie below the unit's last one
                if constexpr (!FULL) {
                    smask = bits64(mine.lo - key0, mine.hi - key0);
                    tmask = bits64(0, w.u.sp.hi - key0);
                }
                float x[64];
                if constexpr (!DEAD) {
                    ok = ok && wait(L::SFULL + buf, (uint32_t)(gi >> 1) & 1u, 8);
                    tc_fence_after();
                    uint32_t r[64];
                    tmem_ld32(tmem_base + lane_addr + kColS + buf * kChunkKeys + half * 64, *reinterpret_cast<uint32_t(*)[32]>(r));
                    tmem_ld32(tmem_base + lane_addr + kColS + buf * kChunkKeys + half * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 64; ++c) x[c] = __uint_as_float(r[c]);
                }
                if constexpr (!FULL && !DEAD) {
                    // Keys behind the last one count as zeros in V (a weight of 0 does not make a stale NaN one); a key that only some rows see must be
                    // finite, or the sequence is done again row by row. All 128 threads of the half share the rows: half a row's columns each.
                    ok = ok && wait(L::VLAND + st, vph, 9);
                    const int key = key0 + (row & 63);
                    const bool dead = !((tmask >> (row & 63)) & 1ull);
                    const bool some = !dead && (key < all_lo || key >= all_hi);
                    uint4 *vr0 = reinterpret_cast<uint4 *>(smem + L::OFF_V + st * L::V_STAGE + (half * 64 + (row & 63)) * 128) + (row >> 6) * 4;
                    if (dead) {
#pragma unroll
                        for (int c = 0; c < VCH; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) vr0[c * (128 * 128 / 16) + i] = make_uint4(0, 0, 0, 0);
                    } else if (some && (D == HD || rank == 0)) {
                        uint32_t odd = 0;
#pragma unroll
                        for (int c = 0; c < VCH; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint4 v = vr0[c * (128 * 128 / 16) + i];
                                const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int e = 0; e < 4; ++e) odd |= ((q[e] & 0x7f80u) == 0x7f80u) | ((q[e] & 0x7f800000u) == 0x7f800000u);
                            }
                        if (odd) part.careful[s.b] = 1;
                    }
                }
                float mx = -INFINITY;
                if constexpr (!DEAD) {
                    if (!FULL && smask != ~0ull) {
                        const uint32_t lo = (uint32_t)smask, hi = (uint32_t)(smask >> 32);
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            if (!(lo & (1u << c))) x[c] = -INFINITY;
                            if (!(hi & (1u << c))) x[32 + c] = -INFINITY;
                        }
                    }
                    float mx4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                    for (int c = 4; c + 7 < 64; c += 8) {
                        mx4[0] = max3_nan_f32(mx4[0], x[c], x[c + 1]); mx4[1] = max3_nan_f32(mx4[1], x[c + 2], x[c + 3]);
                        mx4[2] = max3_nan_f32(mx4[2], x[c + 4], x[c + 5]); mx4[3] = max3_nan_f32(mx4[3], x[c + 6], x[c + 7]);
                    }
                    mx4[0] = max3_nan_f32(mx4[0], x[60], x[61]); mx4[1] = max3_nan_f32(mx4[1], x[62], x[63]);
                    mx = max_nan_f32(max_nan_f32(mx4[0], mx4[1]), max_nan_f32(mx4[2], mx4[3]));
                    if (!(mx < INFINITY)) l = __int_as_float(0x7fc00000);      // (a logit that is NaN or +inf; the polynomial below would lose it)
                }
                // The two threads of a row agree on its maximum. Past this barrier both have their logits in registers, so P may overwrite them.
                xmax[(buf * 128 + row) * 2 + half] = mx;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                mx = fmaxf(xmax[(buf * 128 + row) * 2], xmax[(buf * 128 + row) * 2 + 1]);
                if (jj == 0) m_ref = mx;
                else {
                    const bool grow = (mx - m_ref) * part.scale_log2 > kChunkGrow;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float alpha = grow ? ex2((m_ref - mx) * part.scale_log2) : 1.f;
                        if (grow) m_ref = mx;
                        l *= alpha;
                        ok = ok && wait(L::PVDONE + ((gi - 1) & 1), (uint32_t)((gi - 1) >> 1) & 1u, 10);
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < HD / 64; ++c) {
                            uint32_t o[32];
                            const uint32_t o_addr = tmem_base + lane_addr + half * (HD / 2) + c * 32;
                            tmem_ld32(o_addr, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st32(o_addr, o);
                        }
                        tmem_wait_st();
                    }
                }
                if constexpr (!DEAD) {
                    const float mr = m_ref == -INFINITY ? 0.f : m_ref * part.scale_log2;
                    const uint64_t sc2 = pack_f32x2(part.scale_log2, part.scale_log2), nm2 = pack_f32x2(-mr, -mr);
                    const Ex2PolyConsts pk = ex2_poly_consts();
                    uint64_t sum2[4] = {0ull, 0ull, 0ull, 0ull};
                    uint32_t packed[32];
#pragma unroll
                    for (int c = 0; c < 64; c += 2) {
                        float y0, y1, p0, p1;
                        unpack_f32x2(fma_f32x2(pack_f32x2(x[c], x[c + 1]), sc2, nm2), y0, y1);
                        if (((c >> 1) & 7) < kChunkPoly) ex2_poly_f32x2(y0, y1, pk, p0, p1);
                        else { p0 = ex2(y0); p1 = ex2(y1); }
                        sum2[(c >> 1) & 3] = add_f32x2(sum2[(c >> 1) & 3], pack_f32x2(p0, p1));
                        packed[c >> 1] = pack_bf16(p0, p1);
                    }
                    float a, b;
                    unpack_f32x2(add_f32x2(add_f32x2(sum2[0], sum2[1]), add_f32x2(sum2[2], sum2[3])), a, b);
                    if (!FULL && smask == 0ull) a = b = 0.f;              // (the polynomial gives masked keys 2^-125: a row that sees nothing has no sum)
                    l += a + b;
                    if (!FULL && smask != ~0ull) {
                        // ... and their weights must be exactly 0
#pragma unroll
                        for (int c = 0; c < 64; c += 2) {
                            if (((c >> 1) & 7) < kChunkPoly) {
                                const uint32_t two = (uint32_t)(smask >> c) & 3u;
                                packed[c >> 1] &= ((two & 1u) ? 0x0000FFFFu : 0u) | ((two & 2u) ? 0xFFFF0000u : 0u);
                            }
                        }
                    }
                    tmem_st32(tmem_base + lane_addr + kColS + buf * kChunkKeys + half * 32, packed);
                    tmem_wait_st();
                }
                if (FULL || DEAD) ok = ok && wait(L::VLAND + st, vph, 11);       // (the arrival below says that this CTA's V is in place, too)
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(leader_pfull[buf]);
            };
            for (int jj = 0; jj < w.n; ++jj) {
                const int key0 = (w.t0 + jj) * kChunkKeys + half * 64;
                if (key0 >= all_lo && key0 + 64 <= all_hi) tile(std::integral_constant<int, 0>{}, jj);
                else if (key0 < w.u.sp.hi) tile(std::integral_constant<int, 1>{}, jj);
                else tile(std::integral_constant<int, 2>{}, jj);
            }
            gt += w.n;
            const int g_last = gt - 1;
            if (w.n > 0) {
                ok = ok && wait(L::PVDONE + (g_last & 1), (uint32_t)(g_last >> 1) & 1u, 12);
                if (bad_unit[ui & 7] == (uint32_t)ui + 1u || !ok) l = __int_as_float(0x7fc00000);
            }
            // the row's sums, through the maxima's buffer that the last tile did not use
            float *xsum = xmax + ((g_last & 1) ^ 1) * 256;
            xsum[half * 128 + row] = l;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            l += xsum[(half ^ 1) * 128 + row];
            tc_fence_after();
            if (w.n > 0 && tid == 0 && bad_unit[ui & 7] == (uint32_t)ui + 1u) report_bad_page(p.g.status, s.b);
            const float inv = l == 0.f || w.n == 0 || (m_ref == -INFINITY && l == l) ? 0.f : 1.f / l;
            const bool unit_live = token0 < s.n;             // (a pair's second tile may have no row)
            if (!whole) {
                if (half == 0 && row_live) part.ml[(size_t)slot * kChunkRows + rank * 128 + row] = make_float2(m_ref == -INFINITY ? -INFINITY : m_ref * part.scale_log2, l);
#pragma unroll 1
                for (int c = 0; c < D / 64; ++c) {
                    uint32_t o[32];
                    const int col = half * (D / 2) + c * 32;
                    tmem_ld32(tmem_base + lane_addr + col, o);
                    tmem_wait_ld();
                    if (c == D / 64 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0 && w.n > 0) mbar_arrive_cluster(leader_ofree);
                    }
                    if (row_live) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) st_global_v8(partial8(part, slot, D, (int)rank * 128 + row, col + 8 * i), *reinterpret_cast<const uint32_t(*)[8]>(o + 8 * i));
                    }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");        // every thread has read the sums before the next unit's maxima land there
                if (w.k0 == 0 && threadIdx.x == 64 && rank == 0) {
                    const int f = 2 * w.u.tile * rows_here;
                    PageSplit m2 = {s.b, s.row0, f, min(2 * rows_here, s.n * G - f), w.u.h, page_owner(w.u.at + w.u.cost - 1, total, nc), rows_here, 0};
                    part.meta[pair] = m2;
                }
            } else {
                // O / l, 64 columns at a time through the two halves of the staging area, then whole 128-byte pieces of rows to memory
                size_t dst[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = (tid >> 3) + 32 * k, t = token0 + r / G;
                    dst[k] = unit_live && r < rows_here && t < s.n ? ((size_t)(s.row0 + t) * p.g.Hq + w.u.h * G + r % G) * D + (tid & 7) * 8 : ~(size_t)0;
                }
#pragma unroll 1
                for (int rnd = 0; rnd < D / 64; ++rnd) {
                    uint32_t o[32];
                    tmem_ld32(tmem_base + lane_addr + rnd * 64 + half * 32, o);
                    tmem_wait_ld();
                    if (rnd == D / 64 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0 && w.n > 0) mbar_arrive_cluster(leader_ofree);
                    }
                    uint8_t *srow = smem + L::OFF_STAGE + (rnd & 1) * (128 * 128) + row * 128;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float f[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] = inv == 0.f ? 0.f : __uint_as_float(o[8 * c + k]) * inv;      // (the accumulator of a unit without keys was never written)
                        *reinterpret_cast<uint4 *>(srow + (((half * 4 + c) ^ (row & 7)) << 4)) =
                            make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
                    }
                    asm volatile("bar.sync 1, 256;" ::: "memory");
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = (tid >> 3) + 32 * k;
                        if (dst[k] != ~(size_t)0)
                            *reinterpret_cast<uint4 *>((__nv_bfloat16 *)p.out + dst[k] + rnd * 64) =
                                *reinterpret_cast<const uint4 *>(smem + L::OFF_STAGE + (rnd & 1) * (128 * 128) + r * 128 + (((tid & 7) ^ (r & 7)) << 4));
                    }
                }
                if (D == 64) asm volatile("bar.sync 1, 256;" ::: "memory");      // (one round: its half, and the sums, may not be overwritten before they are read)
            }
            if (w.n > 0) ++ui;
        } while (step(w));
    }

    tc_fence_before();
    __syncthreads();
    cluster_arrive_relaxed();
    cluster_wait();   // neither CTA leaves while its partner can still touch its shared memory or barriers
    if (warp == 1) tmem_dealloc2(tmem_base, 512);
}

// The pages of a layer that the sequences' new tokens see, widened to bf16 (exact) at the same place of a layer of bf16 pages.
template <int FMT>
__global__ void __launch_bounds__(256)
page_widen_kernel(const PageAttention p, __nv_bfloat16 *k_wide, __nv_bfloat16 *v_wide)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const PageGeom &g = p.g;
    const int pieces = g.d >> 4, per_page = g.Hkv * g.P * pieces;       // pieces of 16 elements
    for (int b = blockIdx.y; b < p.q.B; b += gridDim.y) {
        const PageSeq s = page_seq(p, b);
        if (s.n == 0) continue;
        const PageRange r = page_range(s, p, 0, s.n - 1);
        const int first = r.lo >> g.log_p, last = (r.hi + g.P - 1) >> g.log_p;
        const long long n = (long long)max(0, last - first) * per_page;
        for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
            const int page = page_at(p.q, g.n_pages, b, first + (int)(i / per_page));
            if (page < 0) continue;                   // (reported by the kernel that reads it)
            const int in_page = (int)(i % per_page);
            const size_t row = (size_t)page * g.Hkv * g.P + in_page / pieces, at = row * g.d + (in_page % pieces) * 16;
            const uint4 kw = *reinterpret_cast<const uint4 *>((const uint8_t *)g.k + at), vw = *reinterpret_cast<const uint4 *>((const uint8_t *)g.v + at);
            const uint32_t ks = exponent_bf16x2(g.ke[row]), vs = exponent_bf16x2(g.ve[row]);
            auto put = [&](const uint4 &q, uint32_t sc, __nv_bfloat16 *dst) {
                const uint32_t in[4] = {q.x, q.y, q.z, q.w};
                uint32_t o[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[2 * e] = bf16x2_mul(bytes_to_bf16x2<FMT, 0, 1>(in[e], in[e]), sc);
                    o[2 * e + 1] = bf16x2_mul(bytes_to_bf16x2<FMT, 2, 3>(in[e], in[e]), sc);
                }
                st_global_v8(dst, o);
            };
            put(kw, ks, k_wide + at);
            put(vw, vs, v_wide + at);
        }
    }
}

bool page_chunk_takes(int dtype, int G, int d) { return dtype == REFLEX_DTYPE_BF16 && d >= 64 && G <= 128; }

cudaError_t launch_page_widen(const PageAttention &a, void *k_wide, void *v_wide, int format, int sm_count, cudaStream_t st)
{
    const int by = std::min(a.q.B, 64);
    const dim3 grid((unsigned)std::max(1, 8 * sm_count / by), (unsigned)by);
    count_launch();
    if (format == REFLEX_PAGE_E4M3) page_widen_kernel<REFLEX_PAGE_E4M3><<<grid, 256, 0, st>>>(a, (__nv_bfloat16 *)k_wide, (__nv_bfloat16 *)v_wide);
    else page_widen_kernel<REFLEX_PAGE_INT8><<<grid, 256, 0, st>>>(a, (__nv_bfloat16 *)k_wide, (__nv_bfloat16 *)v_wide);
    return cudaGetLastError();
}

template <int HD, int D>
static cudaError_t launch_chunk(const PageAttention &a, const PagePartials &part, const void *k, const void *v, int pairs, cudaStream_t st)
{
    using L = Chunk<HD, D>;
    static std::atomic<unsigned long long> done{0};
    cudaError_t e = once_per_device(done, [] { return cudaFuncSetAttribute(page_chunk_kernel<HD, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::TOTAL); });
    if (e != cudaSuccess) return e;
    const int G = a.g.Hq / a.g.Hkv, tokens = 128 / G, box = std::min(a.g.P, 64);
    const int rows = a.g.n_pages * a.g.Hkv * a.g.P;
    CUtensorMap tq, tk, tv;
    const cuuint64_t qd[3] = {(cuuint64_t)D, (cuuint64_t)a.g.Hq, (cuuint64_t)a.n_rows}, qs[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.g.Hq * D * 2};
    const cuuint32_t qb[3] = {64, (cuuint32_t)G, (cuuint32_t)tokens};
    const cuuint64_t kd[2] = {(cuuint64_t)D, (cuuint64_t)rows}, ks[1] = {(cuuint64_t)D * 2};
    const cuuint32_t kb[2] = {64, (cuuint32_t)box};
    if (!encode_map_bf16(&tq, a.qry, 3, qd, qs, qb) || !encode_map_bf16(&tk, k, 2, kd, ks, kb) || !encode_map_bf16(&tv, v, 2, kd, ks, kb)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3(kChunkThreads);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    count_launch();
    return cudaLaunchKernelEx(&cfg, page_chunk_kernel<HD, D>, tq, tk, tv, a, part, tokens, box);
}

cudaError_t launch_page_chunk(const PageAttention &a, const PagePartials &part, const void *k, const void *v, int pairs, cudaStream_t st)
{
    if (a.g.d == 64) return launch_chunk<128, 64>(a, part, k, v, pairs, st);
    if (a.g.d == 128) return launch_chunk<128, 128>(a, part, k, v, pairs, st);
    return launch_chunk<256, 256>(a, part, k, v, pairs, st);
}

}  // namespace reflex
