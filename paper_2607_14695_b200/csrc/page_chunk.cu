// Attention of a chunk of new tokens over pages (reflex_pages_attention) on the tensor cores: tcgen05.mma.cta_group::2, M = 256.
//
// A pair of CTAs takes 256 (token, head) rows of a sequence and KV head, 128 each, and walks the keys in tiles of 128. Of every tile a CTA holds half:
// 64 keys of K, and half of the columns of V; TMA brings them from the pages, one box per page (or per 64 tokens of a larger page), to
// where the swizzled tile has them. S = Q K^T and O = P V accumulate in tensor memory; P (bf16) is written over the logits it came from and is
// the A operand of P V from there. Per CTA:
//   warps 0, 2   TMA producers: its Q tile and its half of K; its columns of V. Warp 0 walks the pair's share of the work and lists its units for the others.
//   warps 1, 3   MMA issuers (leader CTA): Q K^T runs one tile (two at head_dim <= 128) ahead of P V
//   warps 4..    softmax: two threads per row, 64 keys each, eight warps a tile. At head_dim 128 and 64 there are two such groups, which take the tiles
//                in turn: each then has the time of two tiles for its chain of loads, maximum, exponentials and stores, and a scheduler
//                has four of its warps. The threads of a row agree on the reference maximum at one named barrier per 32 rows, where the group
//                that has had the tile before leaves the row's reference, too; O is rescaled only where it has grown by more than 2^8.
// What bounds it: at head_dim 256 the tensor pipe (2048 of some 2350 cycles a tile; with set-up, ends of units and the uneven last tiles it is busy for 67
// % of the launch; operand reads then take two thirds of the shared memory's bandwidth), at 128 and 64 the softmax (some 700 issue slots a scheduler and
// tile, which the helper warps need as well; a quarter of the exponentials by a polynomial instead of the special-function unit cost more of them than the
// unit saved: 310 us for 301 at 4 x 4160 causal tokens, 16 heads of 128). Measured in a warm graph (in brackets a pass among others, caches cold): that
// prefill in 283 to 292 us (327 to 339), 1.0 PFLOP/s of the products that its mask leaves; a frame of 256 tokens of each of 16 sequences of 3376, 8 heads
// of 256 on one KV head, 8-bit pages, in 111 to 113 us (122 to 127) with widening (15) and merging (12). Heads of 64 run as heads of 128 whose upper chunk
// is left out of Q K^T and whose upper columns of O are never read: P V costs twice, underneath the softmax.
//
// The grid is one pair per SM pair; the tiles of all units form one line that the pairs share evenly (PageLine), so uneven sequences, causal masks and single
// sequences fill the device alike. A unit that more than one pair works on leaves fp32 partials for page_merge_kernel.
// 8-bit pages are first widened to bf16, exactly, into one layer's worth of workspace (page_widen_kernel): a page is used by every row tile and by both
// CTAs of a pair. (Unpacking it inside each has not been built: at head_dim 128 and 64 the softmax takes the issue slots, at 256 there are slots
// left, 0.27 issues a cycle, and it is the widening's 15 us that it could save.)
//
// Every wait is bounded; one that runs out is reported in the status word and makes the results NaN.
#include <math.h>

#include <algorithm>

#include "page_attention.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

using namespace ptx;

constexpr int kChunkKeys = 128;
constexpr int kChunkRows = 256;                // of a unit
constexpr unsigned long long kChunkWaitNs = 1000000000ull;
constexpr float kChunkGrow = 8.0f;             // log2 units: O is rescaled only where a maximum grows by more than 2^8

// A unit costs SET_UP blocks before its first tile: what its Q, its masks and its results take, in tiles. (A share that ends among them
// leaves the unit to the next pair.)
struct ChunkSpan { int tile0, tiles, lo, hi, count; };    // key tiles [tile0, tile0 + tiles), keys [lo, hi); blocks
template <int SET_UP>
struct ChunkSpanOf {
    const PageAttention &p;
    int tokens;                                // of a unit
    __device__ __forceinline__ int tiles(const PageSeq &s) const { return (s.n + tokens - 1) / tokens; }
    __device__ __forceinline__ ChunkSpan operator()(const PageSeq &s, int tile) const
    {
        const PageRange r = page_range(s, p, tile * tokens, min(s.n, (tile + 1) * tokens) - 1);
        ChunkSpan c;
        c.tile0 = r.lo / kChunkKeys;
        c.lo = r.lo; c.hi = r.hi;
        c.tiles = r.hi > r.lo ? (r.hi + kChunkKeys - 1) / kChunkKeys - c.tile0 : 0;
        c.count = SET_UP + max(1, c.tiles);
        return c;
    }
};

// A pair's share of a unit, as warp 0 lists it for the others: tiles of keys [t0, t0 + n); none at all behind the last one (n = -1).
struct ChunkUnit {
    int b, row0, n_rows, len;      // the sequence
    int token, h;                  // first token of the pair's rows, KV head
    int t0, n, lo, hi;             // keys [lo, hi) of these tiles: no row sees others
    int slot;                      // of its partial result, -1: the whole unit is the pair's
    int unused[5];
};
static_assert(sizeof(ChunkUnit) == 64, "list of units");

template <int HD, int D> struct Chunk {
    static constexpr int CH = D / 64;                           // 64-column chunks of Q and K
    static constexpr int VCH = HD / 128;                        // chunks of V of this CTA
    static constexpr int NST = HD == 256 ? 2 : 4;               // stages of K, and of V
    static constexpr int NS = HD == 256 ? 2 : 3;                // buffers of logits and weights in tensor memory
    static constexpr bool SPLIT = HD == 128;                    // a warp of its own for either product
    static constexpr int NG = HD == 256 ? 1 : 2;                // softmax groups of 8 warps
    static constexpr int THREADS = 128 + 256 * NG;
    static constexpr int NU = 8;                                // units in the list
    static constexpr int SET_UP = HD == 256 ? 6 : 4;            // (attention of 16 frames at 256: 2 % faster with 6 than with 4; causal prefill at 128: 281 with 4, 288 with 6)
    static constexpr int QFULL = 0, QEMPTY = 1, KFULL = 2, KEMPTY = KFULL + NST, VLAND = KEMPTY + NST, VEMPTY = VLAND + NST, SFULL = VEMPTY + NST, PFULL = SFULL + NS,
                         PVDONE = PFULL + NS, OFREE = PVDONE + 4, UFULL = OFREE + 1, UEMPTY = UFULL + NU, COUNT = UEMPTY + NU;
    static constexpr uint32_t BAR_BYTES = (8 * COUNT + 104 + 127) / 128 * 128;                // ... tensor memory's address, abort flag, bad units, tiles
    static constexpr uint32_t Q_BYTES = CH * 128 * 128;
    static constexpr uint32_t K_STAGE = CH * 64 * 128;
    static constexpr uint32_t V_STAGE = VCH * 128 * 128;
    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_K = OFF_Q + Q_BYTES;
    static constexpr uint32_t OFF_V = OFF_K + NST * K_STAGE;
    static constexpr uint32_t OFF_STAGE = OFF_V + NST * V_STAGE;      // of each group: 128 rows x 64 columns of the result
    static constexpr uint32_t OFF_BAR = OFF_STAGE + NG * 128 * 128;
    static constexpr uint32_t OFF_UNITS = OFF_BAR + BAR_BYTES;       // [NU] ChunkUnit
    static constexpr uint32_t OFF_MAX = OFF_UNITS + NU * 64;          // [2 tiles of each group][128 rows][2 halves] maxima of the logits
    static constexpr uint32_t OFF_REF = OFF_MAX + 2 * NG * 128 * 2 * 4;    // [NG][128] reference maxima, as a group leaves them to the other one
    static constexpr uint32_t OFF_SUM = OFF_REF + NG * 128 * 4;       // [2 units][2 NG][128] (reference, sum) of a row's threads
    static constexpr uint32_t OFF_ROWS = OFF_SUM + 2 * 2 * NG * 128 * 8;
    static constexpr uint32_t NEED = OFF_ROWS + 128 * 4;
    static constexpr uint32_t TOTAL = NEED + 1024 > 232448 ? 232448 : NEED + 1024;
    static_assert(NEED <= TOTAL, "shared memory");
};

// bits [lo, hi) of a 64-bit word, whatever lo and hi are
__device__ __forceinline__ uint64_t bits64(int lo, int hi)
{
    lo = max(lo, 0); hi = min(hi, 64);
    if (hi <= lo) return 0ull;
    return (hi >= 64 ? ~0ull : (1ull << hi) - 1ull) & ~((1ull << lo) - 1ull);
}

template <int HD, int D>
__global__ void __launch_bounds__(Chunk<HD, D>::THREADS, 1)         // clusters of two
page_chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const PageAttention p, const PagePartials part, int tile_tokens, int box)
{
    using L = Chunk<HD, D>;
    constexpr int CH = L::CH, VCH = L::VCH, NST = L::NST, NS = L::NS, NG = L::NG;
    constexpr bool SPLIT = L::SPLIT;
    constexpr uint32_t kColS = HD;
    static_assert(HD + L::NS * kChunkKeys <= 512, "tensor memory");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw_addr);
    const uint32_t bar0 = base + L::OFF_BAR;
    auto bar = [&](int i) -> uint32_t { return bar0 + 8u * (uint32_t)i; };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::OFF_BAR + 8 * L::COUNT);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    volatile uint32_t *bad_unit = tmem_slot + 2;          // [8]: number (from 1) of the last unit of that residue which met a bad page
    volatile uint32_t *tile_info = bad_unit + 8;           // [16]: (g + 1) << 4 and what the issuers have to know of tile g (written by the leader's K producer ahead of the arrival on KFULL)
    constexpr uint32_t kFirst = 1u, kLast = 2u, kSecond = 4u, kEnd = 8u;       // of its unit; has live keys in its second half; there is no such tile
    if ((base - raw_addr) + L::NEED > L::TOTAL) {          // (the same for every CTA: all of them leave)
        if (threadIdx.x == 0) report_page_wait(p.g.status, kSitePageChunk + 15u);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int G = p.g.Hq / p.g.Hkv;
    // The K producer walks the line. It looks for its pair's place first of all: what the line is made of does not change under this kernel (only the widening of
    // pages runs beside its start).
    using Line = PageLine<ChunkSpanOf<L::SET_UP>>;
    Line line{p, {p, 2 * tile_tokens}};
    typename Line::Place place;
    int total = 0, x0 = 0, x1 = 0, nc = 0;
    if (warp == 0) {
        total = line.begin(lane);
        nc = min(pairs, total);
        const PageShares shares(total, max(1, nc));
        if (pair < nc) {
            x0 = shares.of(pair); x1 = shares.of(pair + 1);
            place = line.find(x0, lane);
        }
    }

    if (threadIdx.x == 0) {
        // (weights, and the accumulator's release: an arrival per warp of a group of either CTA; a unit of the list: of every softmax warp here)
        for (int i = 0; i < L::COUNT; ++i)
            mbar_init(bar(i), i >= L::PFULL && i < L::PFULL + NS || i == L::OFREE ? 16u : i >= L::UEMPTY ? 8u * NG : 1u);
        *abort_flag = 0u;
        for (int i = 0; i < 24; ++i) bad_unit[i] = 0u;           // (and tile_info)
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
        report_page_wait(p.g.status, kSitePageChunk + code);
        return false;
    };

    constexpr uint16_t both = 3;               // CTAs of the pair, for commits
    auto all = [&](bool good) -> bool { return __all_sync(0xffffffffu, good); };
    const ChunkUnit *units = reinterpret_cast<const ChunkUnit *>(smem + L::OFF_UNITS);
    auto unit_ready = [&](int i) -> bool { return all(wait(L::UFULL + i % L::NU, (uint32_t)(i / L::NU) & 1u, 1)); };      // the i-th of the list may be read

    // the tiles of the share as one sequence: number g, tile jj of unit number i of the list, ui of those that have keys
    struct Cursor { int b, h, t0, n, lo, hi, q_row, jj, g, ui, i; bool valid; };
    auto settle = [&](Cursor &c) {          // the i-th unit, or the first one behind it with a tile
        for (;; ++c.i) {
            c.valid = unit_ready(c.i);
            if (!c.valid) return;
            const ChunkUnit &u = units[c.i % L::NU];
            c.n = u.n;
            if (c.n != 0) {
                c.valid = c.n > 0;
                c.b = u.b; c.h = u.h; c.t0 = u.t0; c.lo = u.lo; c.hi = u.hi;
                c.q_row = u.row0 + u.token + (int)rank * tile_tokens;
                c.jj = 0;
                return;
            }
        }
    };
    auto begin = [&]() -> Cursor {
        Cursor c = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, false};
        settle(c);
        return c;
    };
    auto advance = [&](Cursor &c) {
        ++c.g;
        if (++c.jj == c.n) { ++c.ui; ++c.i; settle(c); }
    };
    // Where a warp's tile of keys lies, box by box: lane i has the row of box i in the layer's pages (0 where it holds no key below the unit's
    // last, or where the table is wrong: `bad`, if one of its keys can be seen; pages in front of all windows may be gone). It is looked up a tile ahead, since a table entry takes some 500 cycles to come.
    const int per_half = 64 / box;               // boxes of 64 keys
    auto boxes = [&](int key0, int hi) -> int { return (min(max(hi - key0, 0), 64) + box - 1) / box; };
    auto look_up = [&](const Cursor &c, bool &bad) -> int {
        const int key = (c.t0 + c.jj) * kChunkKeys + lane * box;
        bad = false;
        if (!c.valid || lane >= 2 * per_half || key >= c.hi) return 0;
        const int page = page_at(p.q, p.g.n_pages, c.b, key >> p.g.log_p);
        bad = page < 0 && key + box > c.lo;
        return page < 0 ? 0 : (int)page_row(p.g, page, c.h) + (key & (p.g.P - 1));
    };

    if (warp == 0) {
        // ---------------- the list of units; Q and K by TMA (the warp stays converged, one lane issues) ----------------
        // A unit costs SET_UP blocks ahead of its tiles; a share that ends among them leaves the unit to the next pair.
        const PageShares shares(total, max(1, nc));
        ChunkUnit *list = reinterpret_cast<ChunkUnit *>(smem + L::OFF_UNITS);
        if (lane == 0 && rank == 0) part.meta[pair].b = -1;
        bool bad, ok = true;
        Cursor c = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, false};
        int x = x0;
        auto publish = [&](const ChunkUnit &u) {
            if (c.i >= L::NU) ok = ok && all(wait(L::UEMPTY + c.i % L::NU, (uint32_t)(c.i / L::NU - 1) & 1u, 13));
            if (ok && lane == 0) {
                list[c.i % L::NU] = u;
                mbar_arrive(bar(L::UFULL + c.i % L::NU));
            }
            ++c.i;
        };
        auto next_unit = [&] {                   // lists units up to the next one with a tile, or to the end
            c.valid = false;
            while (x < x1 && ok) {
                const int to = min(place.at + place.cost, x1);
                const int k0 = max(0, x - place.at - L::SET_UP), k1 = max(0, to - place.at - L::SET_UP);
                if (k1 > 0) {
                    const bool whole = k0 == 0 && k1 == place.cost - L::SET_UP;
                    const ChunkUnit u = {place.s.b, place.s.row0, place.s.n, place.s.len, place.tile * 2 * tile_tokens, place.h, place.sp.tile0 + k0, max(0, min(k1, place.sp.tiles) - k0), place.sp.lo, place.sp.hi,
                                         whole ? -1 : 2 * pair + (k0 == 0 ? 1 : 0), {0, 0, 0, 0, 0}};
                    publish(u);
                    if (k0 == 0 && !whole && rank == 0 && lane == 0) {
                        const int first = u.token * G;
                        const PageSplit m = {u.b, u.row0, first, min(2 * tile_tokens * G, u.n_rows * G - first), u.h, shares.owner(place.at + place.cost - 1), tile_tokens * G, 0};
                        part.meta[pair] = m;
                    }
                    c.b = u.b; c.h = u.h; c.t0 = u.t0; c.n = u.n; c.lo = u.lo; c.hi = u.hi;
                    c.q_row = u.row0 + u.token + (int)rank * tile_tokens;
                    c.jj = 0;
                    c.valid = u.n > 0 && ok;
                }
                x = to;
                if (x < x1) line.next(place);
                if (c.valid) return;
            }
            const ChunkUnit none = {0, 0, 0, 0, 0, 0, 0, -1, 0, 0, -1, {0, 0, 0, 0, 0}};
            publish(none);
        };
        next_unit();
        int row = look_up(c, bad);
        while (c.valid) {
            const int st = c.g % NST, key0 = (c.t0 + c.jj) * kChunkKeys, hi = c.hi;
            if (c.g >= NST) ok = wait(L::KEMPTY + st, (uint32_t)(c.g / NST - 1) & 1u, 1);
            if (!__all_sync(0xffffffffu, ok)) break;
            const int nb = boxes(key0 + 64 * (int)rank, hi);
            if (rank == 0 && lane == 0) {
                tile_info[c.g & 15] = ((uint32_t)c.g + 1u) << 4 | (c.jj == 0 ? kFirst : 0u) | (c.jj + 1 == c.n ? kLast : 0u) | (key0 + 64 < hi ? kSecond : 0u);
                mbar_expect_tx(bar(L::KFULL + st), (uint32_t)((boxes(key0, hi) + boxes(key0 + 64, hi)) * box * 128 * CH));
            }
            __syncwarp();
            const uint32_t dst = base + L::OFF_K + st * L::K_STAGE, full = bar(L::KFULL + st) & kPeerBitMask;
            for (int i = 0; i < nb; ++i) {
                const int r = __shfl_sync(0xffffffffu, row, (int)rank * per_half + i);
#pragma unroll
                for (int ch = 0; ch < CH; ++ch) tma2_load_2d_elect(dst + ch * (64 * 128) + i * box * 128, &tm_k, full, ch * 64, r);
            }
            if (c.jj == 0) {
                // the unit's Q, once the last Q K^T of the unit before has read the buffer
                if (c.ui >= 1) ok = wait(L::QEMPTY, (uint32_t)(c.ui - 1) & 1u, 2);
                if (!__all_sync(0xffffffffu, ok)) break;
                const uint32_t bytes = (uint32_t)(G * tile_tokens * 128 * CH);
                if (rank == 0) mbar_expect_tx_elect(bar(L::QFULL), 2 * bytes);
#pragma unroll
                for (int ch = 0; ch < CH; ++ch) tma2_load_3d_elect(base + L::OFF_Q + ch * (128 * 128), &tm_q, bar(L::QFULL) & kPeerBitMask, ch * 64, c.h * G, c.q_row);
            }
            ++c.g;
            if (++c.jj == c.n) { ++c.ui; next_unit(); }
            row = look_up(c, bad);
        }
        if (rank == 0 && !c.valid && ok) {
            if (c.g >= NST) ok = wait(L::KEMPTY + c.g % NST, (uint32_t)(c.g / NST - 1) & 1u, 1);
            if (ok && lane == 0) {
                tile_info[c.g & 15] = ((uint32_t)c.g + 1u) << 4 | kEnd;
                mbar_arrive(bar(L::KFULL + c.g % NST));
            }
        }
    } else if (warp == 2) {
        // ---------------- V by TMA: this CTA's columns (heads of 64: the upper columns are nobody's) ----------------
        Cursor c = begin();
        bool bad, ok = true;
        int row = look_up(c, bad);
        while (c.valid) {
            const int st = c.g % NST, key0 = (c.t0 + c.jj) * kChunkKeys, hi = c.hi;
            if (c.g >= NST) ok = wait(L::VEMPTY + st, (uint32_t)(c.g / NST - 1) & 1u, 3);
            if (!__all_sync(0xffffffffu, ok)) break;
            if (__any_sync(0xffffffffu, bad) && lane == 0) bad_unit[c.ui & 7] = (uint32_t)c.ui + 1u;
            __syncwarp();
            const int nb = D == HD || rank == 0 ? boxes(key0, hi) + boxes(key0 + 64, hi) : 0;       // (the second half has boxes only where the first is full)
            if (lane == 0) mbar_expect_tx(bar(L::VLAND + st), (uint32_t)(nb * box * 128 * VCH));      // (by the lane that may have marked the unit)
            __syncwarp();
            const uint32_t dst = base + L::OFF_V + st * L::V_STAGE;
            for (int i = 0; i < nb; ++i) {
                const int r = __shfl_sync(0xffffffffu, row, i);
#pragma unroll
                for (int ch = 0; ch < VCH; ++ch) tma_load_2d_elect(dst + ch * (128 * 128) + i * box * 128, &tm_v, bar(L::VLAND + st), ((int)rank * VCH + ch) * 64, r);
            }
            advance(c);
            row = look_up(c, bad);
        }
    } else if (warp == 1 || warp == 3) {
        // ---------------- S = Q K^T and O += P V (leader CTA; the warps stay converged, one lane issues) ----------------
        // Beside the busy warps of its scheduler a warp takes 450 to 700 cycles for the 8 MMAs of a product of head_dim 128, and 200 or 300 around them: there
        // warp 3 issues P V (1850 cycles a tile with one warp for both). At 256 the MMAs take longer than that, and the order of one warp's issue saves the wait for P V's
        // end ahead of the logits that take the place of its weights.
        // Everything that an MMA is issued with is kept uniform (votes and reductions say so to the compiler), or each of its operands is moved to the
        // uniform registers anew. What a tile is comes with its keys: walking the list of units here took 1200 cycles a tile.
        if (rank == 0 && (SPLIT || warp == 1)) {
            constexpr uint32_t idesc_qk = umma_idesc_bf16(256, kChunkKeys, false), idesc_pv = umma_idesc_bf16(256, HD, true);
            const uint64_t qdesc0 = umma_desc_sw128(base + L::OFF_Q, 16, 1024), kdesc0 = umma_desc_sw128(base + L::OFF_K, 16, 1024), vdesc0 = umma_desc_sw128(base + L::OFF_V, 128 * 128, 1024);
            const uint32_t tm = __reduce_or_sync(0xffffffffu, tmem_base);
            const uint32_t q_lo = (uint32_t)qdesc0, k_lo = (uint32_t)kdesc0, v_lo = (uint32_t)vdesc0, d_hi = (uint32_t)(qdesc0 >> 32), v_hi = (uint32_t)(vdesc0 >> 32);
            int q = 0, v = 0, uq = 0, uv = 0;                          // next tile of either product, and units begun
            int q_st = 0, q_buf = 0, v_st = 0, v_buf = 0;              // ... their stages and buffers
            uint32_t q_sph = 0u, v_bph = 0u;                           // parities of KFULL of tile q and PFULL of tile v
            auto issue_qk = [&](uint32_t info) {
                tc_fence_after();
#pragma unroll
                for (int ch = 0; ch < CH; ++ch)
                    umma2_ss4_elect(tm + kColS + q_buf * kChunkKeys, q_lo + ch * (128 * 128 / 16), d_hi, k_lo + (uint32_t)q_st * (L::K_STAGE / 16) + ch * (64 * 128 / 16), d_hi, idesc_qk, ch > 0 ? 1u : 0u);
                umma2_commit_mc_elect(bar(L::SFULL + q_buf), both);
                umma2_commit_mc_elect(bar(L::KEMPTY + q_st), both);
                if (info & kLast) umma2_commit_mc_elect(bar(L::QEMPTY), both);
                ++q;
                if (++q_st == NST) { q_st = 0; q_sph ^= 1u; }
                if (++q_buf == NS) q_buf = 0;
            };
            auto issue_pv = [&](uint32_t info) -> bool {
                if (!all(wait(L::PFULL + v_buf, v_bph, 6))) return false;
                if (info & kFirst) {
                    if (uv >= 1 && !all(wait(L::OFREE, (uint32_t)(uv - 1) & 1u, 7))) return false;
                    ++uv;
                }
                tc_fence_after();
                const uint32_t p_tmem = tm + kColS + v_buf * kChunkKeys, v_at = v_lo + (uint32_t)v_st * (L::V_STAGE / 16);
                umma2_ts4_elect(tm, p_tmem, v_at, v_hi, idesc_pv, (info & kFirst) ^ kFirst);
                if (info & kSecond) umma2_ts4_elect(tm, p_tmem + 64, v_at + 64 * 128 / 16, v_hi, idesc_pv, 1u);       // (else its weights are zero and its V was never loaded)
                umma2_commit_mc_elect(bar(L::PVDONE + (v & 3)), both);
                umma2_commit_mc_elect(bar(L::VEMPTY + v_st), both);
                ++v;
                if (++v_st == NST) v_st = 0;
                if (++v_buf == NS) { v_buf = 0; v_bph ^= 1u; }
                return true;
            };
            if (SPLIT && warp == 1) {
                for (;;) {
                    if (!all(wait(L::KFULL + q_st, q_sph, 4))) break;
                    const uint32_t info = __reduce_or_sync(0xffffffffu, tile_info[q & 15]);
                    if (info & kEnd) break;
                    if (info & kFirst) {
                        if (!all(wait(L::QFULL, (uint32_t)uq & 1u, 5))) break;
                        ++uq;
                    }
                    // the logits go where the weights of tile q - NS were
                    if (q >= NS && !all(wait(L::PVDONE + ((q - NS) & 3), (uint32_t)((q - NS) >> 2) & 1u, 14))) break;
                    issue_qk(info);
                }
            } else if (SPLIT) {
                for (;;) {
                    // (a tile's entry is there long before its weights, but for the last one, which says that there is none)
                    uint32_t info = __reduce_or_sync(0xffffffffu, tile_info[v & 15]);
                    if (info >> 4 != (uint32_t)v + 1u) {
                        const unsigned long long t_start = globaltimer_ns();
                        for (uint32_t n = 1; info >> 4 != (uint32_t)v + 1u; ++n) {
                            info = __reduce_or_sync(0xffffffffu, tile_info[v & 15]);
                            if ((n & 255u) == 0u && !all(*abort_flag == 0u && globaltimer_ns() - t_start < kChunkWaitNs)) break;
                        }
                        if (info >> 4 != (uint32_t)v + 1u) { *abort_flag = 1u; report_page_wait(p.g.status, kSitePageChunk + 15u); break; }
                    }
                    if ((info & kEnd) || !issue_pv(info)) break;
                }
            } else {
                bool ok = true, end = false;
                // The next tile's keys are there (true), or P V of tile v is due first. (Waiting for the keys alone could be for ever: their unit may find room in the list only
                // once the unit of tile v is done.)
                auto keys_or_due = [&]() -> bool {
                    const uint32_t keys = bar(L::KFULL + q_st), due = bar(L::PFULL + v_buf);
                    if (all(mbar_try_wait(keys, q_sph))) return true;
                    const unsigned long long t_start = globaltimer_ns();
                    for (uint32_t n = 1;; ++n) {
                        if (all(mbar_try_wait(keys, q_sph))) return true;
                        if (q > v && all(mbar_test_wait(due, v_bph))) return false;
                        if ((n & 255u) == 0u) {
                            if (!all(*abort_flag == 0u)) break;
                            if (!all(globaltimer_ns() - t_start < kChunkWaitNs)) { report_page_wait(p.g.status, kSitePageChunk + 4u); break; }
                        }
                    }
                    *abort_flag = 1u;
                    ok = false;
                    return false;
                };
                while (ok) {
                    // Q K^T runs one tile ahead, but for a tile whose weights are there already: the end of a unit waits for nothing else.
                    while (!end && q < v + NS && (q == v || !all(mbar_test_wait(bar(L::PFULL + v_buf), v_bph)))) {
                        if (!keys_or_due()) break;
                        const uint32_t info = __reduce_or_sync(0xffffffffu, tile_info[q & 15]);
                        end = (info & kEnd) != 0u;
                        if (end) break;
                        if (info & kFirst) {
                            // a unit whose Q has not come yet does not hold up the products of the last one
                            if (q > v) { if (!all(mbar_test_wait(bar(L::QFULL), (uint32_t)uq & 1u))) break; }
                            else { ok = all(wait(L::QFULL, (uint32_t)uq & 1u, 5)); if (!ok) break; }
                            ++uq;
                        }
                        issue_qk(info);
                    }
                    if (!ok || q == v) break;
                    ok = issue_pv(__reduce_or_sync(0xffffffffu, tile_info[v & 15]));
                }
            }
        }
    } else {
        // ---------------- softmax, rescaling, results ----------------
        const int sw = warp - 4, group = sw >> 3, half = (sw >> 2) & 1, quarter = warp & 3;
        const int row = quarter * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
        const uint32_t leader_pfull = mapa(bar(L::PFULL), 0), leader_ofree = mapa(bar(L::OFREE), 0);
        float *maxima = reinterpret_cast<float *>(smem + L::OFF_MAX);
        float *ref = reinterpret_cast<float *>(smem + L::OFF_REF);
        float2 *sums = reinterpret_cast<float2 *>(smem + L::OFF_SUM);
        const int gtid = (threadIdx.x - 128) & 255;
        auto group_sync = [&] { asm volatile("bar.sync %0, 256;" ::"r"(11 + group) : "memory"); };
        const float sc = part.scale_log2;
        int *out_row = reinterpret_cast<int *>(smem + L::OFF_ROWS);          // [128] where a row of a tile lies behind its first one
        if (group == 0 && half == 0) out_row[row] = (row / G * p.g.Hq + row % G) * D;
        const int row_token = row / G;
        bool ok = true;
        int gt = 0, ui = 0;
        // Row exchange: the 64 threads of a group's quarter meet at barrier 1 + quarter + 4 group. With two groups the other one's quarter has
        // arrived there, too, with its last tile (for the first tile of all: here).
        if (NG == 2 && group == 1) asm volatile("bar.arrive %0, 128;" ::"r"(1 + quarter) : "memory");
        for (int ul = 0; unit_ready(ul); ++ul) {
            const ChunkUnit &u = units[ul % L::NU];
            const int n = u.n, t0 = u.t0, lo = u.lo, hi = u.hi;
            if (n < 0) break;
            auto leave = [&] {                     // this warp is done with the list's entry
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(L::UEMPTY + ul % L::NU));
            };
            PageRange mine;                          // keys that this row sees
            int all_lo, all_hi;                      // keys that every row of the pair sees (either CTA's V meets the rows of both)
            {
                const PageSeq s = {u.b, u.row0, u.n_rows, u.len};
                const int t = min(u.token + (int)rank * tile_tokens + row_token, s.n - 1);
                mine = page_range(s, p, t, t);
                all_lo = page_range(s, p, min(s.n, u.token + 2 * tile_tokens) - 1, 0).lo;
                all_hi = page_range(s, p, 0, u.token).hi;
            }
            float m_ref = -INFINITY, l = 0.f;
            // (With two groups one instance of this code for whole and for masked tiles: three, with 64 keys unrolled in each, were 40 KB that the instruction caches had to
            // fetch again at every change, 3000 cycles of a unit. With one group, where the tile's chain is what the tensor pipe waits for, two: 16 frames in 113.5 us, not 119.)
            auto tile = [&](auto mode, const int jj) {          // 0: whole, 1: masked, 2: either
                constexpr int MODE = decltype(mode)::value;
                const int gi = gt + jj, buf = gi % NS, st = gi % NST;
                const uint32_t vph = (uint32_t)(gi / NST) & 1u;
                const int key0 = (t0 + jj) * kChunkKeys + half * 64;
                const uint32_t s_addr = tmem_base + lane_addr + kColS + buf * kChunkKeys + half * 64;
                const bool masked = MODE == 1 || (MODE == 2 && (key0 < all_lo || key0 + 64 > all_hi));
                const uint64_t mask = masked ? bits64(mine.lo - key0, mine.hi - key0) : ~0ull;       // keys that this row sees
                float mx = -INFINITY;
                // One group keeps its logits in registers (168 of them a thread); two groups (96) read them from tensor memory a second time.
                uint32_t r[NG == 1 ? 2 : 1][32];
                auto hide = [&](uint32_t (&v)[32], int c) {
                    const uint32_t bits = (uint32_t)(mask >> (32 * c));
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(bits & (1u << i))) v[i] = 0xff800000u;
                };
                ok = ok && wait(L::SFULL + buf, (uint32_t)(gi / NS) & 1u, 8);
                tc_fence_after();
                tmem_ld32(s_addr, r[0]);
                if constexpr (NG == 1) tmem_ld32(s_addr + 32, r[1]);
                auto maximum = [&](uint32_t (&v)[32], int c) {
                    if (masked) hide(v, c);
                    float x[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(v[i]);
                    float mx4[4] = {mx, x[0], x[1], x[2]};
#pragma unroll
                    for (int i = 3; i + 7 < 32; i += 8) {
                        mx4[0] = max3_nan_f32(mx4[0], x[i], x[i + 1]); mx4[1] = max3_nan_f32(mx4[1], x[i + 2], x[i + 3]);
                        mx4[2] = max3_nan_f32(mx4[2], x[i + 4], x[i + 5]); mx4[3] = max3_nan_f32(mx4[3], x[i + 6], x[i + 7]);
                    }
                    mx4[0] = max3_nan_f32(mx4[0], x[27], x[28]); mx4[1] = max3_nan_f32(mx4[1], x[29], x[30]); mx4[2] = max_nan_f32(mx4[2], x[31]);
                    mx = max_nan_f32(max_nan_f32(mx4[0], mx4[1]), max_nan_f32(mx4[2], mx4[3]));
                };
                if constexpr (NG == 1) {
                    tmem_wait_ld();
                    maximum(r[0], 0);
                    maximum(r[1], 1);
                } else {
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        tmem_wait_ld();
                        maximum(r[0], c);
                        tmem_ld32(s_addr + (c == 0 ? 32 : 0), r[0]);
                    }
                }
                if (!(mx < INFINITY)) l = __int_as_float(0x7fc00000);      // (a logit that is NaN or +inf)
                // (two places for a group's tiles in turn: what a thread has not read yet is not written before the group's next barrier)
                const int meet = ((gi & (2 * NG - 1)) * 128 + row) * 2;
                maxima[meet + half] = mx;
                asm volatile("bar.sync %0, %1;" ::"r"(1 + quarter + 4 * group), "n"(64 * NG) : "memory");
                const float2 of_row = *reinterpret_cast<const float2 *>(maxima + meet);
                const float top = fmaxf(of_row.x, of_row.y);
                // The row's reference so far, as the other group has left it with the tile before. (A place for each group: both threads of a row read, one
                // writes. The other group writes its place again behind its next barrier here, where both have arrived after they read it.)
                const float was = NG == 1 || jj == 0 ? m_ref : ref[(group ^ 1) * 128 + row];
                const bool grow = jj == 0 || (top - was) * sc > kChunkGrow;
                const float to = grow ? top : was;
                if (NG == 2) {
                    if (half == 0) ref[group * 128 + row] = to;
                    asm volatile("bar.arrive %0, 128;" ::"r"(1 + quarter + 4 * (group ^ 1)) : "memory");
                }
                if (m_ref != to) { l *= m_ref == -INFINITY ? (l == l ? 0.f : 1.f) : ex2((m_ref - to) * sc); m_ref = to; }
                if (jj > 0 && __any_sync(0xffffffffu, grow)) {
                    const float alpha = grow ? ex2((was - to) * sc) : 1.f;
                    if constexpr (NG == 2) tmem_wait_ld();                  // (the second reading of the logits, which is then in its registers)
                    ok = ok && wait(L::PVDONE + ((gi - 1) & 3), (uint32_t)((gi - 1) >> 2) & 1u, 10);
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D / 2; c += 16) {
                        uint32_t o[16];
                        const uint32_t o_addr = tmem_base + lane_addr + half * (D / 2) + c;
                        tmem_ld16(o_addr, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        tmem_st16(o_addr, o);
                    }
                    tmem_wait_st();
                }
                if (masked) {
                    ok = ok && wait(L::VLAND + st, vph, 9);
                    // Keys that no row sees count as zeros in V (a weight of 0 does not make a stale NaN one); a key that only some rows see must be
                    // finite, or the sequence is done again row by row. The 128 threads of a half share its 64 keys: half of this CTA's columns each.
                    const int key = key0 + (row & 63);
                    uint4 *v0 = reinterpret_cast<uint4 *>(smem + L::OFF_V + st * L::V_STAGE + (half * 64 + (row & 63)) * 128) + (row >> 6) * 4;
                    if (key < lo || key >= hi) {
#pragma unroll 1
                        for (int c = 0; c < 4 * VCH; ++c) v0[(c >> 2) * (128 * 128 / 16) + ((c + row) & 3)] = make_uint4(0, 0, 0, 0);
                    } else if ((key < all_lo || key >= all_hi) && (D == HD || rank == 0)) {
                        uint32_t odd = 0;
#pragma unroll 1
                        for (int c = 0; c < 4 * VCH; ++c) {
                            const uint4 v = v0[(c >> 2) * (128 * 128 / 16) + ((c + row) & 3)];
                            const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) odd |= ((q[e] & 0x7f80u) == 0x7f80u) | ((q[e] & 0x7f800000u) == 0x7f800000u);
                        }
                        if (odd) part.careful[u.b] = 1;
                    }
                    fence_proxy_async_smem();
                }
                const float mr = m_ref == -INFINITY ? 0.f : m_ref * sc + kWeightShift;
                const uint64_t sc2 = pack_f32x2(sc, sc), nm2 = pack_f32x2(-mr, -mr);
                uint64_t sum2[2] = {0ull, 0ull};
                auto weights = [&](uint32_t (&v)[32], int c) {
                    uint32_t packed[16];
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float x0, x1;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), sc2, nm2), x0, x1);
                        const float p0 = ex2(x0), p1 = ex2(x1);
                        sum2[(i >> 1) & 1] = add_f32x2(sum2[(i >> 1) & 1], pack_f32x2(p0, p1));
                        packed[i >> 1] = pack_bf16(p0, p1);
                    }
                    // (weights of keys 32 c .. of the half take the columns of its logits 16 c ..: read, and by this thread alone)
                    tmem_st16(s_addr + 16 * c, packed);
                };
                if constexpr (NG == 1) {
                    weights(r[0], 0);
                    weights(r[1], 1);
                } else {
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        tmem_wait_ld();
                        if (masked) hide(r[0], c);
                        weights(r[0], c);
                        if (c == 0) tmem_ld32(s_addr + 32, r[0]);
                    }
                }
                float a, b;
                unpack_f32x2(add_f32x2(sum2[0], sum2[1]), a, b);
                l += a + b;
                tmem_wait_st();
                if (!masked) ok = ok && wait(L::VLAND + st, vph, 11);       // (the arrival below says that this CTA's V is in place, too)
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(leader_pfull + 8u * (uint32_t)buf);
            };
#pragma unroll 1
            for (int jj = NG == 1 || (gt & 1) == group ? 0 : 1; jj < n; jj += NG) {          // (groups take the tiles of the whole share in turn)
                if constexpr (NG == 2) tile(std::integral_constant<int, 2>{}, jj);
                else {
                    const int key0 = (t0 + jj) * kChunkKeys + half * 64;
                    if (key0 < all_lo || key0 + 64 > all_hi) tile(std::integral_constant<int, 1>{}, jj);
                    else tile(std::integral_constant<int, 0>{}, jj);
                }
            }
            gt += n;
            // The group that has had the last tile finishes the unit; the other one leaves it its references and sums and goes on to the next unit, whose first tile
            // is its own. (It cannot come by with those of the unit after that before they are read: it meets this group at the barrier of the unit between. A unit without
            // tiles, whose rows see nothing, has no barrier: it leaves no sums.)
            const int g_last = gt - 1, parity = NG == 2 ? ui & 1 : 0;
            const bool finishes = NG == 1 || ((n > 0 ? g_last : gt) & 1) == group;
            if (n > 0 && !ok) l = __int_as_float(0x7fc00000);
            if (n > 0) sums[((parity * NG + group) * 2 + half) * 128 + row] = make_float2(m_ref, l);
            if (!finishes) {
                if (n > 0) {
                    asm volatile("bar.arrive %0, 512;" ::"r"(9 + parity) : "memory");
                    ++ui;
                }
                leave();
                continue;
            }
            if (n > 0) {
                ok = ok && wait(L::PVDONE + (g_last & 3), (uint32_t)(g_last >> 2) & 1u, 12);
                if (NG == 2) asm volatile("bar.sync %0, 512;" ::"r"(9 + parity) : "memory"); else group_sync();
                // the row's sum: references may differ, the latest one is the largest
                float2 part_of[2 * NG];
                m_ref = -INFINITY;
#pragma unroll
                for (int q = 0; q < 2 * NG; ++q) {
                    part_of[q] = sums[(parity * 2 * NG + q) * 128 + row];
                    m_ref = fmaxf(m_ref, part_of[q].x);
                }
                l = 0.f;
#pragma unroll
                for (int q = 0; q < 2 * NG; ++q) l += part_of[q].x == m_ref ? part_of[q].y : part_of[q].x == -INFINITY ? part_of[q].y * 0.f : part_of[q].y * ex2((part_of[q].x - m_ref) * sc);
            }
            const bool met_bad = n > 0 && bad_unit[ui & 7] == (uint32_t)ui + 1u;
            if (met_bad || !ok) l = __int_as_float(0x7fc00000);
            if (met_bad && gtid == 0) report_bad_page(p.g.status, u.b);
            tc_fence_after();
            const float inv = l == 0.f || n == 0 || (m_ref == -INFINITY && l == l) ? 0.f : 1.f / l;
            auto release = [&] {                     // all of this thread's columns of O are in registers: the next unit may overwrite it
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && n > 0) mbar_arrive_cluster(leader_ofree);
            };
            const int token0 = u.token + (int)rank * tile_tokens, live_rows = min(tile_tokens * G, (u.n_rows - token0) * G), slot = u.slot;
            const bool row_live = row < live_rows;
            if (slot >= 0) {
                if (half == 0 && row_live) part.ml[(size_t)slot * kChunkRows + rank * 128 + row] = make_float2(m_ref == -INFINITY ? -INFINITY : m_ref * part.scale_log2, l);
#pragma unroll 1
                for (int c = 0; c < D / 2; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(tmem_base + lane_addr + half * (D / 2) + c, o);
                    tmem_wait_ld();
                    if (c + 32 == D / 2) release();
                    if (row_live) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) st_global_v8(partial8(part, slot, D, (int)rank * 128 + row, half * (D / 2) + c + i), *reinterpret_cast<const uint32_t(*)[8]>(o + i));
                    }
                }
            } else {
                // O / l, 64 columns at a time through the group's staging area, then whole 128-byte pieces of rows to memory
                __nv_bfloat16 *tile_out = (__nv_bfloat16 *)p.out + ((size_t)(u.row0 + token0) * p.g.Hq + u.h * G) * D;
#pragma unroll 1
                for (int rnd = 0; rnd < D / 64; ++rnd) {
                    uint32_t o[32];
                    tmem_ld32(tmem_base + lane_addr + rnd * 64 + half * 32, o);
                    tmem_wait_ld();
                    if (rnd == D / 64 - 1) release();
                    uint8_t *area = smem + L::OFF_STAGE + group * (128 * 128), *srow = area + row * 128;
                    if (rnd > 0) group_sync();        // (read before it is written again)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float f[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] = inv == 0.f ? 0.f : __uint_as_float(o[8 * c + k]) * inv;      // (the accumulator of a unit without keys was never written)
                        *reinterpret_cast<uint4 *>(srow + (((half * 4 + c) ^ (row & 7)) << 4)) =
                            make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
                    }
                    group_sync();
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = k * 32 + (gtid >> 3);
                        if (r < live_rows)
                            *reinterpret_cast<uint4 *>(tile_out + out_row[r] + (gtid & 7) * 8 + rnd * 64) = *reinterpret_cast<const uint4 *>(area + r * 128 + (((gtid & 7) ^ (r & 7)) << 4));
                    }
                }
            }
            leave();
            group_sync();          // (the staging area, and the sums of one group, may be written again)
            if (n > 0) ++ui;
        }
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
            const uint32_t ks = exponent_bf16x2<FMT>(g.ke[row]), vs = exponent_bf16x2<FMT>(g.ve[row]);
            auto put = [&](const uint4 &q, uint32_t sc, __nv_bfloat16 *dst) {
                const uint32_t in[4] = {q.x, q.y, q.z, q.w};
                uint32_t o[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[2 * e] = bf16x2_mul(expand2<FMT, 0, 1>(biased<FMT>(in[e])), sc);
                    o[2 * e + 1] = bf16x2_mul(expand2<FMT, 2, 3>(biased<FMT>(in[e])), sc);
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
    cfg.blockDim = dim3(L::THREADS);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = k != a.g.k ? 2 : 1;         // (early start behind the widening alone: what it reads first is not written there)
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
