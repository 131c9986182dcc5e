// Rows into pages (reflex_pages_write: keys rotated, both quantised on the way) and back (reflex_pages_read). Both are bound by memory.
// Measured in a warm graph: 16 prefixes of 4160 tokens into E4M3 pages (102 MB in and out) in 20.5 us (5.0 TB/s), back in 15.7; 1.7 GB of int8 pages back into bf16 in
// 270 us (6.4 TB/s); the row of one token of each of 64 streams, rotated, in 4.2 us, which is the launch and one chain of table, position, row, maximum and store.
#include "pages.cuh"
#include "sm100_ptx.cuh"

namespace reflex {

constexpr int kRowThreads = 256;

// largest magnitude of 8 elements as its bit pattern in fp32 (the order of magnitudes is that of their patterns; a NaN's are above all others)
template <typename T>
__device__ __forceinline__ uint32_t largest8(const Raw8<T> &r)
{
    if constexpr (sizeof(T) == 2) {
        const uint32_t m = __vmaxu2(__vmaxu2(r.w[0].x & 0x7fff7fffu, r.w[0].y & 0x7fff7fffu), __vmaxu2(r.w[0].z & 0x7fff7fffu, r.w[0].w & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    } else {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) m = max(max(m, max(r.w[i].x & 0x7fffffffu, r.w[i].y & 0x7fffffffu)), max(r.w[i].z & 0x7fffffffu, r.w[i].w & 0x7fffffffu));
        return m;
    }
}

// The 16 elements that this thread has of a row, into the row's place in the page; `top`: their largest magnitude. The TPR threads of a row agree on the row's.
template <int FMT, int TPR>
__device__ __forceinline__ void put_bytes(const PageGeom &g, void *pool, uint8_t *exps, size_t row, bool live, int e0, int e1, int lane_in_row, uint32_t top, float *a, float *b)
{
#pragma unroll
    for (int o = TPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (!live) return;
    const int e = row_exponent<FMT>(top);
    if (top > 0x7f000000u) {             // (larger than 2^127, or not finite: such a row holds zeros, and its elements are not looked at)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] = e == 255 ? 0.f : fminf(fmaxf(a[i], -0x1p127f), 0x1p127f);
            b[i] = e == 255 ? 0.f : fminf(fmaxf(b[i], -0x1p127f), 0x1p127f);
        }
    }
    const float inv = e == 255 ? 1.f : __int_as_float((254 - e) << 23);       // 2^-(e - 127)
    uint8_t *dst = (uint8_t *)pool + row * g.d;
    *reinterpret_cast<uint2 *>(dst + e0) = make_uint2(quantise4<FMT>(a, inv), quantise4<FMT>(a + 4, inv));
    *reinterpret_cast<uint2 *>(dst + e1) = make_uint2(quantise4<FMT>(b, inv), quantise4<FMT>(b + 4, inv));
    if (lane_in_row == 0) exps[row] = (uint8_t)e;
}

// A thread has 16 elements of a token's key rows and value rows, for several heads: eight pairs of the rotation (or, behind R, 16 neighbours).
template <typename T, int FMT, int TPR, bool TURNS>
__global__ void __launch_bounds__(kRowThreads, TURNS ? 2 : 4)
page_write_kernel(const PageGeom g, const reflex_page_batch q, const T *k, int64_t ldk, const T *v, int64_t ldv, int n_rows, const PageRotation r, int heads_per_thread)
{
    extern __shared__ int cu_s[];
    load_cu(q, cu_s);
    constexpr int per_block = kRowThreads / TPR;
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int R = TURNS ? r.rot.R : 0;
    const bool turns = lane * 16 < R, adj = TURNS && r.rot.adjacent != 0;
    const int e0 = turns && !adj ? lane * 8 : lane * 16, e1 = turns && !adj ? lane * 8 + R / 2 : lane * 16 + 8;
    TurnRate rate[TURNS ? 8 : 1];
    uint32_t axes = 0;              // four bits each
    uint32_t marks = 0;             // pairs that do not turn, and from bit 8 on those that have no angle (see rotary_axes_kernel)
    if (TURNS && turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int axis = r.rot.axis[lane * 8 + i];
            rate[TURNS ? i : 0] = turn_rate(r.rot.freq[lane * 8 + i]);
            if (axis >= r.rot.axes) rate[TURNS ? i : 0].lo = rate[TURNS ? i : 0].hi = 0u;
            else axes |= (uint32_t)axis << (4 * i);
            if ((rate[TURNS ? i : 0].lo | rate[TURNS ? i : 0].hi) == 0u) marks |= 1u << i;
            else if (!turnable(r.rot.freq[lane * 8 + i])) marks |= 256u << i;
        }
    }
    __syncthreads();
    const int h0 = blockIdx.y * heads_per_thread, h1 = min(g.Hkv, h0 + heads_per_thread);
    const int end = min(n_rows, cu_s[q.B]);
    // (whole warps stay in the loop: the threads of a row exchange their maxima)
    for (int64_t t0 = (int64_t)blockIdx.x * per_block; t0 < end; t0 += (int64_t)gridDim.x * per_block) {
        const int64_t t = t0 + sub;
        const bool exists = t < end && t >= cu_s[0];
        const T *kr = k + (exists ? t : 0) * ldk, *vr = v + (exists ? t : 0) * ldv;
        bool live = exists;
        size_t base = 0;
        float s[TURNS ? 8 : 1], c[TURNS ? 8 : 1];
        for (int h = h0; h < h1; ++h) {
            Raw8<T> ka = {}, kb = {}, va = {}, vb = {};
            if (exists) {
                ka = raw8(kr + (size_t)h * g.d + e0); kb = raw8(kr + (size_t)h * g.d + e1);
                va = raw8(vr + (size_t)h * g.d + e0); vb = raw8(vr + (size_t)h * g.d + e1);
            }
            if (h == h0 && exists) {            // (while the first rows are on their way)
                if (TURNS && turns) {
#pragma unroll
                    for (int i = 0; i < (TURNS ? 8 : 1); ++i) {
                        turn(rate[i], r.pos[(size_t)((axes >> (4 * i)) & 15u) * n_rows + t], s[i], c[i]);
                        if (marks & (256u << i)) s[i] = c[i] = __int_as_float(0x7fc00000);
                    }
                }
                const int b = find_seq(cu_s, q.B, (int)t);
                const int64_t at = (int64_t)q.len[b] - cu_s[b + 1] + t;
                const int page = at >= 0 && at <= 0x7fffffff ? page_at(q, g.n_pages, b, (int)(at >> g.log_p)) : -1;
                live = page >= 0;
                if (live) base = page_row(g, page, 0) + (size_t)(at & (g.P - 1));
                else if (lane == 0 && blockIdx.y == 0) report_bad_page(g.status, b);
            }
            const size_t row = base + ((size_t)h << g.log_p);
            const uint32_t still = marks & 255u;
            float u[8], w[8];
            if (TURNS || FMT != REFLEX_PAGE_SAME) { widen8(ka, u); widen8(kb, w); }
            if (TURNS && turns) {
                if (adj) {
#pragma unroll
                    for (int i = 0; i < (TURNS ? 8 : 1); ++i) {
                        float &p0 = i < 4 ? u[2 * i] : w[2 * i - 8], &p1 = i < 4 ? u[2 * i + 1] : w[2 * i - 7];
                        const float u0 = p0, w0 = p1;
                        p0 = u0 * c[i] - w0 * s[i];
                        p1 = u0 * s[i] + w0 * c[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < (TURNS ? 8 : 1); ++i) {
                        const float u0 = u[i], w0 = w[i];
                        u[i] = u0 * c[i] - w0 * s[i];
                        w[i] = u0 * s[i] + w0 * c[i];
                    }
                }
                // (asked for again, not kept: registers for it cost every row more)
                if (still && exists) { ka = raw8(kr + (size_t)h * g.d + e0); kb = raw8(kr + (size_t)h * g.d + e1); }
                if (FMT != REFLEX_PAGE_SAME && still) {
                    Raw8<float> u0, w0, u1 = narrow8<float>(u), w1 = narrow8<float>(w);
                    float f[8];
                    widen8(ka, f); u0 = narrow8<float>(f);
                    widen8(kb, f); w0 = narrow8<float>(f);
                    if (adj) keep_pairs<float, true>(still, u0, w0, u1, w1); else keep_pairs<float, false>(still, u0, w0, u1, w1);
                    widen8(u1, u); widen8(w1, w);
                }
            }
            if constexpr (FMT == REFLEX_PAGE_SAME) {
                if (live) {
                    T *kd = (T *)g.k + row * g.d, *vd = (T *)g.v + row * g.d;
                    Raw8<T> ya = ka, yb = kb;
                    if (TURNS && turns) {
                        ya = narrow8<T>(u);
                        yb = narrow8<T>(w);
                        if (still) { if (adj) keep_pairs<T, true>(still, ka, kb, ya, yb); else keep_pairs<T, false>(still, ka, kb, ya, yb); }
                    }
                    put8(kd + e0, ya); put8(kd + e1, yb);
                    put8(vd + e0, va); put8(vd + e1, vb);
                }
            } else {
                uint32_t top;
                if (TURNS) {
                    top = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = max(top, max(__float_as_uint(u[i]) & 0x7fffffffu, __float_as_uint(w[i]) & 0x7fffffffu));
                } else top = max(largest8<T>(ka), largest8<T>(kb));
                put_bytes<FMT, TPR>(g, g.k, g.ke, row, live, e0, e1, lane, top, u, w);
                widen8(va, u); widen8(vb, w);
                put_bytes<FMT, TPR>(g, g.v, g.ve, row, live, e0, e1, lane, max(largest8<T>(va), largest8<T>(vb)), u, w);
            }
        }
    }
}

// 16 elements of a row from its page: as they lie there (bytes in the first register), and out in dtype
template <typename T, int FMT> struct Piece { uint4 w[FMT == REFLEX_PAGE_SAME ? (int)sizeof(T) : 1]; int e; };
template <typename T, int FMT>
__device__ __forceinline__ Piece<T, FMT> take16(const void *pool, const uint8_t *exps, size_t row, int d, int e0)
{
    constexpr int W = FMT == REFLEX_PAGE_SAME ? (int)sizeof(T) : 1;          // 16-byte pieces
    Piece<T, FMT> p;
#pragma unroll
    for (int i = 0; i < W; ++i) p.w[i] = reinterpret_cast<const uint4 *>((const uint8_t *)pool + (row * d + e0) * W)[i];
    p.e = FMT == REFLEX_PAGE_SAME ? 0 : exps[row];
    return p;
}
// (sectors: dst is a multiple of 32 bytes; outputs are promised 16)
template <typename T, int FMT>
__device__ __forceinline__ void give16(const Piece<T, FMT> &p, bool ok, T *dst, bool sectors)
{
    if constexpr (FMT == REFLEX_PAGE_SAME) {
        const uint32_t nan = sizeof(T) == 2 ? 0x7fc07fc0u : 0x7fc00000u;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4 *>(dst)[i] = ok ? p.w[i] : make_uint4(nan, nan, nan, nan);
    } else {
        const uint32_t sc = exponent_bf16x2<FMT>(ok ? p.e : 255);
        const uint32_t in[4] = {p.w[0].x, p.w[0].y, p.w[0].z, p.w[0].w};
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = bf16x2_mul(expand2<FMT, 0, 1>(biased<FMT>(in[i])), sc);
            o[2 * i + 1] = bf16x2_mul(expand2<FMT, 2, 3>(biased<FMT>(in[i])), sc);
        }
        if constexpr (sizeof(T) == 2) {
            if (sectors) ptx::st_global_v8(dst, o);
            else {
                reinterpret_cast<uint4 *>(dst)[0] = make_uint4(o[0], o[1], o[2], o[3]);
                reinterpret_cast<uint4 *>(dst)[1] = make_uint4(o[4], o[5], o[6], o[7]);
            }
        } else {
            float f[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) { f[2 * i] = __uint_as_float(o[i] << 16); f[2 * i + 1] = __uint_as_float(o[i] & 0xffff0000u); }
            store8((float *)dst, f);
            store8((float *)dst + 8, f + 8);
        }
    }
}

// A block takes DEPTH pieces of 16 elements per thread of one (sequence, layer), K and V, in the order in which the pages hold them: [page][head][slot][piece];
// all are asked for before the first is written.
template <typename T, int FMT, int DEPTH>
__global__ void __launch_bounds__(kRowThreads)
page_read_kernel(const PageGeom g, const reflex_page_batch q, const int32_t *start, T *k_out, T *v_out, int n_layers, int S_out, int log_pieces)
{
    const int b = blockIdx.z, l = blockIdx.y;
    const int len = q.len[b], from = start ? max(0, start[b]) : 0;
    const int first_page = from >> g.log_p;
    const int64_t end = min((int64_t)len, (int64_t)from + S_out);               // positions [from, end)
    const size_t layer_rows = (size_t)g.n_pages * g.Hkv * g.P * l;
    const size_t out0 = ((size_t)b * n_layers + l) * S_out;
    const int per_head = g.log_p + log_pieces;                                  // (page, head) blocks of 2^per_head pieces
    const int64_t i0 = (int64_t)blockIdx.x * (DEPTH * kRowThreads) + threadIdx.x;
    const bool sectors = ((reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 31u) == 0;
    Piece<T, FMT> pk[DEPTH], pv[DEPTH];
    int64_t out[DEPTH];                  // -1: none
    bool ok[DEPTH];
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) {
        const int64_t v = i0 + j * kRowThreads;
        const int64_t block = v >> per_head;
        const int idx = first_page + (int)(g.Hkv == 1 ? block : (int64_t)((uint32_t)block / (uint32_t)g.Hkv)), h = g.Hkv == 1 ? 0 : (int)((uint32_t)block % (uint32_t)g.Hkv);
        const int piece = (int)v & ((1 << log_pieces) - 1), slot = (int)(v >> log_pieces) & (g.P - 1);
        const int64_t pos = ((int64_t)idx << g.log_p) + slot;
        out[j] = -1;
        if (pos < from || pos >= end) continue;
        const int page = page_at(q, g.n_pages, b, idx);
        ok[j] = page >= 0;
        if (page < 0 && piece == 0) report_bad_page(g.status, b);
        const size_t row = layer_rows + (page < 0 ? 0 : page_row(g, page, h) + slot);
        out[j] = (int64_t)(((out0 + (size_t)(pos - from)) * g.Hkv + h) * g.d + piece * 16);
        pk[j] = take16<T, FMT>(g.k, g.ke, row, g.d, piece * 16);
        pv[j] = take16<T, FMT>(g.v, g.ve, row, g.d, piece * 16);
    }
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) {
        if (out[j] < 0) continue;
        give16<T, FMT>(pk[j], ok[j], k_out + out[j], sectors);
        give16<T, FMT>(pv[j], ok[j], v_out + out[j], sectors);
    }
}

template <typename F>
static cudaError_t by_format(int dtype, int format, F &&go)
{
    auto fmt = [&](auto t) {
        if (format == REFLEX_PAGE_SAME) go(t, std::integral_constant<int, REFLEX_PAGE_SAME>{});
        else if (format == REFLEX_PAGE_E4M3) go(t, std::integral_constant<int, REFLEX_PAGE_E4M3>{});
        else go(t, std::integral_constant<int, REFLEX_PAGE_INT8>{});
    };
    if (dtype == REFLEX_DTYPE_F32) fmt(float{}); else fmt(__nv_bfloat16{});
    return cudaGetLastError();
}

cudaError_t launch_page_write(const PageGeom &g, const reflex_page_batch &q, const void *k, int64_t ldk, const void *v, int64_t ldv, int n_rows,
                              const PageRotation &r, int dtype, int format, cudaStream_t st)
{
    const int tpr = g.d / 16, per_block = kRowThreads / tpr;
    const long long blocks = ((long long)n_rows + per_block - 1) / per_block, share = blocks * g.Hkv / (148 * 8);
    const int hpt = share < 1 ? 1 : share > g.Hkv ? g.Hkv : (int)share;
    const int groups = (g.Hkv + hpt - 1) / hpt;
    const int most = (148 * 16 + groups - 1) / groups;
    const dim3 grid((unsigned)(blocks > most ? most : blocks), (unsigned)groups);
    const size_t smem = (size_t)(q.B + 1) * 4;
    count_launch();
    return by_format(dtype, format, [&](auto zero, auto f) {
        using T = decltype(zero);
        constexpr int FMT = decltype(f)::value;
        auto go = [&](auto w) {
            if (r.rot.R) page_write_kernel<T, FMT, decltype(w)::value, true><<<grid, kRowThreads, smem, st>>>(g, q, (const T *)k, ldk, (const T *)v, ldv, n_rows, r, hpt);
            else page_write_kernel<T, FMT, decltype(w)::value, false><<<grid, kRowThreads, smem, st>>>(g, q, (const T *)k, ldk, (const T *)v, ldv, n_rows, r, hpt);
        };
        if (tpr == 2) go(std::integral_constant<int, 2>{});
        else if (tpr == 4) go(std::integral_constant<int, 4>{});
        else if (tpr == 8) go(std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, 16>{});
    });
}

cudaError_t launch_page_read(const PageGeom &g, const reflex_page_batch &q, const int32_t *start, void *k_out, void *v_out, int n_layers, int S_out, int dtype,
                             int format, cudaStream_t st)
{
    // (a sequence that starts inside a page reaches into one page more)
    const int64_t pieces = (((int64_t)S_out + g.P - 1) / g.P + 1) * g.Hkv * g.P * (g.d / 16);
    const int log_pieces = g.d == 32 ? 1 : g.d == 64 ? 2 : g.d == 128 ? 3 : 4;
    count_launch();
    return by_format(dtype, format, [&](auto zero, auto f) {
        using T = decltype(zero);
        constexpr int FMT = decltype(f)::value;
        auto go = [&](auto depth) {
            constexpr int DEPTH = decltype(depth)::value;
            const dim3 grid((unsigned)((pieces + DEPTH * kRowThreads - 1) / (DEPTH * kRowThreads)), (unsigned)n_layers, (unsigned)q.B);
            page_read_kernel<T, FMT, DEPTH><<<grid, kRowThreads, 0, st>>>(g, q, start, (T *)k_out, (T *)v_out, n_layers, S_out, log_pieces);
        };
        // one piece a thread where that gives no more blocks than fit the device at once, else as many as keep 64 bytes or more of K and of V in flight
        if (pieces * n_layers * q.B <= 148ll * 8 * kRowThreads) go(std::integral_constant<int, 1>{});
        else go(std::integral_constant<int, FMT == REFLEX_PAGE_SAME ? 8 / (int)sizeof(T) / 2 : 4>{});
    });
}

}  // namespace reflex
