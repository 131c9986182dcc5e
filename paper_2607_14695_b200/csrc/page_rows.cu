// Rows into pages (reflex_pages_write: keys rotated, both quantised on the way) and back (reflex_pages_read). Both are bound by memory.
#include "pages.cuh"

namespace reflex {

constexpr int kRowThreads = 256;

// One row's 16 elements of this thread into its place in the page. The TPR threads of a row agree on its largest magnitude first.
// e0, e1: the first elements of the two chunks of 8 that the thread holds.
template <typename T, int FMT, int TPR>
__device__ __forceinline__ void put_row(const PageGeom &g, void *pool, uint8_t *exps, size_t row, bool live, int e0, int e1, int lane_in_row, const float *a, const float *b)
{
    if constexpr (FMT == REFLEX_PAGE_SAME) {
        if (!live) return;
        store8((T *)pool + row * g.d + e0, a);
        store8((T *)pool + row * g.d + e1, b);
    } else {
        // magnitudes as bit patterns: their order is that of the numbers, and a NaN's is above all of them
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, max(__float_as_uint(a[i]) & 0x7fffffffu, __float_as_uint(b[i]) & 0x7fffffffu));
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (!live) return;
        const int e = row_exponent<FMT>(top);
        const float inv = e == 255 ? 0.f : __int_as_float((254 - e) << 23);       // 2^-(e - 127); a row that is NaN holds zeros (its elements are not looked at)
        uint8_t *dst = (uint8_t *)pool + row * g.d;
        uint2 wa = make_uint2(0u, 0u), wb = wa;
        if (e != 255) {
            wa = make_uint2(quantise4<FMT>(a, inv), quantise4<FMT>(a + 4, inv));
            wb = make_uint2(quantise4<FMT>(b, inv), quantise4<FMT>(b + 4, inv));
        }
        *reinterpret_cast<uint2 *>(dst + e0) = wa;
        *reinterpret_cast<uint2 *>(dst + e1) = wb;
        if (lane_in_row == 0) exps[row] = (uint8_t)e;
    }
}

template <typename T, int FMT, int TPR>
__global__ void __launch_bounds__(kRowThreads)
page_write_kernel(const PageGeom g, const reflex_page_batch q, const T *k, int64_t ldk, const T *v, int64_t ldv, int n_rows, const PageRotation r, int heads_per_thread)
{
    extern __shared__ int cu_s[];
    load_cu(q, cu_s);
    constexpr int per_block = kRowThreads / TPR;
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int R = r.rot.R;
    const bool turns = lane * 16 < R, adj = r.rot.adjacent != 0;
    const int e0 = turns && !adj ? lane * 8 : lane * 16, e1 = turns && !adj ? lane * 8 + R / 2 : lane * 16 + 8;
    TurnRate rate[8];
    int axis[8];
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            axis[i] = r.rot.axis[lane * 8 + i];
            rate[i] = turn_rate(r.rot.freq[lane * 8 + i]);
            if (axis[i] >= r.rot.axes) { axis[i] = 0; rate[i].lo = rate[i].hi = 0u; }
        }
    }
    __syncthreads();
    const int h0 = blockIdx.y * heads_per_thread, h1 = min(g.Hkv, h0 + heads_per_thread);
    const int end = min(n_rows, cu_s[q.B]);
    // (whole warps stay in the loop: the threads of a row exchange their maxima)
    for (int64_t t0 = (int64_t)blockIdx.x * per_block; t0 < end; t0 += (int64_t)gridDim.x * per_block) {
        const int64_t t = t0 + sub;
        bool live = t < end && t >= cu_s[0];
        size_t base = 0;
        if (live) {
            const int b = find_seq(cu_s, q.B, (int)t);
            const int64_t at = (int64_t)q.len[b] - cu_s[b + 1] + t;
            const int page = at >= 0 && at <= 0x7fffffff ? page_at(q, g.n_pages, b, (int)(at >> g.log_p)) : -1;
            live = page >= 0;
            if (live) base = page_row(g, page, 0) + (size_t)(at & (g.P - 1));
            else if (lane == 0 && blockIdx.y == 0) report_bad_page(g.status, b);
        }
        float s[8], c[8];
        if (turns && live) {
#pragma unroll
            for (int i = 0; i < 8; ++i) turn(rate[i], r.pos[(size_t)axis[i] * n_rows + t], s[i], c[i]);
        }
        for (int h = h0; h < h1; ++h) {
            float a[8], b[8], va[8], vb[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = b[i] = va[i] = vb[i] = 0.f;
            if (live) {
                const T *kr = k + t * ldk + (size_t)h * g.d, *vr = v + t * ldv + (size_t)h * g.d;
                load8(kr + e0, a); load8(kr + e1, b);
                load8(vr + e0, va); load8(vr + e1, vb);
            }
            if (turns && live) {
                if (adj) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &u = i < 4 ? a[2 * i] : b[2 * i - 8], &w = i < 4 ? a[2 * i + 1] : b[2 * i - 7];
                        const float u0 = u, w0 = w;
                        u = u0 * c[i] - w0 * s[i];
                        w = u0 * s[i] + w0 * c[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u0 = a[i], w0 = b[i];
                        a[i] = u0 * c[i] - w0 * s[i];
                        b[i] = u0 * s[i] + w0 * c[i];
                    }
                }
            }
            const size_t row = base + ((size_t)h << g.log_p);
            put_row<T, FMT, TPR>(g, g.k, g.ke, row, live, e0, e1, lane, a, b);
            put_row<T, FMT, TPR>(g, g.v, g.ve, row, live, e0, e1, lane, va, vb);
        }
    }
}

// 16 elements of a row from its page: raw bits in, dtype out
template <typename T, int FMT>
__device__ __forceinline__ void get16(const void *pool, const uint8_t *exps, size_t row, int d, int e0, bool ok, T *dst)
{
    if constexpr (FMT == REFLEX_PAGE_SAME) {
        constexpr int W = (int)sizeof(T);          // 16-byte pieces in 16 elements: 2 or 4
        uint4 w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = ok ? reinterpret_cast<const uint4 *>((const T *)pool + row * d + e0)[i] : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t nan = sizeof(T) == 2 ? 0x7fc07fc0u : 0x7fc00000u;
#pragma unroll
        for (int i = 0; i < W; ++i) reinterpret_cast<uint4 *>(dst)[i] = ok ? w[i] : make_uint4(nan, nan, nan, nan);
    } else {
        const uint4 w = ok ? *reinterpret_cast<const uint4 *>((const uint8_t *)pool + row * d + e0) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t sc = exponent_bf16x2(ok ? exps[row] : 255);
        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = bf16x2_mul(bytes_to_bf16x2<FMT, 0, 1>(in[i], in[i]), sc);
            o[2 * i + 1] = bf16x2_mul(bytes_to_bf16x2<FMT, 2, 3>(in[i], in[i]), sc);
        }
        if constexpr (sizeof(T) == 2) {
            reinterpret_cast<uint4 *>(dst)[0] = make_uint4(o[0], o[1], o[2], o[3]);
            reinterpret_cast<uint4 *>(dst)[1] = make_uint4(o[4], o[5], o[6], o[7]);
        } else {
            float f[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) { f[2 * i] = __uint_as_float(o[i] << 16); f[2 * i + 1] = __uint_as_float(o[i] & 0xffff0000u); }
            store8((float *)dst, f);
            store8((float *)dst + 8, f + 8);
        }
    }
}

// A block takes `per_block` pieces of 16 elements of one (sequence, layer), in the order in which the pages hold them: [page][head][slot][piece].
template <typename T, int FMT>
__global__ void __launch_bounds__(kRowThreads)
page_read_kernel(const PageGeom g, const reflex_page_batch q, const int32_t *start, T *k_out, T *v_out, int n_layers, int S_out, int per_block)
{
    const int b = blockIdx.z, l = blockIdx.y;
    const int len = q.len[b], from = start ? max(0, start[b]) : 0;
    const int first_page = from >> g.log_p;
    const int pieces = g.d >> 4;
    const int page_pieces = g.Hkv * g.P * pieces;
    const int64_t end = min((int64_t)len, (int64_t)from + S_out);               // positions [from, end)
    const size_t layer_rows = (size_t)g.n_pages * g.Hkv * g.P * l;
    const size_t out0 = ((size_t)b * n_layers + l) * S_out;
    const int64_t i0 = (int64_t)blockIdx.x * per_block;
    if (((i0 / page_pieces + first_page) << g.log_p) >= end) return;
    for (int i = threadIdx.x; i < per_block; i += kRowThreads) {
        const int64_t v = i0 + i;
        const int idx = (int)(v / page_pieces) + first_page, in_page = (int)(v % page_pieces);
        const int piece = in_page % pieces, hs = in_page / pieces, slot = hs & (g.P - 1), h = hs >> g.log_p;
        const int64_t pos = ((int64_t)idx << g.log_p) + slot;
        if (pos < from || pos >= end) continue;
        const int page = page_at(q, g.n_pages, b, idx);
        if (page < 0 && piece == 0) report_bad_page(g.status, b);
        const size_t row = layer_rows + (page < 0 ? 0 : page_row(g, page, h) + slot);
        const size_t o = ((out0 + (size_t)(pos - from)) * g.Hkv + h) * g.d + piece * 16;
        get16<T, FMT>(g.k, g.ke, row, g.d, piece * 16, page >= 0, k_out + o);
        get16<T, FMT>(g.v, g.ve, row, g.d, piece * 16, page >= 0, v_out + o);
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
    const int blocks = (n_rows + per_block - 1) / per_block;
    int hpt = (int)((long long)blocks * g.Hkv / (148 * 8));
    hpt = hpt < 1 ? 1 : hpt > g.Hkv ? g.Hkv : hpt;
    const int groups = (g.Hkv + hpt - 1) / hpt;
    const int most = (148 * 16 + groups - 1) / groups;
    const dim3 grid((unsigned)(blocks > most ? most : blocks), (unsigned)groups);
    const size_t smem = (size_t)(q.B + 1) * 4;
    count_launch();
    return by_format(dtype, format, [&](auto zero, auto f) {
        using T = decltype(zero);
        constexpr int FMT = decltype(f)::value;
        auto go = [&](auto w) { page_write_kernel<T, FMT, decltype(w)::value><<<grid, kRowThreads, smem, st>>>(g, q, (const T *)k, ldk, (const T *)v, ldv, n_rows, r, hpt); };
        if (tpr == 2) go(std::integral_constant<int, 2>{});
        else if (tpr == 4) go(std::integral_constant<int, 4>{});
        else if (tpr == 8) go(std::integral_constant<int, 8>{});
        else go(std::integral_constant<int, 16>{});
    });
}

cudaError_t launch_page_read(const PageGeom &g, const reflex_page_batch &q, const int32_t *start, void *k_out, void *v_out, int n_layers, int S_out, int dtype,
                             int format, cudaStream_t st)
{
    const int per_block = 4 * kRowThreads;
    // (a sequence that starts inside a page reaches into one page more)
    const int64_t pieces = (((int64_t)S_out + g.P - 1) / g.P + 1) * g.Hkv * g.P * (g.d / 16);
    const dim3 grid((unsigned)((pieces + per_block - 1) / per_block), (unsigned)n_layers, (unsigned)q.B);
    count_launch();
    return by_format(dtype, format, [&](auto zero, auto f) {
        using T = decltype(zero);
        page_read_kernel<T, decltype(f)::value><<<grid, kRowThreads, 0, st>>>(g, q, start, (T *)k_out, (T *)v_out, n_layers, S_out, per_block);
    });
}

}  // namespace reflex
