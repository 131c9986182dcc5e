// Rotary positions with several axes (reflex_rotary_axes): every pair of a row turns by its own frequency times the token's position on
// the pair's axis.
//
// Bound by memory: 2 d elements a row. A thread owns 16 elements (8 pairs) of the rows of a token and turns them for several heads, so
// that a sine and a cosine serve all of them; it keeps its pairs' rates (the only work in double) over all tokens that it takes.
// Measured: 378 MB of bf16 queries and keys, strided, in 64 us (5.9 TB/s); 134 MB of fp32, 16 heads of 128, in 29 us (4.6 TB/s).
#include "pages.cuh"

namespace reflex {

constexpr int kRotThreads = 256;

// slots [0, R / 16) are eight pairs each; the d - R elements behind them are copied, 16 a slot
template <typename T, bool ADJ>
__global__ void __launch_bounds__(kRotThreads, 2)
rotary_axes_kernel(const T *x, int64_t ldx, T *y, int64_t ldy, const PageRotation r, int n, int H, int d, int heads_per_thread)
{
    constexpr int ROWS = 8 / (int)sizeof(T);          // rows whose loads are in flight together: 128 bytes a thread
    const int slots = d >> 4, R = r.rot.R;
    const int per_block = kRotThreads / slots;
    const int slot = threadIdx.x % slots, sub = threadIdx.x / slots;
    if (sub >= per_block) return;
    const bool turns = slot * 16 < R;
    // first elements of the two chunks of 8 that the slot holds: pairs (c, c + R / 2), or neighbours
    const int e0 = turns && !ADJ ? slot * 8 : slot * 16, e1 = turns && !ADJ ? slot * 8 + R / 2 : slot * 16 + 8;
    TurnRate rate[8];
    uint32_t axes = 0;              // four bits each
    // pairs that do not turn (0 times an infinity of the other element is not to be added to them), and from bit 8 on those that have no angle
    uint32_t marks = 0;
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int axis = r.rot.axis[slot * 8 + i];
            rate[i] = turn_rate(r.rot.freq[slot * 8 + i]);
            if (axis >= r.rot.axes) rate[i].lo = rate[i].hi = 0u;
            else axes |= (uint32_t)axis << (4 * i);
            if ((rate[i].lo | rate[i].hi) == 0u) marks |= 1u << i;
            else if (!turnable(r.rot.freq[slot * 8 + i])) marks |= 256u << i;
        }
    }
    const int h0 = blockIdx.y * heads_per_thread, h1 = min(H, h0 + heads_per_thread);
    for (int64_t t = (int64_t)blockIdx.x * per_block + sub; t < n; t += (int64_t)gridDim.x * per_block) {
        const T *xr = x + t * ldx;
        T *yr = y + t * ldy;
        float s[8], c[8];
        for (int h = h0; h < h1; h += ROWS) {
            Raw8<T> a[ROWS], b[ROWS];
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (h + k < h1) { a[k] = raw8(xr + (size_t)(h + k) * d + e0); b[k] = raw8(xr + (size_t)(h + k) * d + e1); }
            }
            if (h == h0 && turns) {          // (while the first rows are on their way)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    turn(rate[i], r.pos[(size_t)((axes >> (4 * i)) & 15u) * n + t], s[i], c[i]);
                    if (r.inverse) s[i] = -s[i];
                }
            }
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (h + k >= h1) break;
                Raw8<T> ya = a[k], yb = b[k];
                if (turns) {
                    float u[8], v[8];
                    widen8(a[k], u);
                    widen8(b[k], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // (adjacent: pair i is elements 2i, 2i + 1 of the 16)
                        float &p0 = ADJ ? (i < 4 ? u[2 * i] : v[2 * i - 8]) : u[i];
                        float &p1 = ADJ ? (i < 4 ? u[2 * i + 1] : v[2 * i - 7]) : v[i];
                        const float u0 = p0, v0 = p1;
                        p0 = u0 * c[i] - v0 * s[i];
                        p1 = u0 * s[i] + v0 * c[i];
                    }
                    ya = narrow8<T>(u);
                    yb = narrow8<T>(v);
                    if (marks) {
                        keep_pairs<T, ADJ>(marks, a[k], b[k], ya, yb);
                        const float nan[8] = {NAN, NAN, NAN, NAN, NAN, NAN, NAN, NAN};
                        keep_pairs<T, ADJ>(marks >> 8, narrow8<T>(nan), narrow8<T>(nan), ya, yb);
                    }
                }
                put8(yr + (size_t)(h + k) * d + e0, ya);
                put8(yr + (size_t)(h + k) * d + e1, yb);
            }
        }
    }
}

cudaError_t launch_rotary_axes(const void *x, int64_t ldx, void *y, int64_t ldy, const PageRotation &r, int n, int H, int d, int dtype, cudaStream_t st)
{
    const int per_block = kRotThreads / (d / 16);
    // heads of a token go to one thread once there are threads enough without them
    const long long blocks = ((long long)n + per_block - 1) / per_block, rows = blocks * H;
    const long long share = rows / (148 * 2);
    const int hpt = share < 1 ? 1 : share > H ? H : (int)share;
    const int groups = (H + hpt - 1) / hpt;
    const int most = (148 * 8 + groups - 1) / groups;
    const dim3 grid((unsigned)(blocks > most ? most : blocks), (unsigned)groups);
    count_launch();
    auto go = [&](auto zero, auto adj) {
        using T = decltype(zero);
        rotary_axes_kernel<T, decltype(adj)::value><<<grid, kRotThreads, 0, st>>>((const T *)x, ldx, (T *)y, ldy, r, n, H, d, hpt);
    };
    if (dtype == REFLEX_DTYPE_F32) { if (r.rot.adjacent) go(float{}, std::true_type{}); else go(float{}, std::false_type{}); }
    else { if (r.rot.adjacent) go(__nv_bfloat16{}, std::true_type{}); else go(__nv_bfloat16{}, std::false_type{}); }
    return cudaGetLastError();
}

}  // namespace reflex
