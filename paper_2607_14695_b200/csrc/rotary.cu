// Rotary positions with several axes (reflex_rotary_axes): every pair of a row turns by its own frequency times the token's position on
// the pair's axis.
//
// Bound by memory: 2 d elements a row. A thread owns 16 elements (8 pairs) of the rows of a token and turns them for several heads, so
// that a sine and a cosine serve all of them; it keeps its pairs' rates (the only work in double) over all tokens that it takes.
#include "pages.cuh"

namespace reflex {

constexpr int kRotThreads = 256;
constexpr int kRotHeads = 4;          // rows whose loads are in flight together

// slots [0, R / 16) are eight pairs each; the d - R elements behind them are copied, 16 a slot
template <typename T, bool ADJ>
__global__ void __launch_bounds__(kRotThreads)
rotary_axes_kernel(const T *x, int64_t ldx, T *y, int64_t ldy, const PageRotation r, int n, int H, int d, int heads_per_thread)
{
    const int slots = d >> 4, R = r.rot.R;
    const int per_block = kRotThreads / slots;
    const int slot = threadIdx.x % slots, sub = threadIdx.x / slots;
    if (sub >= per_block) return;
    const bool turns = slot * 16 < R;
    // first elements of the two chunks of 8 that the slot holds: pairs (c, c + R / 2), or neighbours
    const int e0 = turns && !ADJ ? slot * 8 : slot * 16, e1 = turns && !ADJ ? slot * 8 + R / 2 : slot * 16 + 8;
    TurnRate rate[8];
    int axis[8];
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            axis[i] = r.rot.axis[slot * 8 + i];
            rate[i] = turn_rate(r.rot.freq[slot * 8 + i]);
            if (axis[i] >= r.rot.axes) { axis[i] = 0; rate[i].lo = rate[i].hi = 0u; }
        }
    }
    const int h0 = blockIdx.y * heads_per_thread, h1 = min(H, h0 + heads_per_thread);
    for (int64_t t = (int64_t)blockIdx.x * per_block + sub; t < n; t += (int64_t)gridDim.x * per_block) {
        float s[8], c[8];
        if (turns) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                turn(rate[i], r.pos[(size_t)axis[i] * n + t], s[i], c[i]);
                if (r.inverse) s[i] = -s[i];
            }
        }
        const T *xr = x + t * ldx;
        T *yr = y + t * ldy;
        for (int h = h0; h < h1; h += kRotHeads) {
            float a[kRotHeads][8], b[kRotHeads][8];
#pragma unroll
            for (int k = 0; k < kRotHeads; ++k) {
                if (h + k < h1) { load8(xr + (size_t)(h + k) * d + e0, a[k]); load8(xr + (size_t)(h + k) * d + e1, b[k]); }
            }
#pragma unroll
            for (int k = 0; k < kRotHeads; ++k) {
                if (h + k >= h1) break;
                if (turns) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // (adjacent: pair i is elements 2i, 2i + 1 of the 16)
                        float &u = ADJ ? (i < 4 ? a[k][2 * i] : b[k][2 * i - 8]) : a[k][i];
                        float &v = ADJ ? (i < 4 ? a[k][2 * i + 1] : b[k][2 * i - 7]) : b[k][i];
                        const float u0 = u, v0 = v;
                        u = u0 * c[i] - v0 * s[i];
                        v = u0 * s[i] + v0 * c[i];
                    }
                }
                store8(yr + (size_t)(h + k) * d + e0, a[k]);
                store8(yr + (size_t)(h + k) * d + e1, b[k]);
            }
        }
    }
}

cudaError_t launch_rotary_axes(const void *x, int64_t ldx, void *y, int64_t ldy, const PageRotation &r, int n, int H, int d, int dtype, cudaStream_t st)
{
    const int per_block = kRotThreads / (d / 16);
    // heads of a token go to one thread once there are threads enough without them
    const long long rows = (long long)((n + per_block - 1) / per_block) * H;
    int hpt = (int)(rows / (148 * 8));
    hpt = hpt < 1 ? 1 : hpt > H ? H : hpt;
    const int groups = (H + hpt - 1) / hpt;
    int gx = (n + per_block - 1) / per_block;
    const int most = (148 * 16 + groups - 1) / groups;
    if (gx > most) gx = most;
    const dim3 grid((unsigned)gx, (unsigned)groups);
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
