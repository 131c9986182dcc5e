// Shared by the kernels of the paged prefix (reflex_pages_*, reflex_rotary_axes): geometry, page lookup, 8-bit rows, rotation angles.
#pragma once

#include <cuda_fp8.h>

#include "reflex_internal.cuh"

namespace reflex {

// Pools and geometry of a handle, of one layer where a kernel works on one (the pointers then are the layer's).
struct PageGeom {
    void *k, *v;              // [L][n_pages][Hkv][P][d] in the pages' format
    uint8_t *ke, *ve;         // [L][n_pages][Hkv][P], NULL for REFLEX_PAGE_SAME
    uint32_t *status;
    int n_pages, P, log_p, Hq, Hkv, d;
};

constexpr int kMaxSeqs = 1024;         // sequences of a call: cu fits the shared memory of the kernels that search it
constexpr uint32_t kStatusBadPage = 0x40000000u;

// What a page lookup of sequence b could not follow is reported once (the low bits name the sequence).
__device__ __forceinline__ void report_bad_page(uint32_t *status, int b) { atomicCAS(status, 0u, kStatusBadPage | (uint32_t)b); }

// page of positions [idx * P, (idx + 1) * P) of sequence b, -1 where the table does not give one of the pool's
__device__ __forceinline__ int page_at(const reflex_page_batch &q, int n_pages, int b, int idx)
{
    if ((unsigned)idx >= (unsigned)q.max_pages) return -1;
    const int id = q.table[(size_t)b * q.max_pages + idx];
    return (unsigned)id < (unsigned)n_pages ? id : -1;
}

// first row of a (page, head) block of a layer, in rows of d elements
__device__ __forceinline__ size_t page_row(const PageGeom &g, int page, int h) { return ((size_t)page * g.Hkv + h) << g.log_p; }

// cu into shared memory (all threads of the block), the search of a row in it: the last b with cu[b] <= row, so that empty sequences
// before it are passed over. Any contents give a b in [0, B).
__device__ __forceinline__ void load_cu(const reflex_page_batch &q, int *cu_s)
{
    for (int i = threadIdx.x; i <= q.B; i += blockDim.x) cu_s[i] = q.cu[i];
}
__device__ __forceinline__ int find_seq(const int *cu_s, int B, int row)
{
    int lo = 0, hi = B;      // cu[lo] <= row < cu[hi], as far as cu is in order
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu_s[mid] <= row) lo = mid; else hi = mid;
    }
    return lo;
}

// ---- 8-bit rows ----

template <int FMT> struct PageFormat;
template <> struct PageFormat<REFLEX_PAGE_INT8> { static constexpr int exponent = 6; static constexpr uint32_t mantissa = 0x7E0000u; };   // 127 = 1.984375 * 2^6
template <> struct PageFormat<REFLEX_PAGE_E4M3> { static constexpr int exponent = 8; static constexpr uint32_t mantissa = 0x600000u; };   // 448 = 1.75 * 2^8
constexpr int kPageMinExponent = -100;

// Exponent byte of a row whose largest magnitude has these bits (a pattern above infinity's is a NaN's): 255 unless finite.
template <int FMT>
__device__ __forceinline__ int row_exponent(uint32_t largest)
{
    if (largest >= 0x7f800000u) return 255;
    largest = min(largest, 0x7f000000u);        // 2^127
    const int e = (int)(largest >> 23) - 127 - PageFormat<FMT>::exponent + ((largest & 0x7fffffu) > PageFormat<FMT>::mantissa ? 1 : 0);
    return max(e, kPageMinExponent) + 127;
}

// Four numbers of a row (none above 2^127) as bytes, given 2^-e (exact: a power of two). To a whole number they are rounded by the addition of 1.5 * 2^23,
// which leaves it in the sum's low bits: one FMA, where a conversion runs at a quarter of the rate.
template <int FMT>
__device__ __forceinline__ uint32_t quantise4(const float *x, float inv)
{
    if constexpr (FMT == REFLEX_PAGE_E4M3) {
        const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(x[0] * inv, x[1] * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(x[2] * inv, x[3] * inv), __NV_SATFINITE, __NV_E4M3);
        return __byte_perm(a, b, 0x5410);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(fmaf(x[i], inv, 12582912.f));
        return __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
    }
}

__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

// Four bytes of an 8-bit row as they are before expand() (int8: plus 128, by the sign bits)
template <int FMT> __device__ __forceinline__ uint32_t biased(uint32_t w) { return FMT == REFLEX_PAGE_INT8 ? w ^ 0x80808080u : w; }
// Two bytes, in the low halves of x's halves, as two bf16: exact, times 2^-kExpandShift. Most of it on the FMA pipe: logic operations and byte permutations
// have half its rate, and unpacking is most of what the attention of few tokens issues.
//   int8: a byte u in the low bits of a bf16 is the (subnormal) number u 2^-133; times 2^127, less 128 2^-6, is the whole number times 2^-6.
//   e4m3: sign, four bits of exponent and three of mantissa moved to where bf16 has them (16 x moves them, and the sign bit's 128 times 240 adds what takes it
//   from bit 11 to bit 15) give the number times 2^-120, whether it is normal or not; the product with 2^120 is exact.
template <int FMT> constexpr int kExpandShift = FMT == REFLEX_PAGE_INT8 ? 6 : 0;
template <int FMT>
__device__ __forceinline__ uint32_t expand(uint32_t x)
{
    if constexpr (FMT == REFLEX_PAGE_INT8) return bf16x2_fma(x, 0x7f007f00u, 0xc000c000u);
    else return bf16x2_mul((x & 0x00800080u) * 240u + x * 16u, 0x7b807b80u);
}
// bytes I and J of a biased word, expanded
template <int FMT, int I, int J> __device__ __forceinline__ uint32_t expand2(uint32_t w) { return expand<FMT>(__byte_perm(w, 0u, I | 0x40 | (J << 8) | 0x4000)); }

// What expanded numbers of a row are multiplied with: 2^(e - 127 + kExpandShift) of its exponent byte, as a pair of bf16 and in fp32 (255: NaN; writes leave no
// byte below 27 or above 249)
template <int FMT>
__device__ __forceinline__ uint32_t exponent_bf16x2(int e)
{
    const uint32_t one = e == 255 ? 0x7fc0u : (uint32_t)min(e + kExpandShift<FMT>, 254) << 7;
    return one | (one << 16);
}
template <int FMT> __device__ __forceinline__ float exponent_f32(int e) { return e == 255 ? __int_as_float(0x7fc00000) : __int_as_float(min(e + kExpandShift<FMT>, 254) << 23); }

// ---- rotation angles ----
// A pair's frequency in revolutions per position, modulo 1, as a 64-bit fraction: position times fraction, modulo 2^64, is the fraction of a
// revolution that the position turns by, for any 32-bit position. Its upper 32 bits are kept, 1.5e-9 radians; as a number of half revolutions
// they are then rounded to fp32 (2^-25 at most: against 64 bits a rotation's fp32 error is 4.8e-8, where 64-bit angles leave 3.6e-8).
// (That is as far as 1 / (2 pi) in two doubles goes: from 2^40 on an angle would lose bits, and the fraction of NaN or an infinity is none. `turnable` says so;
// such a pair comes out NaN. What rate they have does not matter, but it is not 0.)
struct TurnRate { uint32_t lo, hi; };
__device__ __forceinline__ bool turnable(float freq) { return fabsf(freq) < 0x1p40f; }
__device__ __forceinline__ TurnRate turn_rate(float freq)
{
    // 1 / (2 pi) to twice the precision of a double
    const double c0 = 0x1.45f306dc9c883p-3, c1 = -0x1.6b01ec5417056p-57;
    if (!turnable(freq)) return {1u, 0u};
    const double f = (double)freq, r0 = f * c0, r1 = fma(f, c0, -r0) + f * c1;
    const double whole = floor(r0), frac = r0 - whole;                     // exact
    const unsigned long long u = __double2ull_rd(frac * 0x1p64) + (unsigned long long)__double2ll_rn(r1 * 0x1p64);
    TurnRate t;
    t.lo = (uint32_t)u;
    t.hi = (uint32_t)(u >> 32);
    return t;
}
__device__ __forceinline__ void turn(TurnRate t, int pos, float &sin_a, float &cos_a)
{
    const uint32_t p = (uint32_t)pos;
    const uint32_t frac = __umulhi(p, t.lo) + p * t.hi - (pos < 0 ? t.lo : 0u);
    sincospif((float)(int32_t)frac * 0x1p-31f, &sin_a, &cos_a);
}

// ---- 8 consecutive elements, as they lie in memory and as fp32 ----
template <typename T> struct Raw8 { uint4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> raw8(const T *p)
{
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const uint4 *>(p)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T> &r, float *f)
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint32_t w[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) { f[2 * j] = __uint_as_float(w[j] << 16); f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
            else f[4 * i + j] = __uint_as_float(w[j]);
        }
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T>
__device__ __forceinline__ Raw8<T> narrow8(const float *f)
{
    Raw8<T> r;
    if constexpr (sizeof(T) == 2) r.w[0] = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            r.w[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3]));
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void put8(T *p, const Raw8<T> &r)
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = r.w[i];
}
// The marked ones of eight pairs, elements i of both chunks (or 2i and 2i + 1 of the two in a row), as they were: to the bit
template <typename T, bool ADJ>
__device__ __forceinline__ void keep_pairs(uint32_t marked, const Raw8<T> &a0, const Raw8<T> &b0, Raw8<T> &a, Raw8<T> &b)
{
    constexpr int PER = 4 / (int)sizeof(T);              // elements of a word
    auto chunk = [&](const Raw8<T> &was, Raw8<T> &is, int second) {
#pragma unroll
        for (int i = 0; i < 8 / PER; ++i) {
            const uint4 &w = was.w[i >> 2];
            uint4 &y = is.w[i >> 2];
            const uint32_t old = (i & 3) == 0 ? w.x : (i & 3) == 1 ? w.y : (i & 3) == 2 ? w.z : w.w;
            uint32_t &now = (i & 3) == 0 ? y.x : (i & 3) == 1 ? y.y : (i & 3) == 2 ? y.z : y.w;
            uint32_t mask = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (marked & (1u << (ADJ ? 4 * second + (i * PER + e) / 2 : i * PER + e))) mask |= PER == 2 ? 0xffffu << (16 * e) : 0xffffffffu;
            now = (now & ~mask) | (old & mask);
        }
    };
    chunk(a0, a, 0);
    chunk(b0, b, 1);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *f)
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ void store8(float *p, const float *f)
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

// ---- launchers ----
struct PageRotation { reflex_rotary rot; const int32_t *pos; int inverse; };      // rot.R == 0: none

cudaError_t launch_rotary_axes(const void *x, int64_t ldx, void *y, int64_t ldy, const PageRotation &r, int n, int H, int d, int dtype, cudaStream_t st);
cudaError_t launch_page_write(const PageGeom &g, const reflex_page_batch &q, const void *k, int64_t ldk, const void *v, int64_t ldv, int n_rows,
                              const PageRotation &r, int dtype, int format, cudaStream_t st);
cudaError_t launch_page_read(const PageGeom &g, const reflex_page_batch &q, const int32_t *start, void *k_out, void *v_out, int n_layers, int S_out, int dtype,
                             int format, cudaStream_t st);

struct PageAttention {
    PageGeom g;
    reflex_page_batch q;
    const void *qry;
    void *out;
    int n_rows, causal, window;
    float scale;
    int g_shift;              // log2(Hq / Hkv), -1 where it is no power of two
    __device__ __forceinline__ int token_of(int row, int G) const { return g_shift >= 0 ? row >> g_shift : row / G; }      // of a (token, head) row
    uint32_t g_magic;         // x / (Hq / Hkv) = __umulhi(x, g_magic) for x < 2^16 (and more than one head in a group)
};
cudaError_t launch_page_plain(const PageAttention &a, int dtype, int format, int sm_count, cudaStream_t st);

}  // namespace reflex
