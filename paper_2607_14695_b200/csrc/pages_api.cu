// Host side of the paged prefix declared in reflex.h: argument checks, geometry, kernel selection. No call allocates device memory.
#include <algorithm>
#include <cstring>
#include <new>

#include "page_attention.cuh"

using namespace reflex;

struct reflex_pages {
    reflex_pages_desc desc;
    char *k, *v, *ke, *ve, *ws;
    int device, sm_count;
};

namespace {

int fail_cuda(cudaError_t e, const char *what) { return api_fail(REFLEX_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool desc_ok(const reflex_pages_desc *d)
{
    if (!d) return false;
    if (d->L < 1 || d->n_pages < 1 || d->Hq < 1 || d->Hkv < 1 || d->Hq % d->Hkv != 0 || d->Hq > 65535) return false;
    if (d->page != 16 && d->page != 32 && d->page != 64 && d->page != 128) return false;
    if (d->d != 32 && d->d != 64 && d->d != 128 && d->d != 256) return false;
    if (d->dtype != REFLEX_DTYPE_BF16 && d->dtype != REFLEX_DTYPE_F32) return false;
    if (d->format != REFLEX_PAGE_SAME && d->format != REFLEX_PAGE_E4M3 && d->format != REFLEX_PAGE_INT8) return false;
    if (d->max_seqs < 1 || d->max_seqs > kMaxSeqs || d->max_rows < 1) return false;
    // rows of a layer are counted in 32 bits by the tensor maps, bytes of a pool in 64
    const unsigned long long rows = (unsigned long long)d->n_pages * d->Hkv * d->page;
    return rows <= 0x7fffffffull && (unsigned long long)d->L * rows <= (1ull << 40);
}

size_t rows_of(const reflex_pages_desc &d) { return (size_t)d.n_pages * d.Hkv * d.page; }
size_t row_bytes(const reflex_pages_desc &d) { return (size_t)d.d * (d.format == REFLEX_PAGE_SAME ? elem_size(d.dtype) : 1); }

// Layout of the workspace: status word, marked sequences, partial results of split units, one layer of pages in bf16 (8-bit formats).
struct PagesLayout { size_t done, careful, arrived, meta, ml, o, wide, bytes; };
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
bool widened(const reflex_pages_desc &d) { return d.format != REFLEX_PAGE_SAME && page_chunk_takes(d.dtype, d.Hq / d.Hkv, d.d); }
PagesLayout pages_layout(const reflex_pages_desc &d)
{
    const size_t rows = page_chunk_takes(d.dtype, d.Hq / d.Hkv, d.d) ? std::max((size_t)2 * kTokenCtas * 16, (size_t)2 * kMostPairs * 256) : (size_t)2 * kTokenCtas * 16;
    PagesLayout w;
    w.done = 128;
    w.careful = 256;
    w.arrived = w.careful + kMaxSeqs;
    w.meta = w.arrived + 256 * sizeof(uint32_t);             // (all before it is zero at first, and after each call but for the status)
    w.ml = w.meta + up256(kMostPairs * sizeof(PageSplit));
    w.o = w.ml + up256(rows * sizeof(float2));
    w.wide = w.o + up256(rows * (size_t)d.d * sizeof(float));
    w.bytes = w.wide + (widened(d) ? 2 * up256(rows_of(d) * (size_t)d.d * 2) : 0);
    return w;
}

PageGeom geometry(const reflex_pages &p, int layer)
{
    const reflex_pages_desc &d = p.desc;
    PageGeom g;
    const size_t rows = rows_of(d) * (size_t)layer;
    g.k = p.k + rows * row_bytes(d);
    g.v = p.v + rows * row_bytes(d);
    g.ke = p.ke ? (uint8_t *)p.ke + rows : nullptr;
    g.ve = p.ve ? (uint8_t *)p.ve + rows : nullptr;
    g.status = (uint32_t *)p.ws;
    g.n_pages = d.n_pages; g.P = d.page; g.Hq = d.Hq; g.Hkv = d.Hkv; g.d = d.d;
    g.log_p = d.page == 16 ? 4 : d.page == 32 ? 5 : d.page == 64 ? 6 : 7;
    return g;
}

// (pools, workspace and the NULL stream are those of the handle's device)
int check_device(const reflex_pages_t *p)
{
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail_cuda(e, "device query");
    if (dev != p->device) return api_fail(REFLEX_ERR_STATE, "the pages belong to device %d, the current device is %d", p->device, dev);
    return REFLEX_OK;
}

// what every call on a handle has to have
int check_call(const reflex_pages_t *p, int layer, int n_layers, const reflex_page_batch *q, bool needs_cu)
{
    if (!p) return api_fail(REFLEX_ERR_INVALID_ARG, "pages is NULL");
    if (n_layers < 1 || layer < 0 || layer > p->desc.L - n_layers)
        return api_fail(REFLEX_ERR_INVALID_ARG, "layers [%d, %lld) outside [0, L=%d)", layer, (long long)layer + n_layers, p->desc.L);
    if (!q) return api_fail(REFLEX_ERR_INVALID_ARG, "batch is NULL");
    if (q->B < 1 || q->B > p->desc.max_seqs) return api_fail(REFLEX_ERR_SHAPE, "B=%d outside [1, max_seqs=%d]", q->B, p->desc.max_seqs);
    if (q->max_pages < 1 || (long long)q->max_pages * p->desc.page > 1ll << 30)
        return api_fail(REFLEX_ERR_SHAPE, "max_pages=%d: a table spans at most 2^30 positions, and one page at least", q->max_pages);
    if (!q->table || !q->len || (needs_cu && !q->cu)) return api_fail(REFLEX_ERR_INVALID_ARG, "table, cu or len of the batch is NULL");
    if (!aligned(q->table, 4) || !aligned(q->len, 4) || !aligned(q->cu, 4)) return api_fail(REFLEX_ERR_ALIGN, "table, cu or len of the batch not aligned to its elements");
    return check_device(p);
}

int check_rotation(const reflex_rotary *r, const int32_t *pos, int d)
{
    if (!r->freq || !r->axis || !pos) return api_fail(REFLEX_ERR_INVALID_ARG, "freq, axis or pos of the rotation is NULL");
    if (!aligned(r->freq, 4) || !aligned(pos, 4)) return api_fail(REFLEX_ERR_ALIGN, "freq or pos not aligned to its elements");
    if (r->R < 16 || r->R % 16 != 0 || r->R > d) return api_fail(REFLEX_ERR_SHAPE, "R=%d must be a multiple of 16 in [16, d=%d]", r->R, d);
    if (r->axes < 1 || r->axes > 8) return api_fail(REFLEX_ERR_SHAPE, "axes=%d outside [1, 8]", r->axes);
    if (r->adjacent != 0 && r->adjacent != 1) return api_fail(REFLEX_ERR_INVALID_ARG, "adjacent must be 0 or 1");
    return REFLEX_OK;
}

}  // namespace

extern "C" {

int reflex_rotary_axes(const void *x, int64_t ldx, void *y, int64_t ldy, const int32_t *pos, const reflex_rotary *rot, int n, int H, int d,
                       int inverse, int dtype, void *stream)
{
    if (dtype != REFLEX_DTYPE_BF16 && dtype != REFLEX_DTYPE_F32) return api_fail(REFLEX_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (inverse != 0 && inverse != 1) return api_fail(REFLEX_ERR_INVALID_ARG, "inverse must be 0 or 1");
    if (!rot) return api_fail(REFLEX_ERR_INVALID_ARG, "rot is NULL");
    if (n < 0 || H < 1 || H > 65535) return api_fail(REFLEX_ERR_SHAPE, "n=%d must be >= 0, H=%d in [1, 65535]", n, H);
    if (d < 16 || d % 16 != 0 || d > 1024) return api_fail(REFLEX_ERR_SHAPE, "d=%d must be a multiple of 16 in [16, 1024]", d);
    if (n == 0) return REFLEX_OK;
    if (!x || !y) return api_fail(REFLEX_ERR_INVALID_ARG, "x / y is NULL");
    const int rc = check_rotation(rot, pos, d);
    if (rc) return rc;
    if (ldx < (int64_t)H * d || ldy < (int64_t)H * d || ldx % 8 != 0 || ldy % 8 != 0)
        return api_fail(REFLEX_ERR_SHAPE, "ldx=%lld, ldy=%lld must be multiples of 8, at least H d = %lld", (long long)ldx, (long long)ldy, (long long)H * d);
    if (x == y && ldx != ldy) return api_fail(REFLEX_ERR_INVALID_ARG, "in place, ldx=%lld and ldy=%lld must be the same", (long long)ldx, (long long)ldy);
    if (!aligned(x, 16) || !aligned(y, 16)) return api_fail(REFLEX_ERR_ALIGN, "x / y not 16-byte aligned");
    const PageRotation r{*rot, pos, inverse};
    const cudaError_t e = launch_rotary_axes(x, ldx, y, ldy, r, n, H, d, dtype, (cudaStream_t)stream);
    return e == cudaSuccess ? REFLEX_OK : fail_cuda(e, "rotary launch");
}

size_t reflex_pages_pool_bytes(const reflex_pages_desc *d) { return desc_ok(d) ? (size_t)d->L * rows_of(*d) * row_bytes(*d) : 0; }
size_t reflex_pages_exp_bytes(const reflex_pages_desc *d) { return desc_ok(d) && d->format != REFLEX_PAGE_SAME ? (size_t)d->L * rows_of(*d) : 0; }
size_t reflex_pages_workspace_bytes(const reflex_pages_desc *d) { return desc_ok(d) ? pages_layout(*d).bytes : 0; }

int reflex_pages_create(const reflex_pages_desc *desc, void *k_pool, void *v_pool, void *k_exp, void *v_exp, void *workspace, void *stream,
                        reflex_pages_t **out)
{
    if (!out) return api_fail(REFLEX_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    if (!desc_ok(desc))
        return api_fail(REFLEX_ERR_SHAPE, "invalid pages descriptor (need page in {16,32,64,128}, Hq %% Hkv == 0, d in {32,64,128,256}, max_seqs in [1, %d], "
                        "sizes >= 1, a layer's rows below 2^31)", kMaxSeqs);
    if (!k_pool || !v_pool || !workspace) return api_fail(REFLEX_ERR_INVALID_ARG, "k_pool, v_pool and workspace must be non-NULL");
    const bool bytes = desc->format != REFLEX_PAGE_SAME;
    if (bytes && (!k_exp || !v_exp)) return api_fail(REFLEX_ERR_INVALID_ARG, "8-bit pages need k_exp and v_exp");
    if (!bytes && (k_exp || v_exp)) return api_fail(REFLEX_ERR_INVALID_ARG, "pages in dtype have no exponents: k_exp and v_exp must be NULL");
    if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(k_exp, 16) || !aligned(v_exp, 16) || !aligned(workspace, 256))
        return api_fail(REFLEX_ERR_ALIGN, "pools and exponents must be 16-byte aligned and the workspace 256-byte aligned");
    reflex_pages *p = new (std::nothrow) reflex_pages();
    if (!p) return api_fail(REFLEX_ERR_INVALID_ARG, "out of host memory");
    p->desc = *desc;
    p->k = (char *)k_pool; p->v = (char *)v_pool; p->ke = (char *)k_exp; p->ve = (char *)v_exp; p->ws = (char *)workspace;
    cudaError_t e = cudaGetDevice(&p->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, p->device);
    if (e == cudaSuccess) e = cudaMemsetAsync(workspace, 0, pages_layout(p->desc).meta, (cudaStream_t)stream);
    if (e != cudaSuccess) { delete p; return fail_cuda(e, "pages set-up"); }
    *out = p;
    return REFLEX_OK;
}

int reflex_pages_destroy(reflex_pages_t *p)
{
    if (!p) return api_fail(REFLEX_ERR_INVALID_ARG, "pages is NULL");
    delete p;
    return REFLEX_OK;
}

int reflex_pages_check_status(reflex_pages_t *p, void *stream)
{
    if (!p) return api_fail(REFLEX_ERR_INVALID_ARG, "pages is NULL");
    const int rc = check_device(p);
    if (rc) return rc;
    uint32_t word = 0;
    cudaError_t e = cudaMemcpyAsync(&word, p->ws, sizeof(word), cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return fail_cuda(e, "status read-back");
    if (word & 0x80000000u)
        return api_fail(REFLEX_ERR_TIMEOUT, "a device-side wait ran out (status 0x%08x: wait site %u, %s, block %u); results of that launch are invalid", word, (word >> 16) & 0x7FFFu,
                        wait_site_kernel((word >> 16) & 0x7FFFu), word & 0xFFFFu);
    if (word & kStatusBadPage)
        return api_fail(REFLEX_ERR_STATE, "sequence %u: a page outside the pool, or a position outside the page table", word & ~kStatusBadPage);
    return REFLEX_OK;
}

int reflex_pages_write(reflex_pages_t *p, int layer, const reflex_page_batch *batch, const void *k, int64_t ldk, const void *v, int64_t ldv,
                       int n_rows, const reflex_rotary *rot, const int32_t *pos, void *stream)
{
    int rc = check_call(p, layer, 1, batch, true);
    if (rc) return rc;
    const reflex_pages_desc &d = p->desc;
    if (n_rows < 0) return api_fail(REFLEX_ERR_SHAPE, "n_rows=%d is negative", n_rows);
    if (n_rows == 0) return REFLEX_OK;
    if (!k || !v) return api_fail(REFLEX_ERR_INVALID_ARG, "k / v is NULL");
    const int64_t width = (int64_t)d.Hkv * d.d;
    if (ldk < width || ldv < width || ldk % 8 != 0 || ldv % 8 != 0)
        return api_fail(REFLEX_ERR_SHAPE, "ldk=%lld, ldv=%lld must be multiples of 8, at least Hkv d = %lld", (long long)ldk, (long long)ldv, (long long)width);
    if (!aligned(k, 16) || !aligned(v, 16)) return api_fail(REFLEX_ERR_ALIGN, "k / v not 16-byte aligned");
    PageRotation r;
    memset(&r, 0, sizeof(r));
    if (rot) {
        rc = check_rotation(rot, pos, d.d);
        if (rc) return rc;
        r.rot = *rot;
        r.pos = pos;
    } else if (pos) return api_fail(REFLEX_ERR_INVALID_ARG, "positions without a rotation");
    const cudaError_t e = launch_page_write(geometry(*p, layer), *batch, k, ldk, v, ldv, n_rows, r, d.dtype, d.format, (cudaStream_t)stream);
    return e == cudaSuccess ? REFLEX_OK : fail_cuda(e, "page write launch");
}

int reflex_pages_read(reflex_pages_t *p, int layer, int n_layers, const reflex_page_batch *batch, const int32_t *start, void *k_out, void *v_out,
                      int S_out, void *stream)
{
    const int rc = check_call(p, layer, n_layers, batch, false);
    if (rc) return rc;
    if (S_out < 0 || n_layers > 65535) return api_fail(REFLEX_ERR_SHAPE, "S_out=%d must be >= 0, n_layers=%d at most 65535", S_out, n_layers);
    if (S_out == 0) return REFLEX_OK;
    if (!k_out || !v_out) return api_fail(REFLEX_ERR_INVALID_ARG, "k_out / v_out is NULL");
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(start, 4)) return api_fail(REFLEX_ERR_ALIGN, "k_out / v_out not 16-byte aligned, or start not to its elements");
    const cudaError_t e = launch_page_read(geometry(*p, layer), *batch, start, k_out, v_out, n_layers, S_out, p->desc.dtype, p->desc.format, (cudaStream_t)stream);
    return e == cudaSuccess ? REFLEX_OK : fail_cuda(e, "page read launch");
}

int reflex_pages_attention(reflex_pages_t *p, int layer, const reflex_page_batch *batch, const void *q, void *out, int n_rows, float scale,
                           int causal, int window, void *stream)
{
    const int rc = check_call(p, layer, 1, batch, true);
    if (rc) return rc;
    const reflex_pages_desc &d = p->desc;
    if (n_rows < 0 || n_rows > d.max_rows) return api_fail(REFLEX_ERR_SHAPE, "n_rows=%d outside [0, max_rows=%d]", n_rows, d.max_rows);
    if (causal != 0 && causal != 1) return api_fail(REFLEX_ERR_INVALID_ARG, "causal must be 0 or 1");
    if (window < 0) return api_fail(REFLEX_ERR_INVALID_ARG, "window=%d is negative", window);
    if (!(scale <= 2.0e38f)) return api_fail(REFLEX_ERR_INVALID_ARG, "scale must be a number of at most 2e38");       // (times log2 e it is finite)
    if (n_rows == 0) return REFLEX_OK;
    if (!q || !out) return api_fail(REFLEX_ERR_INVALID_ARG, "q / out is NULL");
    if (q == out) return api_fail(REFLEX_ERR_INVALID_ARG, "out must not be q");
    if (!aligned(q, 16) || !aligned(out, 16)) return api_fail(REFLEX_ERR_ALIGN, "q / out not 16-byte aligned");
    PageAttention a;
    a.g = geometry(*p, layer);
    a.q = *batch;
    a.qry = q; a.out = out;
    a.n_rows = n_rows; a.causal = causal; a.window = window;
    a.scale = scale > 0.f ? scale : 1.f / sqrtf((float)d.d);
    const int G = d.Hq / d.Hkv;
    a.g_shift = (G & (G - 1)) == 0 ? __builtin_ctz((unsigned)G) : -1;
    a.g_magic = G > 1 ? 0xffffffffu / (uint32_t)G + 1u : 0u;
    const long long per_seq = ((long long)n_rows * G + batch->B - 1) / batch->B;           // (token, head) rows of a sequence and KV head
    const int token_rows = page_token_rows(d.dtype, d.format, d.d, G, (int)std::min(per_seq, 1ll << 20));
    // (the tensor-core kernels count tiles of rows times blocks of 64 keys, and the rows of a KV head to the end of the last tile, in 32 bits)
    if ((token_rows || page_chunk_takes(d.dtype, G, d.d)) &&
        ((long long)n_rows * G > 0x7fffff00ll || ((double)n_rows * G / 8 + batch->B) * d.Hkv * ((double)batch->max_pages * d.page / 64 + 2) > 2.0e9))
        return api_fail(REFLEX_ERR_SHAPE, "n_rows=%d, B=%d and max_pages=%d: more tiles of rows and keys than 31 bits count", n_rows, batch->B, batch->max_pages);
    cudaStream_t st = (cudaStream_t)stream;
    const PagesLayout w = pages_layout(d);
    PagePartials part;
    part.o = (float *)(p->ws + w.o); part.ml = (float2 *)(p->ws + w.ml); part.meta = (PageSplit *)(p->ws + w.meta);
    part.careful = (uint8_t *)(p->ws + w.careful); part.careful_done = (uint32_t *)(p->ws + w.done); part.arrived = (uint32_t *)(p->ws + w.arrived);
    part.scale_log2 = a.scale * 1.4426950408889634f;
    cudaError_t e;
    if (token_rows) {
        part.rows = token_rows;
        e = launch_page_token(a, part, d.format, token_rows, p->sm_count, st);
    } else if (page_chunk_takes(d.dtype, G, d.d)) {
        part.rows = 256;
        const int pairs = std::min(p->sm_count / 2, kMostPairs);
        const void *k = a.g.k, *v = a.g.v;
        e = cudaSuccess;
        if (d.format != REFLEX_PAGE_SAME) {
            k = p->ws + w.wide;
            v = p->ws + w.wide + (w.bytes - w.wide) / 2;
            e = launch_page_widen(a, (void *)k, (void *)v, d.format, p->sm_count, st);
        }
        if (e == cudaSuccess) e = launch_page_chunk(a, part, k, v, pairs, st);
        if (e == cudaSuccess) e = launch_page_merge(a, part, pairs, d.format, p->sm_count, st);
    } else {
        e = launch_page_plain(a, d.dtype, d.format, p->sm_count, st);
    }
    return e == cudaSuccess ? REFLEX_OK : fail_cuda(e, "page attention launch");
}

}  // extern "C"
