"""The paged prefix against its definitions in 64 bits: rotary positions with several axes, rows into 8-bit pages and back, attention of new
tokens over pages."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_14695_b200 import binding as rb  # noqa: E402
from paper_2607_14695_b200 import build as rbuild  # noqa: E402

if torch.cuda.is_available():
    rbuild.build()
import pages_util as U  # noqa: E402
from pages_util import DEV, HALF, Paged  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
FORMATS = [rb.PAGE_SAME, rb.PAGE_E4M3, rb.PAGE_INT8]


def _rot(R, axes, adjacent=False, base=10000.0):
    i = torch.arange(R // 2)
    return rb.Rotary((base ** (-2.0 * i / R)).float().to(DEV), (i % axes).to(torch.uint8).to(DEV), adjacent)


# ---- rotary ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,H,d,R,axes,adjacent,inverse,spare", [
    (1, 1, 32, 32, 1, False, False, 0), (1, 9, 256, 256, 3, False, False, 1), (7, 5, 128, 96, 3, True, True, 0), (301, 3, 64, 32, 2, False, True, 2),
    (33, 10, 128, 128, 4, True, False, 1), (1000, 24, 64, 64, 8, False, False, 0), (5, 2, 1024, 1008, 3, False, False, 0), (129, 4, 48, 16, 3, True, False, 3)])
def test_rotary(dtype, n, H, d, R, axes, adjacent, inverse, spare):
    g = torch.Generator().manual_seed(n + d)
    x = torch.randn(n, H + spare, d, generator=g).to(dtype)
    pos = torch.randint(-4096, 1 << 20, (axes, n), generator=g, dtype=torch.int32)
    pos[:, 0] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, 1, -1, 12345678, 7, 2])[:axes]
    rot = _rot(R, axes, adjacent)
    y = torch.full((n, H + spare, d), math.nan, dtype=dtype, device=DEV)
    out = rb.reflex_rotary_axes(x.to(DEV)[:, :H], y[:, :H], pos.to(DEV), rot, inverse=inverse)
    want = U.rotated(x[:, :H], pos, rot.freq.cpu(), rot.axis.cpu(), adjacent, inverse)
    # sine and cosine to 2^-22 (two units in the last place of fp32 and the fraction's 2^-32 revolutions) and far positions' angles as exact here
    # as 64 bits have them (2^31 * 2^-53), two products and a sum, one rounding at the end
    size = torch.maximum(x[:, :H].double().abs().amax(-1, keepdim=True), want.abs())
    assert ((out.cpu().double() - want).abs() <= HALF[dtype] * want.abs() + size * 2 * (2.0 ** -22 + 2 * 2.0 ** -24 + 2.0 ** -21)).all()
    assert torch.isnan(y[:, H:]).all()


def test_rotary_in_place_and_back():
    x = torch.randn(77, 6, 128, device=DEV)
    pos = torch.randint(0, 5000, (3, 77), dtype=torch.int32, device=DEV)
    rot = _rot(128, 3)
    apart = rb.reflex_rotary_axes(x, torch.empty_like(x), pos, rot)
    y = x.clone()
    assert rb.reflex_rotary_axes(y, y, pos, rot) is y and torch.equal(y, apart)
    rb.reflex_rotary_axes(y, y, pos, rot, inverse=True)
    assert (y - x).abs().max() <= 8 * 2.0 ** -22 * x.abs().max()


def test_rotary_gradient():
    """Inverse = the gradient, against differences in 64 bits of the definition."""
    g = torch.Generator().manual_seed(3)
    x, dy = torch.randn(4, 2, 32, generator=g), torch.randn(4, 2, 32, generator=g)
    pos = torch.randint(0, 900, (3, 4), generator=g, dtype=torch.int32)
    for adjacent in (False, True):
        rot = _rot(16, 3, adjacent)
        grad = rb.reflex_rotary_axes(dy.to(DEV), torch.empty(4, 2, 32, device=DEV), pos.to(DEV), rot, inverse=True).cpu().double()
        loss = lambda t: (U.rotated(t, pos, rot.freq.cpu(), rot.axis.cpu(), adjacent) * dy.double()).sum()      # noqa: E731
        for at in [(0, 0, 0), (1, 1, 9), (2, 0, 15), (3, 1, 31), (2, 1, 1)]:
            h = torch.zeros(4, 2, 32, dtype=torch.float64)
            h[at] = 0.5
            assert abs(float(loss(x.double() + h) - loss(x.double() - h)) - float(grad[at])) <= 8 * 2.0 ** -22 * dy.abs().max()


def test_rotary_nothing_and_unknown_axes():
    rot = _rot(32, 5)
    x = torch.randn(3, 2, 32, device=DEV)
    pos = torch.randint(1, 99, (2, 3), dtype=torch.int32, device=DEV)       # axes 2, 3, 4 have no positions: those pairs stay
    y = rb.reflex_rotary_axes(x, torch.empty_like(x), pos, rot)
    stay = (rot.axis >= 2).repeat(2).cpu()
    assert torch.equal(y.cpu()[..., stay], x.cpu()[..., stay]) and not torch.equal(y, x)
    rb.reflex_rotary_axes(x[:0], x[:0], pos[:, :0].contiguous(), rot)


# ---- rows into pages and back --------------------------------------------------------------------------------------------

def _read(c, layers=1, layer=0, S=None, start=None):
    S = max(1, max(c.lens)) if S is None else S
    out = [torch.full((len(c.lens), layers, S, c.Hkv, c.d), -7.0, dtype=c.dtype, device=DEV) for _ in range(2)]
    rb.reflex_pages_read(c.pages, layer, c.batch, out[0], out[1], start=None if start is None else torch.tensor(start, dtype=torch.int32, device=DEV))
    return [o.cpu() for o in out]


def _same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a.double()), torch.nan_to_num(b.double()))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,page,Hkv,d", [([1], 16, 1, 32), ([17, 0, 64, 5], 16, 2, 64), ([130, 1, 127], 64, 1, 256), ([33, 200], 128, 3, 128), ([70] * 5, 32, 4, 256)])
def test_write_and_read(fmt, dtype, lens, page, Hkv, d):
    c = Paged(lens, lens, page, Hkv, Hkv, d, dtype, fmt, L=2)
    c.poison()
    before = [t.clone() for t in (c.pages.k_pool, c.pages.v_pool)]
    c.write_all(layer=1)
    assert torch.equal(before[0].view(torch.uint8)[0], c.pages.k_pool.view(torch.uint8)[0])            # the other layer is untouched
    used = set(c.table[c.table >= 0].tolist())
    free = [p for p in range(c.n_pages) if p not in used]
    assert torch.equal(before[1].view(torch.uint8)[1, free], c.pages.v_pool.view(torch.uint8)[1, free])
    for got, want in zip(_read(c, layer=1), (c.k[1], c.v[1])):
        for b, n in enumerate(lens):
            assert _same(got[b, 0, :n], want[b].to(dtype))                          # exact: one rounding, into the page
            assert (got[b, 0, n:] == -7.0).all()
    rb.reflex_pages_check_status(c.pages)


@pytest.mark.parametrize("fmt", [rb.PAGE_E4M3, rb.PAGE_INT8])
def test_rows_of_every_size(fmt):
    """Zeros, the smallest and largest numbers, rows on the edge of an exponent, ties, infinities and NaN."""
    top = U.TOP[fmt]
    rows = [torch.zeros(32), torch.full((32,), 1e-44), torch.full((32,), 3.3e38), torch.linspace(-1, 1, 32) * 2.0 ** 127, torch.linspace(-top, top, 32),
            torch.linspace(-top, top, 32) * 1.0001, torch.linspace(-1, 1, 32) * 2.0 ** -95, torch.arange(32) + 0.5, (torch.arange(32) + 0.5) * 4.0, torch.randn(32) * 1e30,
            torch.full((32,), -0.0), torch.tensor([math.inf] + [1.0] * 31), torch.tensor([1.0] * 31 + [-math.inf]), torch.tensor([2.0] * 30 + [math.nan, 1.0])]
    x = torch.stack(rows)[:, None].float()
    c = Paged([len(rows)], [len(rows)], 16, 1, 1, 32, F32, fmt)
    c.write_all(k=x, v=x.flip(0).contiguous())
    k, v = _read(c)
    want, exps = U.held(x, fmt)
    assert _same(k[0, 0], want.float()) and _same(v[0, 0], want.flip(0).float())
    table = c.table[0].tolist()
    assert c.pages.k_exp[0, table[0], 0, :len(rows)].cpu().tolist() == exps[:, 0].tolist()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("adjacent", [False, True])
def test_write_rotates_keys(fmt, adjacent):
    """New tokens behind old ones, uneven, some sequences idle, rows of a packed projection, padding behind the last row."""
    lens, news, d, Hkv = [40, 16, 9, 70], [7, 0, 9, 33], 128, 2
    c = Paged(lens, news, 32, Hkv, Hkv, d, BF16, fmt, spare_rows=5)
    packed = c.normal(c.rows, 3 * Hkv, d)
    pos = torch.randint(0, 3000, (3, c.rows), generator=c.g, dtype=torch.int32)
    rot = _rot(96, 3, adjacent)
    dev = packed.to(DEV)
    c.poison()
    rb.reflex_pages_write(c.pages, 0, c.batch, dev[:, :Hkv], dev[:, Hkv:2 * Hkv], rotary=rot, pos=pos.to(DEV))
    start = [a - n for a, n in zip(lens, news)]
    k, v = _read(c, S=max(news), start=start)
    turned = U.rotated(packed[:, :Hkv], pos, rot.freq.cpu(), rot.axis.cpu(), adjacent)
    for b, n in enumerate(news):
        r = slice(int(c.cu[b]), int(c.cu[b]) + n)
        assert _same(v[b, 0, :n], U.held(packed[r, Hkv:2 * Hkv], fmt)[0].to(BF16))
        want = turned[r]
        size = packed[r, :Hkv].double().abs().amax(-1, keepdim=True) * 1.5
        # the rotation's own error, then one rounding: to bf16, to the row's integers (half a step: half of 2^e) or to e4m3 (2^-4, or half of 2^(e - 9))
        if n == 0:
            continue
        slack = 2.0 ** -20 * size
        if fmt == rb.PAGE_SAME:
            lim = HALF[BF16] * want.abs() + slack
        else:
            step = torch.exp2(U.held(want, fmt)[1].double() - 127)[..., None]
            lim = (0.5 * step if fmt == rb.PAGE_INT8 else torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * step)) + slack
        assert ((k[b, 0, :n].double() - want).abs() <= lim * 1.001).all()
        assert (k[b, 0, n:] == -7.0).all()
    rb.reflex_pages_check_status(c.pages)


def test_read_layers_and_windows():
    c = Paged([50, 3, 0, 64], [0] * 4, 16, 2, 2, 64, BF16, rb.PAGE_INT8, L=4)
    for layer in range(4):
        c.write_all(layer=layer)
    k, v = _read(c, layers=3, layer=1, S=20, start=[37, -5, 0, 60])
    for i, l in enumerate((1, 2, 3)):
        for b, (lo, hi) in enumerate([(37, 50), (0, 3), (0, 0), (60, 64)]):
            assert _same(k[b, i, :hi - lo], c.k[l][b][lo:hi].to(BF16)) and _same(v[b, i, :hi - lo], c.v[l][b][lo:hi].to(BF16))
            assert (k[b, i, hi - lo:] == -7.0).all()
    short = _read(c, layers=1, layer=3, S=10)                                      # tokens past S_out rows are left out
    assert _same(short[0][3, 0], c.k[3][3][:10].to(BF16))


# ---- attention ---------------------------------------------------------------------------------------------------------

CASES = [
    # lens, news, page, Hq, Hkv, d, causal, window
    ([1], [1], 16, 1, 1, 64, True, 0),
    ([37], [1], 16, 8, 1, 256, False, 0),
    ([817, 64, 129], [1, 1, 1], 64, 8, 1, 256, True, 0),
    ([300, 5, 0, 128, 77], [1, 1, 0, 0, 3], 32, 8, 2, 128, True, 0),
    ([257, 200], [2, 9], 128, 14, 2, 128, True, 0),
    ([100, 90], [5, 90], 16, 4, 4, 64, True, 0),
    ([130, 260], [130, 100], 64, 4, 2, 128, True, 0),
    ([400], [90], 64, 8, 1, 256, False, 0),
    ([513, 30, 200], [140, 30, 1], 32, 8, 1, 256, True, 0),
    ([300, 260], [70, 64], 128, 7, 1, 128, True, 100),
    ([300, 260], [70, 64], 16, 8, 2, 64, False, 77),
    ([600], [1], 64, 8, 1, 128, True, 33),
    ([64, 64], [64, 64], 32, 16, 2, 256, True, 1),
    ([3, 2], [5, 4], 16, 8, 1, 256, True, 0),             # more new tokens than tokens: the first ones see nothing
    ([150], [40], 16, 2, 1, 32, True, 0),
    ([140], [3], 16, 24, 1, 64, False, 0),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-p{c[2]}-{c[3]}x{c[4]}x{c[5]}-{'c' if c[6] else 'f'}{c[7]}".replace(" ", ""))
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention(case, fmt, dtype):
    lens, news, page, Hq, Hkv, d, causal, window = case
    if dtype == F32 and sum(news) * Hq * max(lens) > 400000:
        pytest.skip("the plain kernel has smaller cases")
    c = Paged(lens, news, page, Hq, Hkv, d, dtype, fmt, spare_rows=3, seed=len(lens) + d)
    c.poison()
    c.write_all()
    q = c.normal(c.rows, Hq, d)
    out = torch.full((c.rows, Hq, d), -7.0, dtype=dtype, device=DEV)
    for _ in range(2):           # (a second call finds what the first has left in the workspace)
        rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), out, causal=causal, window=window)
        rb.reflex_pages_check_status(c.pages)
        c.check(out, c.attend(q, causal=causal, window=window), str(case))
        assert (out[int(c.cu[-1]):] == -7.0).all()           # rows behind the last sequence


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("news", [[1, 1], [40, 70]])
def test_attention_logits_of_any_size(fmt, news):
    """Wide logits (one key takes all), a scale of its own, and none at all (the mean of the values)."""
    c = Paged([180, 97], news, 64, 8, 1, 128, BF16, fmt, seed=5)
    c.write_all()
    q = c.normal(c.rows, 8, 128, std=12.0)
    out = torch.empty((c.rows, 8, 128), dtype=BF16, device=DEV)
    for x, scale in ((q, 0.0), (q, 1.0), (q, 1e-3), (torch.zeros_like(q), 0.0)):
        rb.reflex_pages_attention(c.pages, 0, c.batch, x.to(DEV), out, scale=scale, causal=True)
        c.check(out, c.attend(x, causal=True, scale=scale or None), f"scale {scale}")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("news", [[1, 1], [33, 60]])
def test_attention_of_masked_and_unmasked_nan(fmt, news):
    """A row that is not finite reaches the tokens that see it, and those only."""
    lens, Hq, d = [200, 150], 8, 128
    c = Paged(lens, news, 32, Hq, 1, d, BF16, fmt, seed=11)
    k, v = c.normal(sum(lens), 1, d), c.normal(sum(lens), 1, d)
    k[190, 0, 3] = math.nan                  # sequence 0, position 190
    v[200 + 20, 0, 7] = math.inf             # sequence 1, position 20
    c.write_all(k=k, v=v)
    q = c.normal(c.rows, Hq, d)
    out = torch.empty((c.rows, Hq, d), dtype=BF16, device=DEV)
    rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), out, causal=True, window=100)
    got = out.cpu()
    sees = [[p - 100 < at <= p for p in range(n - m, n)] for n, m, at in zip(lens, news, (190, 20))]
    for b in range(2):
        for i, s in enumerate(sees[b]):
            row = got[int(c.cu[b]) + i]
            if b == 0:
                assert torch.isfinite(row).all() == (not s), (b, i)
            else:
                assert torch.isfinite(row).all() == (not s), (b, i)


@pytest.mark.parametrize("fmt", [rb.PAGE_SAME, rb.PAGE_INT8])
@pytest.mark.parametrize("news", [[1, 1, 1], [30, 1, 80]])
def test_pages_outside_the_pool(fmt, news):
    """A bad table entry, or a length past the table: nothing is followed, the sequence reads NaN and is named; the others are right."""
    lens = [100, 90, 200]
    c = Paged(lens, news, 32, 8, 1, 128, BF16, fmt, seed=2)
    c.write_all()
    rb.reflex_pages_check_status(c.pages)
    bad = c.table.clone()
    bad[1, 1] = c.n_pages
    batch = rb.PageBatch(bad.to(DEV), c.batch.cu, c.batch.length)
    q = c.normal(c.rows, 8, 128)
    out = torch.zeros((c.rows, 8, 128), dtype=BF16, device=DEV)
    rb.reflex_pages_attention(c.pages, 0, batch, q.to(DEV), out)
    r = slice(int(c.cu[1]), int(c.cu[2]))
    assert torch.isnan(out[r]).all()
    want = c.attend(q)
    out[r] = want[0][r].to(DEV).to(BF16)
    c.check(out, want)
    with pytest.raises(rb.ReflexError) as e:
        rb.reflex_pages_check_status(c.pages)
    assert e.value.code == rb.ERR_STATE and "sequence 1" in str(e.value)


def test_lengths_past_the_table():
    c = Paged([64, 40], [2, 2], 32, 4, 4, 64, BF16, rb.PAGE_E4M3, seed=2)
    c.write_all()
    batch = rb.PageBatch(c.batch.table, c.batch.cu, torch.tensor([64, 70], dtype=torch.int32, device=DEV))
    before = c.pages.k_pool.view(torch.uint8).clone()
    rows = c.normal(4, 4, 64).to(DEV)
    rb.reflex_pages_write(c.pages, 0, batch, rows, rows)
    changed = (before != c.pages.k_pool.view(torch.uint8)).any(-1).nonzero()
    assert set(changed[:, 1].tolist()) == {int(c.table[0, 1])}       # sequence 0's new tokens alone
    out = torch.zeros((4, 4, 64), dtype=BF16, device=DEV)
    rb.reflex_pages_attention(c.pages, 0, batch, rows, out)
    assert torch.isnan(out[2:]).all() and torch.isfinite(out[:2]).all()
    with pytest.raises(rb.ReflexError):
        rb.reflex_pages_check_status(c.pages)


def test_the_path_together():
    """Four ticks of an incremental prefill, each frame rotated, written and attended to; the prefix goes to the action expert's static region and the
    newest frame to its ring, and the expert's attention over them is what the pages stand for."""
    L, B, Hq, Hkv, d, page, frame = 2, 2, 8, 1, 256, 32, 24
    N, T, ticks = 48, 8, 4
    seq = [[frame * (t + 1) - 3 * b * (t + 1) for t in range(ticks)] for b in range(B)]        # lengths after every tick
    most = -(-frame * ticks // page)
    pages = rb.Pages(L, B * most + 1, page, Hq, Hkv, d, rb.DTYPE_BF16, rb.PAGE_INT8, max_seqs=B, max_rows=B * frame)
    table = torch.randperm(B * most + 1)[:B * most].to(torch.int32).view(B, most).to(DEV)
    rot = _rot(d, 3)
    g = torch.Generator().manual_seed(8)
    keys = [[torch.zeros(0, Hkv, d, dtype=torch.float64) for _ in range(B)] for _ in range(L)]
    for t in range(ticks):
        new = [seq[b][t] - (seq[b][t - 1] if t else 0) for b in range(B)]
        cu = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
        batch = rb.PageBatch(table, cu, torch.tensor([s[t] for s in seq], dtype=torch.int32, device=DEV))
        n = sum(new)
        pos = torch.randint(0, 500, (3, n), generator=g, dtype=torch.int32)
        for l in range(L):
            qkv = torch.randn(n, Hq + 2 * Hkv, d, generator=g).to(BF16).to(DEV)
            rb.reflex_pages_write(pages, l, batch, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], rotary=rot, pos=pos.to(DEV))
            q = rb.reflex_rotary_axes(qkv[:, :Hq], torch.empty((n, Hq, d), dtype=BF16, device=DEV), pos.to(DEV), rot)
            out = rb.reflex_pages_attention(pages, l, batch, q, torch.empty_like(q), causal=False)
            kv = [torch.zeros((B, 1, frame * ticks, Hkv, d), dtype=BF16, device=DEV) for _ in range(2)]
            rb.reflex_pages_read(pages, l, batch, kv[0], kv[1])
            for b in range(B):
                k, v = [x[b, 0, :seq[b][t], 0].double().cpu() for x in kv]
                r = slice(int(cu[b]), int(cu[b + 1]))
                w = torch.softmax(torch.einsum("nhd,kd->nhk", q[r].double().cpu(), k) / 16, -1)
                want, mass = torch.einsum("nhk,kd->nhd", w, v), torch.einsum("nhk,kd->nhd", w, v.abs())
                assert ((out[r].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 1e-3) * 1.01 * mass).all()
    rb.reflex_pages_check_status(pages)
    S = [s[-2] for s in seq]
    cache = rb.Cache(L, B, Hq, Hkv, d, frame * ticks, N, T, rb.DTYPE_BF16)
    older = rb.PageBatch(table, None, torch.tensor(S, dtype=torch.int32, device=DEV))
    ks, vs = [torch.zeros((B, L, max(S), Hkv, d), dtype=BF16, device=DEV) for _ in range(2)]
    rb.reflex_pages_read(pages, 0, older, ks, vs)
    rb.reflex_cache_init_static(cache, [0, 1], ks, vs, S=S)
    m = min(new)
    newest = rb.PageBatch(table, None, torch.tensor([s[-1] for s in seq], dtype=torch.int32, device=DEV))
    kn, vn = [torch.zeros((B, L, m, Hkv, d), dtype=BF16, device=DEV) for _ in range(2)]
    rb.reflex_pages_read(pages, 0, newest, kn, vn, start=torch.tensor([s[-1] - m for s in seq], dtype=torch.int32, device=DEV))
    rb.reflex_cache_append_sliding(cache, [0, 1], kn, vn)
    x = [torch.randn(B, T, h, d, generator=g).to(BF16).to(DEV) for h in (Hq, Hkv, Hkv)]
    for l in range(L):
        out = rb.reflex_partitioned_attention(cache, l, *x, torch.empty((B, T, Hq, d), dtype=BF16, device=DEV))
        for b in range(B):
            k = torch.cat([ks[b, l, :S[b], 0], kn[b, l, :, 0], x[1][b, :, 0]]).double()
            v = torch.cat([vs[b, l, :S[b], 0], vn[b, l, :, 0], x[2][b, :, 0]]).double()
            w = torch.softmax(torch.einsum("nhd,kd->nhk", x[0][b].double(), k) / 16, -1)
            assert (out[b].double() - torch.einsum("nhk,kd->nhd", w, v)).abs().max() <= 2e-2


# ---- as a program uses them ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("news", [[1, 1], [50, 31]])
def test_captured_and_replayed(news):
    """A graph of rotation, write, attention and read follows lengths, tables and inputs that change between replays, on a stream of its own."""
    page, Hq, Hkv, d = 32, 8, 1, 128
    lens = [[90, 70], [121, 64]]
    c = Paged([128, 128], news, page, Hq, Hkv, d, BF16, rb.PAGE_E4M3)
    c.write_all()
    length = torch.tensor(lens[0], dtype=torch.int32, device=DEV)
    batch = rb.PageBatch(c.batch.table, c.batch.cu, length)
    rot = _rot(d, 2)
    qkv = torch.randn(c.rows, Hq + 2 * Hkv, d, device=DEV).to(BF16)
    pos = torch.randint(0, 400, (2, c.rows), dtype=torch.int32, device=DEV)
    q, out = [torch.empty((c.rows, Hq, d), dtype=BF16, device=DEV) for _ in range(2)]
    kv = [torch.zeros((2, 1, 128, Hkv, d), dtype=BF16, device=DEV) for _ in range(2)]

    def step():
        rb.reflex_rotary_axes(qkv[:, :Hq], q, pos, rot)
        rb.reflex_pages_write(c.pages, 0, batch, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], rotary=rot, pos=pos)
        rb.reflex_pages_attention(c.pages, 0, batch, q, out, causal=True)
        rb.reflex_pages_read(c.pages, 0, batch, kv[0], kv[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for lengths in lens:
        length.copy_(torch.tensor(lengths, dtype=torch.int32))
        qkv.copy_(torch.randn(qkv.shape, device=DEV))
        graph.replay()
        replayed = [t.clone() for t in (out, *kv)]
        out.zero_()
        step()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (out, *kv)))
        c.lens = lengths
        k, v = kv[0].cpu().double(), kv[1].cpu().double()
        c.k[0], c.v[0] = [k[b, 0, :n] for b, n in enumerate(lengths)], [v[b, 0, :n] for b, n in enumerate(lengths)]
        c.check(out, c.attend(q.cpu(), causal=True))
    rb.reflex_pages_check_status(c.pages)


def test_results_do_not_depend_on_the_order_of_blocks():
    c = Paged([700, 300, 431], [1, 90, 33], 64, 8, 1, 256, BF16, rb.PAGE_INT8)
    c.write_all()
    q = c.normal(c.rows, 8, 256).to(DEV)
    first = rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.empty_like(q), causal=True).clone()
    for _ in range(5):
        assert torch.equal(first, rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.empty_like(q), causal=True))


def test_two_handles_at_once_share_pools():
    c = Paged([500, 380], [40, 20], 64, 8, 1, 128, BF16, rb.PAGE_E4M3)
    c.write_all()
    p = c.pages
    other = rb.Pages(1, c.n_pages, 64, 8, 1, 128, rb.DTYPE_BF16, rb.PAGE_E4M3, max_seqs=2, max_rows=60, k_pool=p.k_pool, v_pool=p.v_pool, k_exp=p.k_exp, v_exp=p.v_exp)
    q = [c.normal(c.rows, 8, 128).to(DEV) for _ in range(2)]
    want = [rb.reflex_pages_attention(p, 0, c.batch, x, torch.empty_like(x)).clone() for x in q]
    outs, streams = [torch.empty_like(x) for x in q], [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    for _ in range(10):
        for pages, x, o, s in zip((p, other), q, outs, streams):
            rb.reflex_pages_attention(pages, 0, c.batch, x, o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("lens,Hkv,d", [([5000], 1, 256), ([700, 2000, 33, 1500, 900, 1, 0, 1200], 1, 256), ([1300, 16, 999, 2500], 4, 128), ([3000, 1111], 2, 64)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_one_token_of_long_sequences(fmt, lens, Hkv, d):
    """Sequences whose keys many blocks of threads share, and blocks that have parts of two sequences; the same bits from every call."""
    c = Paged(lens, [min(n, 1) for n in lens], 64, 8, Hkv, d, BF16, fmt, seed=d)
    c.poison()
    c.write_all()
    q = c.normal(c.rows, 8, d)
    first = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV)).clone()
    c.check(first, c.attend(q), str(lens))
    for _ in range(4):
        assert torch.equal(first, rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV)))
    rb.reflex_pages_check_status(c.pages)


@pytest.mark.parametrize("lens,news,Hkv,d,window", [([5000], [40], 1, 256, 0), ([9000, 70], [20, 33], 2, 128, 0), ([4100], [70], 1, 64, 3000)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_a_chunk_of_a_long_sequence(fmt, lens, news, Hkv, d, window):
    """Few rows over many keys: dozens of parts of one result."""
    c = Paged(lens, news, 64, 8, Hkv, d, BF16, fmt, seed=d)
    c.poison()
    c.write_all()
    q = c.normal(c.rows, 8, d)
    first = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV), causal=True, window=window).clone()
    c.check(first, c.attend(q, causal=True, window=window), str(lens))
    for _ in range(3):
        assert torch.equal(first, rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV), causal=True, window=window))
    rb.reflex_pages_check_status(c.pages)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("at", [5, 1990])
def test_infinities_whose_weight_underflows(dtype, at):
    """An infinite value of a key that the others outweigh by 2^300 does not come out finite, wherever in the sequence it is and whoever joins the parts."""
    n, d = 2000, 128
    c = Paged([n], [1], 64, 4, 1, d, dtype, rb.PAGE_SAME)
    k, v = torch.zeros(n, 1, d, dtype=dtype), c.normal(n, 1, d)
    k[:, 0, 0] = 1.0
    k[at, 0, 0] = -1.0
    v[at, 0, 3] = float("inf")
    c.write_all(k=k, v=v)
    q = torch.zeros(1, 4, d, dtype=dtype)
    q[..., 0] = 104.0 * d ** 0.5                     # logits 104 and -104: e^208 = 2^300
    out = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV)).cpu()
    rest = [i for i in range(d) if i != 3]
    assert not torch.isfinite(out[..., 3]).any() and torch.isfinite(out[..., rest]).all()
    mean = (v.double().sum(0) - v[at].double())[:, rest] / (n - 1)
    assert ((out[0][:, rest].double() - mean).abs() <= 2.0 ** -7 * v.double()[:, 0, rest].abs().mean(0) + 1e-6).all()


@pytest.mark.parametrize("dtype,fmt", [(BF16, rb.PAGE_SAME), (BF16, rb.PAGE_INT8), (F32, rb.PAGE_E4M3)])
@pytest.mark.parametrize("news,window", [([1, 1], 0), ([40, 45], 0), ([40, 45], 50)])
def test_lengths_far_past_the_table(dtype, fmt, news, window):
    """The largest length there is: nothing is followed, the sequence reads NaN and is named, and the call ends; the other sequence is right."""
    c = Paged([100, 90], news, 32, 8, 1, 128, dtype, fmt, seed=5)
    c.write_all()
    batch = rb.PageBatch(c.batch.table, c.batch.cu, torch.tensor([100, 2 ** 31 - 1], dtype=torch.int32, device=DEV))
    q = c.normal(c.rows, 8, 128)
    out = torch.zeros((c.rows, 8, 128), dtype=dtype, device=DEV)
    rb.reflex_pages_attention(c.pages, 0, batch, q.to(DEV), out, causal=True, window=window)
    assert torch.isnan(out[news[0]:]).all()
    want = c.attend(q, causal=True, window=window)
    out[news[0]:] = want[0][news[0]:].to(DEV).to(dtype)
    c.check(out, want)
    with pytest.raises(rb.ReflexError) as e:
        rb.reflex_pages_check_status(c.pages)
    assert e.value.code == rb.ERR_STATE and "sequence 1" in str(e.value)


def test_a_table_of_too_many_positions_is_refused():
    c = Paged([100], [1], 32, 8, 1, 128, BF16, rb.PAGE_SAME)
    q = torch.zeros(1, 8, 128, dtype=BF16, device=DEV)
    b = c.batch
    desc = rb.PageBatchDesc(b.table.data_ptr(), b.cu.data_ptr(), b.length.data_ptr(), 1, (1 << 30) // 32 + 1)
    assert rb.load().reflex_pages_attention(c.pages.handle, 0, ctypes.byref(desc), q.data_ptr(), torch.empty_like(q).data_ptr(), 1, 0.0, 0, 0, None) == rb.ERR_SHAPE


def test_rows_far_into_a_pool():
    """Rows whose byte offsets pass 2^32 in the pool."""
    page, d = 128, 256
    n_pages = (5 << 30) // (page * d)                                    # 5 GB of one-byte rows
    pages = rb.Pages(1, n_pages, page, 8, 1, d, rb.DTYPE_BF16, rb.PAGE_INT8, max_seqs=1, max_rows=300)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device=DEV)
    n = 300
    k, v = [torch.randn(n, 1, d, device=DEV).to(BF16) for _ in range(2)]
    length = torch.tensor([n], dtype=torch.int32, device=DEV)
    for new in (1, n):
        batch = rb.PageBatch(table, torch.tensor([0, new], dtype=torch.int32, device=DEV), length)
        if new == 1:
            rb.reflex_pages_write(pages, 0, rb.PageBatch(table, torch.tensor([0, n], dtype=torch.int32, device=DEV), length), k, v)
            got = [torch.zeros((1, 1, n, 1, d), dtype=BF16, device=DEV) for _ in range(2)]
            rb.reflex_pages_read(pages, 0, batch, got[0], got[1])
            assert torch.equal(got[0][0, 0].cpu(), U.held(k.cpu(), rb.PAGE_INT8)[0].to(BF16)) and torch.equal(got[1][0, 0].cpu(), U.held(v.cpu(), rb.PAGE_INT8)[0].to(BF16))
        q = torch.randn(new, 8, d, device=DEV).to(BF16)
        out = rb.reflex_pages_attention(pages, 0, batch, q, torch.empty_like(q))
        w = torch.softmax(torch.einsum("nhd,kd->nhk", q.double(), got[0][0, 0, :, 0].double()) / 16, -1)
        want, mass = [torch.einsum("nhk,kd->nhd", w, x) for x in (got[1][0, 0, :, 0].double(), got[1][0, 0, :, 0].double().abs())]
        assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 1e-3) * 1.01 * mass).all()
    rb.reflex_pages_check_status(pages)


def test_refusals_of_the_binding():
    c = Paged([64], [4], 16, 8, 2, 64, BF16, rb.PAGE_INT8)
    k, q = torch.zeros(4, 2, 64, dtype=BF16, device=DEV), torch.zeros(4, 8, 64, dtype=BF16, device=DEV)
    out = torch.zeros((1, 1, 64, 2, 64), dtype=BF16, device=DEV)
    write = lambda *a, **kw: rb.reflex_pages_write(c.pages, 0, c.batch, *a, **kw)      # noqa: E731
    for bad in (lambda: write(k.float(), k), lambda: write(k, k[:3]), lambda: write(k.cpu(), k), lambda: write(k.transpose(0, 1), k),
                lambda: write(k, k.cpu()), lambda: write(q, q),
                lambda: write(k, k, rotary=_rot(64, 1), pos=torch.zeros((1, 3), dtype=torch.int32, device=DEV)),
                lambda: write(k, k, rotary=_rot(64, 1), pos=torch.zeros((1, 4), dtype=torch.int64, device=DEV)),
                lambda: rb.reflex_pages_attention(c.pages, 0, c.batch, q, q[:3].clone()), lambda: rb.reflex_pages_attention(c.pages, 0, c.batch, q.float(), q.float()),
                lambda: rb.reflex_pages_attention(c.pages, 0, c.batch, k, k.clone()),
                lambda: rb.reflex_pages_attention(c.pages, 0, rb.PageBatch(c.batch.table, c.batch.cu[:1], c.batch.length), q, q.clone()),
                lambda: rb.reflex_pages_attention(c.pages, 0, rb.PageBatch(c.batch.table.long(), c.batch.cu, c.batch.length), q, q.clone()),
                lambda: rb.reflex_pages_read(c.pages, 0, c.batch, out, out.float()), lambda: rb.reflex_pages_read(c.pages, 0, c.batch, out[..., :32], out[..., :32])):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for bad, code in ((lambda: rb.reflex_pages_attention(c.pages, 1, c.batch, q, q.clone()), rb.ERR_INVALID_ARG),
                      (lambda: rb.reflex_pages_attention(c.pages, 0, c.batch, q, q), rb.ERR_INVALID_ARG),
                      (lambda: rb.reflex_pages_attention(c.pages, 0, c.batch, torch.cat([q, q]), torch.cat([q, q])), rb.ERR_SHAPE),
                      (lambda: rb.reflex_pages_attention(c.pages, 0, c.batch, q, q.clone(), window=-1), rb.ERR_INVALID_ARG),
                      (lambda: write(k, k, pos=torch.zeros((1, 4), dtype=torch.int32, device=DEV)), rb.ERR_INVALID_ARG),
                      (lambda: write(k, k, rotary=_rot(128, 1), pos=torch.zeros((1, 4), dtype=torch.int32, device=DEV)), rb.ERR_SHAPE),
                      (lambda: rb.reflex_pages_read(c.pages, 0, c.batch, torch.cat([out, out], 1), torch.cat([out, out], 1)), rb.ERR_INVALID_ARG)):
        with pytest.raises(rb.ReflexError) as e:
            bad()
        assert e.value.code == code
    with pytest.raises(ValueError):
        rb.Pages(1, 4, 16, 8, 2, 64, rb.DTYPE_BF16, rb.PAGE_INT8, k_pool=torch.zeros(1, 4, 2, 16, 64, dtype=torch.int8, device=DEV)[..., :32])


def _attend64(q, k, v, scale, causal, window=0, length=None, allowed=2.0 ** -8 + 2e-4):
    """One sequence in 64 bits on the GPU: q [n][Hq][d], k, v [len][Hkv][d] (length: the sequence's, where it is not the rows that k has). (result, bound of the
    error as in Paged.check)."""
    (n, Hq, d), (have, Hkv) = q.shape, k.shape[:2]
    length = have if length is None else length
    p, j = torch.arange(length - n, length, device=DEV)[:, None], torch.arange(have, device=DEV)[None]
    seen = (j < length) & (j <= p if causal else True) & (j > p - window if window else True)
    out, lim = [torch.zeros((n, Hq, d), dtype=torch.float64, device=DEV) for _ in range(2)]
    for h in range(Hq):
        x, kh, vh = q[:, h].double(), k[:, h * Hkv // Hq].double(), v[:, h * Hkv // Hq].double()
        logits = (x @ kh.T * scale).masked_fill(~seen, -math.inf)
        w = torch.softmax(logits, -1).nan_to_num(0.0)              # (rows that see nothing are 0)
        slip = ((x.abs() @ kh.abs().T).masked_fill(~seen, 0.0).amax(-1, keepdim=True)) * scale * d * 2.0 ** -24
        out[:, h] = w @ vh
        lim[:, h] = HALF[BF16] * out[:, h].abs() + (allowed + have * 2.0 ** -24 + 2 * slip) * (1 + HALF[BF16]) * (w @ vh.abs()) + 1e-30
    return out, lim


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 4, 2), (128, 4, 2), (256, 2, 1)])
@pytest.mark.parametrize("every", [128, 256])
def test_logits_that_grow_from_tile_to_tile(d, Hq, Hkv, every):
    """Causal attention over 4160 keys whose logits grow by 2^9 every tile or two: the accumulator is rescaled all the way, and every call gives the same bits."""
    n = 4160
    c = Paged([n], [n], 64, Hq, Hkv, d, BF16, rb.PAGE_SAME, seed=d)
    k, v, q = c.normal(n, Hkv, d, std=0.2), c.normal(n, Hkv, d), c.normal(n, Hq, d, std=0.2)
    k[:, :, 0] = (torch.arange(n) // every)[:, None].to(BF16)
    q[:, :, 0] = 6.25                           # of 9.02 log2 units a step
    k, v, q = k.to(DEV), v.to(DEV), q.to(DEV)
    rb.reflex_pages_write(c.pages, 0, c.batch, k, v)
    first = rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.empty_like(q), scale=1.0, causal=True).clone()
    want, lim = _attend64(q, k, v, 1.0, True)
    assert ((first.double() - want).abs() <= lim).all()
    for _ in range(30):
        assert torch.equal(first, rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.empty_like(q), scale=1.0, causal=True))
    rb.reflex_pages_check_status(c.pages)


@pytest.mark.parametrize("d,Hkv", [(64, 2), (128, 2), (256, 1)])
def test_units_without_a_key_between_others(d, Hkv):
    """Hundreds of sequences, of which every second or third has new tokens and no token that they see: every pair of blocks takes a dozen units, with and without keys in
    turn (lists of units begin anew). The rows that see nothing are 0, the others are right, and every call gives the same bits."""
    shapes = [(64, 256), (20, 0), (33, 390), (64, 250), (25, 0), (17, 129)]
    news, lens = [[shapes[b % 6][i] for b in range(300)] for i in range(2)]
    c = Paged(lens, news, 64, Hkv, Hkv, d, BF16, rb.PAGE_SAME, seed=d)
    k, v, q = c.normal(sum(lens), Hkv, d, std=1.5).to(DEV), c.normal(sum(lens), Hkv, d).to(DEV), c.normal(c.rows, Hkv, d).to(DEV)
    at = torch.tensor([0] + lens).cumsum(0).tolist()
    rb.reflex_pages_write(c.pages, 0, rb.PageBatch(c.batch.table, torch.tensor(at, dtype=torch.int32, device=DEV), c.batch.length), k, v)
    first = rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.full_like(q, 7.0)).clone()
    for b, (n, length) in enumerate(zip(news, lens)):
        r = slice(int(c.cu[b]), int(c.cu[b + 1]))
        want, lim = _attend64(q[r], k[at[b]:at[b + 1]], v[at[b]:at[b + 1]], d ** -0.5, False) if length else (torch.zeros_like(q[r]).double(), 0.0)
        assert ((first[r].double() - want).abs() <= lim).all(), b
    for _ in range(10):
        assert torch.equal(first, rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.full_like(q, 7.0)))
    rb.reflex_pages_check_status(c.pages)


def _at_16(t):
    """The same rows 16 bytes behind a multiple of 32."""
    step = 16 // t.element_size()
    room = torch.zeros(t.numel() + 2 * step, dtype=t.dtype, device=t.device)
    assert room.data_ptr() % 32 == 0
    y = room[step:step + t.numel()].view(t.shape)
    y.copy_(t)
    return y


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("news", [[1, 1], [40, 70]])
def test_rows_at_16_bytes(fmt, dtype, news):
    """Every tensor of rows 16 bytes behind a multiple of 32, which is all that is asked of it: the same bits."""
    d, Hq, Hkv = 128, 4, 2
    c = Paged([90, 170], news, 32, Hq, Hkv, d, dtype, fmt)
    c.write_all()
    rot = _rot(d, 2)
    pos = torch.randint(0, 400, (2, c.rows), dtype=torch.int32, device=DEV)
    rows = c.normal(c.rows, Hq + 2 * Hkv, d).to(DEV)
    results = []
    for place in (lambda t: t, _at_16):
        x = place(rows)
        q, out = [place(torch.zeros((c.rows, Hq, d), dtype=dtype, device=DEV)) for _ in range(2)]
        kv = [place(torch.zeros((2, 1, 170, Hkv, d), dtype=dtype, device=DEV)) for _ in range(2)]
        rb.reflex_rotary_axes(x[:, :Hq], q, pos, rot)
        rb.reflex_pages_write(c.pages, 0, c.batch, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], rotary=rot, pos=pos)
        rb.reflex_pages_attention(c.pages, 0, c.batch, q, out, causal=True)
        rb.reflex_pages_read(c.pages, 0, c.batch, kv[0], kv[1])
        kv_mixed = [kv[0].clone(), place(torch.zeros_like(kv[1]))]                 # (one of the two at a multiple of 32)
        rb.reflex_pages_read(c.pages, 0, c.batch, kv_mixed[0], kv_mixed[1])
        results.append([t.clone() for t in (q, out, *kv, *kv_mixed)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("Hq,Hkv,n_rows,max_pages", [(1024, 4, 65536, 1024), (4096, 1, 600000, 1), (4096, 1, 524288, 1), (1024, 8, 65536, 1024)])
def test_lines_of_more_work_than_31_bits_count_are_refused(Hq, Hkv, n_rows, max_pages):
    """... whichever kernel would count it: groups of 129 to 4096 heads as well. (Nothing is launched: the rows do not exist.)"""
    pages = rb.Pages(1, 4, 128, Hq, Hkv, 128, rb.DTYPE_BF16, rb.PAGE_INT8, max_seqs=1, max_rows=n_rows)
    table, cu, length, rows = [torch.zeros(max(n, 64), dtype=torch.int32, device=DEV) for n in (max_pages, 2, 1, 64)]
    desc = rb.PageBatchDesc(table.data_ptr(), cu.data_ptr(), length.data_ptr(), 1, max_pages)
    before = rb.reflex_kernel_launch_count()
    assert rb.load().reflex_pages_attention(pages.handle, 0, ctypes.byref(desc), rows.data_ptr(), rows.data_ptr() + 64, n_rows, 0.0, 0, 0, None) == rb.ERR_SHAPE
    assert rb.reflex_kernel_launch_count() == before


@pytest.mark.parametrize("dtype,fmt", [(BF16, rb.PAGE_SAME), (BF16, rb.PAGE_INT8), (F32, rb.PAGE_SAME)])
@pytest.mark.parametrize("lens,news", [([5, 40], [9, 1]), ([30, 200], [70, 90])])
@pytest.mark.parametrize("causal", [False, True])
def test_the_largest_window(dtype, fmt, lens, news, causal):
    """A window that limits nothing, over rows in front of the first token too (more new tokens than tokens)."""
    c = Paged(lens, news, 16, 8, 1, 128, dtype, fmt, seed=4)
    c.write_all()
    q = c.normal(c.rows, 8, 128)
    want = c.attend(q, causal=causal)
    for window in (2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30):
        out = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.full_like(q, 7.0, device=DEV), causal=causal, window=window)
        c.check(out, want, str(window))
    assert causal or bool((want[0][0] != 0).all())           # the first row, far in front of the first token, sees all of them


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (BF16, 256), (F32, 64)])
@pytest.mark.parametrize("news", [[1, 1, 1], [40, 70, 33]])
@pytest.mark.parametrize("page,gone", [(16, -1), (64, 10 ** 6)])
def test_pages_in_front_of_the_window_may_be_gone(fmt, dtype, d, news, page, gone):
    """A sequence keeps the pages that its window reaches. The table's entries of the others, and rows that are not finite in front of the window, change nothing."""
    lens, window = [700, 333, 1090], 100
    c = Paged(lens, news, page, 4, 1, d, dtype, fmt, seed=d + news[0])
    total = sum(lens)
    k, v = c.normal(total, 1, d, std=1.5), c.normal(total, 1, d)
    table, at = c.table.clone(), 0
    for b, (n, m) in enumerate(zip(lens, news)):
        first = max(0, n - m - window + 1)                 # that the first new token sees
        k[at + first - 1], v[at + first - 1] = math.nan, math.inf
        table[b, :first // page] = gone
        at += n
    c.write_all(k=k, v=v)
    q = c.normal(c.rows, 4, d)
    batch = rb.PageBatch(table.to(DEV), c.batch.cu, c.batch.length)
    for causal in (True, False):
        out = rb.reflex_pages_attention(c.pages, 0, batch, q.to(DEV), torch.full_like(q, 7.0, device=DEV), causal=causal, window=window)
        c.check(out, c.attend(q, causal=causal, window=window), f"causal {causal}")
        rb.reflex_pages_check_status(c.pages)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("adjacent", [False, True])
def test_pairs_that_do_not_turn_stay_as_they_are(dtype, adjacent):
    """Frequency 0, or an axis without positions: to the bit, whatever lies in the pair's other element (infinities, NaN, -0)."""
    n, H, d, R = 6, 3, 64, 48
    g = torch.Generator().manual_seed(1)
    x = torch.randn(n, H, d, generator=g).to(dtype)
    odd = torch.tensor([math.inf, -math.inf, math.nan, -0.0, 0.0])
    at = torch.randint(0, n * H * d, (n * H * 12,), generator=g)
    x.view(-1)[at] = odd[torch.arange(len(at)) % 5].to(dtype)
    rot = _rot(R, 3, adjacent)
    rot.freq[::5] = 0.0                                                       # pairs 0, 5, 10 ...
    pos = torch.randint(1, 3000, (2, n), generator=g, dtype=torch.int32)      # no positions of axis 2
    still = (rot.freq == 0).cpu() | (rot.axis >= 2).cpu()
    columns = torch.cat([still.repeat_interleave(2) if adjacent else still.repeat(2), torch.ones(d - R, dtype=torch.bool)])
    bits = lambda t: t.contiguous().view(torch.int16 if dtype == BF16 else torch.int32)        # noqa: E731
    y = rb.reflex_rotary_axes(x.to(DEV), torch.empty((n, H, d), dtype=dtype, device=DEV), pos.to(DEV), rot).cpu()
    assert torch.equal(bits(y[..., columns]), bits(x[..., columns]))
    c = Paged([n], [n], 16, H, H, d, dtype, rb.PAGE_SAME)
    rb.reflex_pages_write(c.pages, 0, c.batch, x.to(DEV), x.to(DEV), rotary=rot, pos=pos.to(DEV))
    k, v = _read(c)
    assert torch.equal(bits(k[0, 0][..., columns]), bits(x[..., columns])) and torch.equal(bits(v[0, 0]), bits(x))
    assert _same(k[0, 0], y)                                                  # both turn alike


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("adjacent", [False, True])
def test_frequencies_without_an_angle(dtype, adjacent):
    """NaN, infinities and what no angle is kept for make their pairs NaN, and no others (an axis without positions: not turned, whatever its frequency)."""
    n, d, R = 5, 64, 32
    x = torch.randn(n, 2, d).to(dtype)
    rot = _rot(R, 3, adjacent)
    odd = {0: math.nan, 3: math.inf, 6: -math.inf, 9: 2.0 ** 40, 12: -3e38, 2: math.nan, 5: math.inf}           # pairs 2 and 5: axis 2
    for i, f in odd.items():
        rot.freq[i] = f
    rot.freq[7], rot.freq[10] = 1.5 * 2 ** 20, -(2.0 ** 24) + 1
    pos = torch.randint(-3000, 3000, (2, n), dtype=torch.int32)
    pos[:, 0] = 0
    lost = torch.tensor([i in odd and i % 3 < 2 for i in range(R // 2)])
    lost = torch.cat([lost.repeat_interleave(2) if adjacent else lost.repeat(2), torch.zeros(d - R, dtype=torch.bool)])
    freq = torch.where(torch.isfinite(rot.freq) & (rot.freq.abs() < 2.0 ** 40), rot.freq, 0.0).cpu()
    want = U.rotated(x, pos, freq, rot.axis.cpu(), adjacent)
    # (angles of 2^24 * 3000 in 64 bits lose 2^-53 of themselves in the reference: 2^-17 of a radian)
    lim = HALF[dtype] * want.abs() + x.double().abs().amax(-1, keepdim=True) * 2 * (2.0 ** -17 + 2.0 ** -20)
    y = rb.reflex_rotary_axes(x.to(DEV), torch.empty((n, 2, d), dtype=dtype, device=DEV), pos.to(DEV), rot).cpu()
    assert torch.isnan(y[..., lost]).all() and ((y.double() - want).abs() <= lim)[..., ~lost].all()
    c = Paged([n], [n], 16, 2, 2, d, dtype, rb.PAGE_SAME)
    rb.reflex_pages_write(c.pages, 0, c.batch, x.to(DEV), x.to(DEV), rotary=rot, pos=pos.to(DEV))
    assert _same(_read(c)[0][0, 0], y)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("news,at", [(1, 5), (1, 4950), (40, 5), (40, 4950)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_large_values_whose_weight_underflows(dtype, fmt, news, at):
    """A value of 1e38 of a key that another one outweighs by 2^300 adds nothing, wherever in the sequence it is and whoever joins the parts (40 rows: dozens of them)."""
    n, d = 5000, 128
    c = Paged([n], [news], 64, 4, 1, d, dtype, fmt)
    k, v = torch.zeros(n, 1, d, dtype=dtype), c.normal(n, 1, d)
    k[:, 0, 0] = -1.0
    k[2500, 0, 0] = 1.0
    v[at, 0, 3::5] = 1e38
    c.write_all(k=k, v=v)
    q = torch.zeros(news, 4, d, dtype=dtype)
    q[..., 0] = 104.0 * d ** 0.5                     # logits -104, and 104 of the one key: e^208 = 2^300
    out = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV))
    one = c.attend(q[:1].expand(news, -1, -1)) if news == 1 else None
    if one is None:                                  # (all rows are alike)
        c.news, c.cu, c.rows = [1], torch.tensor([0, 1], dtype=torch.int32), 1
        one = c.attend(q[:1])
        for i in range(news):
            c.check(out[i:i + 1], one, f"row {i}")
    else:
        c.check(out, one)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (BF16, 256), (F32, 64)])
@pytest.mark.parametrize("news", [1, 40])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [2.0 ** 127, 1e-26])
def test_values_of_any_size(dtype, d, news, fmt, size):
    """Values of half to all of 2^127, all of one sign, and of 1e-26, under logits that rise by almost 2^8 behind the first keys: their weighted sum is finite ahead of the division,
    and as exact as any other."""
    n = 1500
    c = Paged([n, 300], [news, 1], 32, 4, 1, d, dtype, fmt, seed=d)
    k, v = torch.zeros(n + 300, 1, d, dtype=dtype), ((0.5 + 0.5 * torch.rand(n + 300, 1, d, generator=c.g)) * size).to(dtype)
    v[:, :, 1::2] *= -1.0
    k[150:, :, 0] = 1.0
    c.write_all(k=k, v=v)
    q = c.normal(c.rows, 4, d)
    q[..., 0] = 5.4 * d ** 0.5                       # logits 0, then 5.4 = 7.8 log2 units
    out = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.zeros_like(q, device=DEV), causal=True)
    c.check(out, c.attend(q, causal=True))


def test_rotary_of_as_many_tokens_as_there_can_be():
    """2^31 - 1 tokens, in place (69 GB of rows): counts of tokens do not pass 32 bits on the way to the launch."""
    n, d = 2 ** 31 - 1, 16
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("rows and positions take 77 GB")
    x, pos = torch.zeros((n, 1, d), dtype=BF16, device=DEV), torch.zeros((1, n), dtype=torch.int32, device=DEV)
    at = [0, 1, 2 ** 30, n - 257, n - 1]
    for i in at:
        x[i, 0], pos[0, i] = 1.0, i
    rot = _rot(d, 1)
    rb.reflex_rotary_axes(x, x, pos, rot)
    for i in at:
        want = U.rotated(torch.ones(1, 1, d), torch.tensor([[i]]), rot.freq.cpu(), rot.axis.cpu())
        # (angles of 2^31 in 64 bits: 2^-22; products and sum; half a step of the result)
        assert ((x[i, 0].cpu().double() - want[0, 0]).abs() <= HALF[BF16] * want[0, 0].abs() + 2 * (2.0 ** -22 + 2.0 ** -20)).all(), i
    del x, pos
    torch.cuda.empty_cache()


@pytest.mark.parametrize("raw", [False, True])
def test_pages_made_for_another_stream(raw):
    """Calls on the stream that the pages were made for come behind the zeroing of the pools, which the current stream does (6 GB here)."""
    side = torch.cuda.Stream()
    n, d, page = 64, 128, 16
    k, v = [torch.randn(n, 1, d, device=DEV).to(BF16) for _ in range(2)]
    n_pages = (3 << 30) // (page * d * 2)
    table = torch.tensor([[n_pages - 1, 5, n_pages // 2, 7]], dtype=torch.int32, device=DEV)
    batch = rb.PageBatch(table, torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV))
    out = [torch.zeros((1, 1, n, 1, d), dtype=BF16, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    on = side.cuda_stream if raw else side
    pages = rb.Pages(1, n_pages, page, 1, 1, d, rb.DTYPE_BF16, max_seqs=1, max_rows=n, stream=on)
    rb.reflex_pages_write(pages, 0, batch, k, v, stream=on)
    side.synchronize()
    torch.cuda.synchronize()
    rb.reflex_pages_read(pages, 0, batch, out[0], out[1])
    assert torch.equal(out[0][0, 0], k) and torch.equal(out[1][0, 0], v)
    with torch.cuda.stream(side):                   # and the other way round: made for the NULL stream while another one is current
        pages = rb.Pages(1, 4, page, 1, 1, d, rb.DTYPE_BF16, max_seqs=1, max_rows=n, stream=0)
    rb.reflex_pages_check_status(pages)


def _check_each(c, q, out, causal, window=0):
    """Every sequence of c (filled by write_all) against 64 bits, on the GPU."""
    for b, n in enumerate(c.news):
        if n == 0:
            continue
        r = slice(int(c.cu[b]), int(c.cu[b + 1]))
        want, lim = _attend64(q[r], c.k[0][b].to(DEV), c.v[0][b].to(DEV), c.d ** -0.5, causal, window)
        assert ((out[r].double() - want).abs() <= lim).all(), b


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["tokens", "a chunk among tokens", "chunks among tokens", "idle"])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 4, 2), (128, 16, 2), (256, 8, 1)])
def test_more_sequences_than_a_warp_has_lanes(fmt, kind, d, Hq, Hkv):
    """100 sequences: the walk along the line of work goes on in further blocks of 32; batches whose sequences are nothing like their average."""
    B = 100
    lens = [1 + (b * 97) % 130 for b in range(B)]
    news = {"tokens": [1] * B, "a chunk among tokens": [1] * 70 + [300] + [1] * 29, "chunks among tokens": [90 if b % 9 == 4 else 1 for b in range(B)],
            "idle": [0] * 40 + [2] + [0] * 58 + [40]}[kind]
    lens = [max(x, n) for x, n in zip(lens, news)]
    c = Paged(lens, news, 16, Hq, Hkv, d, BF16, fmt, seed=d, spare_rows=2)
    c.poison()
    k = c.normal(sum(lens), Hkv, d, std=1.5)
    c.write_all(k=k, v=c.normal(sum(lens), Hkv, d))
    q = c.normal(c.rows, Hq, d).to(DEV)
    first = rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.full_like(q, 7.0), causal=True).clone()
    _check_each(c, q, first, True)
    assert (first[int(c.cu[-1]):] == 7.0).all()
    for _ in range(3):
        assert torch.equal(first, rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.full_like(q, 7.0), causal=True))
    rb.reflex_pages_check_status(c.pages)


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 1), (128, 8, 1), (256, 8, 1)])
@pytest.mark.parametrize("news", [1, 2])
@pytest.mark.parametrize("every", [16, 100, 1000])
def test_logits_that_grow_under_few_tokens(d, Hq, Hkv, news, every):
    """The kernel of few tokens: running maxima that grow by 2^9 every block of keys, or from one part of a sequence to the next."""
    n = 4000
    c = Paged([n, 900], [news, news], 64, Hq, Hkv, d, BF16, rb.PAGE_SAME, seed=d)
    k, v, q = c.normal(n + 900, Hkv, d, std=0.2), c.normal(n + 900, Hkv, d), c.normal(c.rows, Hq, d, std=0.2)
    k[:, :, 0] = (torch.arange(n + 900) % n // every)[:, None].to(BF16)
    q[:, :, 0] = 6.25                           # of 9.02 log2 units a step
    c.write_all(k=k, v=v)
    out = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.empty_like(q, device=DEV), scale=1.0, causal=True)
    for b in range(2):
        r = slice(int(c.cu[b]), int(c.cu[b + 1]))
        want, lim = _attend64(q[r].to(DEV), c.k[0][b].to(DEV), c.v[0][b].to(DEV), 1.0, True)
        assert ((out[r].double() - want).abs() <= lim).all(), b


@pytest.mark.parametrize("dtype,fmt", [(BF16, rb.PAGE_SAME), (BF16, rb.PAGE_E4M3), (F32, rb.PAGE_SAME)])
@pytest.mark.parametrize("news", [1, 40])
def test_the_largest_scales(dtype, fmt, news):
    """A scale of 2e38 is one (times log2 e still finite); above it, and NaN, are refused."""
    c = Paged([200], [news], 32, 4, 1, 128, dtype, fmt)
    k, v = c.normal(200, 1, 128), c.normal(200, 1, 128)
    c.write_all(k=k * 2.0 ** -60, v=v)
    q = c.normal(c.rows, 4, 128) * 2.0 ** -70                   # q k of about 2^-127, logits of about 1
    out = rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.empty_like(q, device=DEV), scale=2e38 if news == 1 else 1.5e38)
    # (products and sums down there are subnormal: steps of 2^-149 each, of which 2 * 128 and the weights' exponents are a logit's error)
    want, mass, slip = c.attend(q, scale=2e38 if news == 1 else 1.5e38)
    c.check(out, (want, mass, slip + 2 * 128 * 2.0 ** -149 * 2e38))
    for scale in (3e38, math.inf, math.nan):
        with pytest.raises(rb.ReflexError) as e:
            rb.reflex_pages_attention(c.pages, 0, c.batch, q.to(DEV), torch.empty_like(q, device=DEV), scale=scale)
        assert e.value.code == rb.ERR_INVALID_ARG


@pytest.mark.parametrize("d,G", [(64, 8), (128, 8), (256, 8), (256, 1)])
@pytest.mark.parametrize("fmt", [rb.PAGE_SAME, rb.PAGE_E4M3])
def test_long_runs_of_units_without_a_key(d, G, fmt):
    """New tokens that see nothing (sequences of no token; more new tokens than tokens, causal) fill the lists of units between those that see something, and behind the last one."""
    lens = [130, 0, 300, 0, 64, 5, 700, 0, 0, 90, 2, 0]
    news = [40, 900, 70, 2500, 64, 1200, 33, 300, 700, 90, 800, 2000]
    c = Paged(lens, news, 32, 4 * G, 4, d, BF16, fmt, seed=d + G)
    c.poison()
    c.write_all()
    q = c.normal(c.rows, 4 * G, d).to(DEV)
    for causal in (True, False):
        out = rb.reflex_pages_attention(c.pages, 0, c.batch, q, torch.full_like(q, 7.0), causal=causal)
        rb.reflex_pages_check_status(c.pages)
        for b, (n, length) in enumerate(zip(news, lens)):
            r = slice(int(c.cu[b]), int(c.cu[b + 1]))
            if length == 0:
                assert (out[r] == 0).all(), b
                continue
            want, lim = _attend64(q[r], c.k[0][b].to(DEV), c.v[0][b].to(DEV), d ** -0.5, causal)
            assert ((out[r].double() - want).abs() <= lim).all(), b
