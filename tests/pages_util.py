"""The paged prefix in 64 bits, written from its definitions (rotation, 8-bit rows, pages, attention), for the tests."""
import math

import torch

from paper_2607_14695_b200 import binding as rb

DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}     # half a step, relative
TOP = {rb.PAGE_INT8: 127.0, rb.PAGE_E4M3: 448.0}


def rotated(x, pos, freq, axis, adjacent=False, inverse=False):
    """x [n][H][d]; a loop over the pairs."""
    y = x.double().clone()
    for i, (f, a) in enumerate(zip(freq.double().tolist(), axis.tolist())):
        t = pos[a].double() * f * (-1.0 if inverse else 1.0) if a < pos.shape[0] else torch.zeros(x.shape[0], dtype=torch.float64)
        u, w = (2 * i, 2 * i + 1) if adjacent else (i, i + len(freq))
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        y[..., u] = x[..., u].double() * c - x[..., w].double() * s
        y[..., w] = x[..., u].double() * s + x[..., w].double() * c
    return y


def held(x, fmt):
    """What a page holds of rows x [..., d] in 64 bits: (values, exponent bytes). Rows in dtype: as they are."""
    x = x.double()
    if fmt == rb.PAGE_SAME:
        return x, None
    flat = x.reshape(-1, x.shape[-1])
    out, exps = torch.empty_like(flat), torch.empty(flat.shape[0], dtype=torch.uint8)
    for r, row in enumerate(flat):
        if not torch.isfinite(row).all():
            out[r], exps[r] = math.nan, 255
            continue
        row = row.clamp(-2.0 ** 127, 2.0 ** 127)
        e, top = -100, row.abs().max().item()
        while top > TOP[fmt] * 2.0 ** e:
            e += 1
        u = row * 2.0 ** -e
        if fmt == rb.PAGE_INT8:
            q = torch.round(u)
        else:               # e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6
            step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
            q = torch.round(u / step) * step
        out[r], exps[r] = q * 2.0 ** e, e + 127
    return out.reshape(x.shape), exps.reshape(x.shape[:-1])


class Paged:
    """Sequences in pages of a random order, on both sides: rb.Pages on the GPU, and the rows that they stand for in 64 bits."""

    def __init__(self, lens, news, page, Hq, Hkv, d, dtype, fmt, L=1, seed=0, spare_rows=0, spare_pages=3, max_seqs=None):
        self.g = torch.Generator().manual_seed(seed)
        self.lens, self.news, self.page, self.Hq, self.Hkv, self.d, self.dtype, self.fmt, self.L = lens, news, page, Hq, Hkv, d, dtype, fmt, L
        B, used = len(lens), [-(-n // page) for n in lens]
        self.n_pages = max(1, sum(used) + spare_pages)
        order = torch.randperm(self.n_pages, generator=self.g).to(torch.int32)
        self.table = torch.full((B, max(1, max(used))), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(used):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.cu = torch.tensor([0] + list(torch.tensor(news).cumsum(0).tolist()), dtype=torch.int32)
        self.rows = int(self.cu[-1]) + spare_rows
        self.pages = rb.Pages(L, self.n_pages, page, Hq, Hkv, d, rb.DTYPE_F32 if dtype == torch.float32 else rb.DTYPE_BF16, fmt, max_seqs=max_seqs or B, max_rows=max(1, self.rows))
        self.batch = rb.PageBatch(self.table.to(DEV), self.cu.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV))
        self.k = [[torch.zeros(n, Hkv, d, dtype=torch.float64) for n in lens] for _ in range(L)]
        self.v = [[torch.zeros(n, Hkv, d, dtype=torch.float64) for n in lens] for _ in range(L)]

    def normal(self, *shape, std=1.0):
        return (torch.randn(*shape, generator=self.g) * std).to(self.dtype)

    def poison(self):
        """Whatever no token was written to is NaN, or as near to it as the format comes."""
        for pool in (self.pages.k_pool, self.pages.v_pool):
            pool.view(torch.uint8).fill_(0x7F if self.fmt != rb.PAGE_SAME else 0xFF)
        for e in (self.pages.k_exp, self.pages.v_exp):
            if e is not None:
                e.fill_(255)

    def write_all(self, layer=0, k=None, v=None):
        """All tokens of all sequences (as one chunk each)."""
        total = sum(self.lens)
        k = self.normal(total, self.Hkv, self.d, std=1.5) if k is None else k
        v = self.normal(total, self.Hkv, self.d) if v is None else v
        cu = torch.tensor([0] + torch.tensor(self.lens).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
        rb.reflex_pages_write(self.pages, layer, rb.PageBatch(self.batch.table, cu, self.batch.length), k.to(DEV), v.to(DEV))
        at = 0
        for b, n in enumerate(self.lens):
            self.k[layer][b], self.v[layer][b] = held(k[at:at + n], self.fmt)[0], held(v[at:at + n], self.fmt)[0]
            at += n
        return k, v

    def attend(self, q, layer=0, causal=False, window=0, scale=None):
        """(result, sum of weights times |v|, bound of a logit's error in fp32) of every row in 64 bits; rows behind the last sequence are None."""
        G, scale = self.Hq // self.Hkv, self.d ** -0.5 if scale is None else scale
        out, mass, slip = [torch.zeros(self.rows, self.Hq, self.d, dtype=torch.float64) for _ in range(2)] + [torch.zeros(self.rows, self.Hq, dtype=torch.float64)]
        for b, (n, length) in enumerate(zip(self.news, self.lens)):
            r0 = int(self.cu[b])
            for i in range(n):
                p = length - n + i
                hi, lo = (min(length, p + 1) if causal else length), (max(0, p - window + 1) if window else 0)
                if hi <= lo:
                    continue
                for h in range(self.Hq):
                    k, v = self.k[layer][b][lo:hi, h // G], self.v[layer][b][lo:hi, h // G]
                    x = q[r0 + i, h].double()
                    w = torch.softmax((k @ x) * scale, 0)
                    out[r0 + i, h], mass[r0 + i, h] = w @ v, w @ v.abs()
                    slip[r0 + i, h] = (k.abs() @ x.abs()).max() * scale * self.d * 2.0 ** -24
        return out, mass, slip

    def check(self, got, want, what=""):
        """got against attend()'s answer. Weights: rounded to bf16 before they meet V (2^-8 each), exponentials good to 1e-4 (tensor cores) or 2^-20,
        logits to `slip` in fp32 (twice, in numerator and sum); sums of fp32 products: 2^-24 a term, at most as many as keys; one rounding at the end."""
        out, mass, slip = want
        got = got[:int(self.cu[-1])].double().cpu()
        out, mass, slip = [t[:int(self.cu[-1])] for t in want]
        fast = self.dtype == torch.bfloat16
        rel = (2.0 ** -8 + 2e-4 if fast else 2.0 ** -19) + max(self.lens) * 2.0 ** -24 + 2 * slip[..., None]
        lim = HALF[self.dtype] * out.abs() + rel * (1 + HALF[self.dtype]) * mass + 1e-30
        err = (got - out).abs()
        assert torch.isfinite(got).all(), f"{what}: {(~torch.isfinite(got)).sum()} values not finite"
        bad = err > lim
        assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((err / lim).max()):.2f} of it; first {bad.nonzero()[0].tolist()}"
