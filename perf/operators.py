"""Cases of the paged prefix: what a vision-language backbone does, tick by tick, to the keys and values of an observation.

The action expert attends to a prefix that the backbone encodes. In streaming use only the newest frame is encoded: its tokens
are rotated by their positions in time, height and width, their keys and values go into pages (quantised as they are written),
they attend to everything the pages hold, and the finished prefix is read back for the expert. Four operators:

  rotary     rotary positions with several axes, forward and inverse (the inverse is also the gradient)
  write      keys and values of new tokens into the pages, keys rotated on the way, 8-bit formats quantised; the written rows
             are read back, so that the result is the values that the pages stand for
  read       whole sequences of all layers read back from the pages
  attention  a chunk of new tokens (one to thousands per sequence) over the pages

Sizes are those of this repository's configurations and tests (8 query heads on one KV head of 256, prefixes of 816 and 4160
tokens, frames of 256 tokens, windows of ten frames, 16 heads on 4 KV heads of 128) and ranges around them.
A row (token, head) in an 8-bit page is d integers or e4m3 numbers times 2^(e - 127), e one byte per row; e = 255 marks a row
that held an infinity or a NaN.
"""
from __future__ import annotations

import torch

own = False

DEV = "cuda:0"
FAR = 2.0 ** 127                       # larger magnitudes are held as this
E_MIN = -100                           # smallest exponent of a row's scale
LARGEST = {"e4m3": (448.0, 1.75, 8), "int8": (127.0, 1.984375, 6)}      # value = mantissa 2^exponent

ROTARY = dict(kind="rotary", dtype="bf16", n=256, H=9, d=256, R=256, axes=3, adjacent=False, inverse=False, spare=1, far=False)
PAGED = dict(dtype="bf16", fmt="e4m3", B=1, n=256, len=816, ragged=False, holes=False, page=64, Hkv=1, d=256)
WRITE = dict(PAGED, kind="write", rotary=True)
READ = dict(PAGED, kind="read", L=18, n=0)
ATTENTION = dict(PAGED, kind="attention", Hq=8, causal=False, window=0, pad=0)


def listed():
    return [
        # the queries and keys of a batch of ten-frame windows, straight from the packed projection
        dict(ROTARY, name="rotary_frames", n=40960),
        # gradient of a long video's rotation in fp32: an odd number of tokens, adjacent pairs, only 96 of 128 dimensions rotated
        dict(ROTARY, name="rotary_video_grad", dtype="f32", n=8191, H=16, d=128, R=96, adjacent=True, inverse=True, spare=0, far=True),
        # the smallest write: one new token for each of 64 streams
        dict(WRITE, name="write_tick", B=64, n=1, len=817),
        # the newest frame of 16 streams, uneven lengths, several heads
        dict(WRITE, name="write_frame", fmt="int8", B=16, n=256, len=1072, ragged=True, page=32, Hkv=4, d=128),
        # long prefixes of 16 streams at once, keys encoded already
        dict(WRITE, name="write_prefix", B=16, n=4160, len=4160, rotary=False),
        # one stream's prefix for the action expert, all layers
        dict(READ, name="read_stream"),
        # the long prefixes of a batch, all layers
        dict(READ, name="read_streams", fmt="int8", B=16, len=4160, ragged=True),
        # one token of one stream over an unquantised prefix: latency
        dict(ATTENTION, name="attention_token", fmt="same", n=1, len=817),
        # one token of each of 64 streams over long uneven contexts
        dict(ATTENTION, name="attention_token_64", fmt="int8", B=64, n=1, len=4416, ragged=True),
        # one robot's incremental prefill: the newest frame over prefix and ten frames
        dict(ATTENTION, name="attention_frame", fmt="same", n=256, len=3376),
        # the same for 16 robots, 8-bit pages
        dict(ATTENTION, name="attention_frames_16", B=16, n=256, len=3376),
        # first prefill of long prompts under a causal mask, grouped heads of 128, uneven lengths
        dict(ATTENTION, name="attention_prefill", fmt="same", B=4, n=4160, len=4160, ragged=True, Hq=16, Hkv=4, d=128, causal=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["rotary", "write", "read", "attention", "attention", "attention"])
    if kind == "rotary":
        d = rng.choice([64, 128, 256])
        H = rng.randint(1, 24)
        return dict(ROTARY, dtype=rng.choice(["bf16", "bf16", "f32"]), n=_log_int(rng, 1, max(1, 40000 * 256 // (d * H))), H=H, d=d, R=rng.choice([d, d, d // 2, 3 * d // 4]),
                    axes=rng.randint(1, 4), adjacent=rng.random() < 0.5, inverse=rng.random() < 0.3, spare=rng.randint(0, 2), far=rng.random() < 0.3)
    heads = dict(Hkv=rng.choice([1, 1, 2, 4, 8]), d=rng.choice([64, 128, 256, 256]), page=rng.choice([16, 32, 64, 128]))
    B = _log_int(rng, 1, 64)
    some = dict(heads, B=B, ragged=rng.random() < 0.6, holes=B >= 4 and rng.random() < 0.3, fmt=rng.choice(["e4m3", "int8", "same"]))
    width = heads["Hkv"] * heads["d"]
    if kind == "write":
        n = _log_int(rng, 1, max(1, min(4160, 16 * 4160 * 256 // (B * width))))
        # (unquantised fp32 pages, or quantised ones of keys as they are: fp32 rows rotated and quantised would differ by a step where rounding ties)
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        rotary = rng.random() < 0.7 if dtype == "bf16" or some["fmt"] == "same" else False
        return dict(WRITE, **some) | dict(n=n, len=n + (rng.randint(0, 2000) if rng.random() < 0.7 else 0), dtype=dtype, rotary=rotary)
    if kind == "read":
        L = rng.randint(1, 18)
        return dict(READ, **some) | dict(L=L, len=_log_int(rng, 1, max(1, min(4160, 16 * 18 * 4160 * 128 // (B * L * width)))), dtype="f32" if rng.random() < 0.15 else "bf16")
    form = rng.choice(["token", "token", "few", "chunk", "chunk", "prefill", "fp32"])
    if form == "fp32":
        return dict(ATTENTION, **some) | dict(dtype="f32", B=min(B, 4), Hkv=rng.choice([1, 2]), Hq=rng.choice([2, 4, 8]), d=64, n=rng.randint(1, 40), len=rng.randint(40, 600), causal=rng.random() < 0.5)
    case = dict(ATTENTION, **some) | dict(Hq=heads["Hkv"] * rng.choice([1, 2, 4, 7, 8]), causal=rng.random() < 0.6)
    if form in ("token", "few"):
        case["n"] = 1 if form == "token" else rng.randint(2, 40)
        case["len"] = case["n"] + _log_int(rng, 1, max(64, min(12800, 64 * 4416 * 128 // (B * width))))
    else:
        case["B"] = min(B, 16)
        case["holes"] = case["holes"] and case["B"] >= 4
        keys = 16 * 2048 * 3376 // (case["B"] * case["Hq"])                # queries times keys of a sequence
        keys = min(keys, (96 << 20) // (case["B"] * heads["Hkv"]) if form == "prefill" else keys) * 256 // max(256, heads["d"])
        case["n"] = _log_int(rng, 40, max(41, min(4160, int(keys ** 0.5) if form == "prefill" else max(41, keys // 1000))))
        case["len"] = case["n"] if form == "prefill" else case["n"] + rng.randint(0, max(1, min(8000, keys // case["n"] - case["n"])))
    if rng.random() < 0.25:
        case["window"] = rng.randint(1, case["len"])
    if rng.random() < 0.3:
        case["pad"] = rng.randint(1, 40)
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _sequences(c):
    """(new tokens, tokens after them) of every sequence. Idle streams (holes) have no new token, some of them no token at all."""
    out = []
    for b in range(c["B"]):
        n, length = c["n"], c["len"]
        if c["ragged"]:
            fresh = c["n"] == c["len"]
            n = n - (b * 13) % max(1, n // 2)
            length = n if fresh else max(n, length - (b * 37) % max(1, length // 2))
        if c["holes"] and b % 4 == 3:
            length = 0 if b % 8 == 7 else (length if c["kind"] == "read" else length - n)
            n = 0
        out.append((n, length))
    return out


class _Inputs:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32).to(dtype)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV, dtype=torch.int32)


def _rotation(R, axes):
    """Frequencies of the R / 2 pairs and the axis each follows, as a model's configuration gives them: axes in turn."""
    i = torch.arange(R // 2, dtype=torch.float64)
    return (10000.0 ** (-2.0 * i / R)).float().to(DEV), (i % axes).to(torch.uint8).to(DEV)


def _pages(c, rnd, L):
    """Pages of L layers in which the sequences' tokens lie in random order of pages, and the device's page table and lengths."""
    seqs, P = _sequences(c), c["page"]
    most = max(1, max(-(-length // P) for _, length in seqs))
    used = [-(-length // P) for _, length in seqs]
    n_pages = sum(used) + 3
    order = torch.randperm(n_pages, generator=rnd.g, device=DEV).to(torch.int32)
    table = torch.full((c["B"], most), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(used):
        table[b, :m] = order[at:at + m]
        at += m
    cu = [0]
    for n, _ in seqs:
        cu.append(cu[-1] + n)
    s = dict(table=table, cu=torch.tensor(cu, dtype=torch.int32, device=DEV), length=torch.tensor([x for _, x in seqs], dtype=torch.int32, device=DEV))
    shape = (L, n_pages, c["Hkv"], P, c["d"])
    kind = {"same": _dtype(c), "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[c["fmt"]]
    for x in ("k", "v"):
        s[x + "_pool"] = torch.zeros(shape, dtype=kind, device=DEV)
        s[x + "_exp"] = torch.zeros(shape[:-1], dtype=torch.uint8, device=DEV) if c["fmt"] != "same" else None
    return s


def _fill(c, s, rnd):
    """What earlier writes have left: normal keys and values, keys with a wider spread."""
    for x, std in (("k", 1.5), ("v", 1.0)):
        pool = s[x + "_pool"]
        for l in range(pool.shape[0]):
            rows = rnd.normal(*pool.shape[1:]) * std
            if c["fmt"] == "same":
                pool[l] = rows
            else:
                q, e = _quantise(rows.to(_dtype(c)).float(), c["fmt"])
                pool[l], s[x + "_exp"][l] = q, e


def prepare(case, seed):
    c, rnd = case, _Inputs(seed)
    if c["kind"] == "rotary":
        x = rnd.normal(c["n"], c["H"] + c["spare"], c["d"], dtype=_dtype(c))[:, :c["H"]]      # heads of a packed row, the rest behind them
        freq, axis = _rotation(c["R"], c["axes"])
        s = dict(c=c, x=x, y=torch.empty((c["n"], c["H"], c["d"]), dtype=x.dtype, device=DEV), freq=freq, axis=axis,
                 pos=rnd.ints(0, 1 << 20 if c["far"] else 4096, c["axes"], c["n"]))
        if own:
            from paper_2607_14695_b200 import binding as rb
            s["rotary"] = rb.Rotary(freq, axis, adjacent=c["adjacent"])
        return s
    seqs = _sequences(c)
    total = sum(n for n, _ in seqs)
    L = c.get("L", 1)
    s = dict(c=c, most=max(1, max(n for n, _ in seqs)), longest=max(1, max(x for _, x in seqs)), **_pages(c, rnd, L))
    dt = _dtype(c)
    if c["kind"] == "write":
        rows = rnd.normal(max(1, total), 2 * c["Hkv"], c["d"], dtype=dt)
        s["k"], s["v"] = rows[:, :c["Hkv"]], rows[:, c["Hkv"]:]
        if c["rotary"]:
            s["freq"], s["axis"] = _rotation(c["d"], 3)
            s["pos"] = rnd.ints(0, 4096, 3, max(1, total))
        s["out"] = [torch.zeros((c["B"], 1, s["most"], c["Hkv"], c["d"]), dtype=dt, device=DEV) for _ in range(2)]
        s["start"] = s["length"] - (s["cu"][1:] - s["cu"][:-1])
    elif c["kind"] == "read":
        _fill(c, s, rnd)
        s["out"] = [torch.zeros((c["B"], L, s["longest"], c["Hkv"], c["d"]), dtype=dt, device=DEV) for _ in range(2)]
        s["start"] = None
    else:
        _fill(c, s, rnd)
        s["q"] = rnd.normal(max(1, total + c["pad"]), c["Hq"], c["d"], dtype=dt)
        s["out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2607_14695_b200 import binding as rb
        s["pages"] = rb.Pages(L, s["k_pool"].shape[1], c["page"], c.get("Hq", c["Hkv"]), c["Hkv"], c["d"], rb.DTYPE_F32 if c["dtype"] == "f32" else rb.DTYPE_BF16,
                              {"same": rb.PAGE_SAME, "e4m3": rb.PAGE_E4M3, "int8": rb.PAGE_INT8}[c["fmt"]], max_seqs=c["B"], max_rows=max(1, total + c.get("pad", 0)),
                              k_pool=s["k_pool"], v_pool=s["v_pool"], k_exp=s["k_exp"], v_exp=s["v_exp"])
        s["batch"] = rb.PageBatch(s["table"], s["cu"], s["length"])
        if c.get("rotary"):
            s["rotary"] = rb.Rotary(s["freq"], s["axis"])
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------

def _turn(x, pos, freq, axis, adjacent, inverse):
    """Rotated rows in 32 bits; the angles, which far positions make large, in 64."""
    R = 2 * freq.numel()
    angle = pos.double()[axis.long()].T * freq.double()                      # [n][R / 2]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if inverse:
        sin = -sin
    x = x.float()
    y = x.clone()
    if adjacent:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y[..., 0:R:2], y[..., 1:R:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y[..., :R // 2], y[..., R // 2:R] = a * cos - b * sin, a * sin + b * cos
    return y


def _quantise(x, fmt):
    """Rows of the last axis as 8-bit numbers and the byte of their power-of-two scale: the smallest under which the largest fits."""
    top, mantissa, exponent = LARGEST[fmt]
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x).clamp(-FAR, FAR)
    m, k = torch.frexp(x.abs().amax(-1))                                       # largest = m 2^k, m in [0.5, 1)
    e = torch.where(m == 0, torch.full_like(k, E_MIN), (k - 1 - exponent + (2 * m > mantissa)).clamp(min=E_MIN))
    q = torch.ldexp(x, -e[..., None])
    q = q.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(q).to(torch.int8)
    return q, torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)


def _values(q, e):
    """What a page's rows stand for, in 32 bits."""
    if e is None:
        return q.float()
    scale = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e.int() - 127)
    return q.float() * torch.where(e == 255, torch.full_like(scale, float("nan")), scale)[..., None]


def _places(s):
    """For every new token, which sequence it belongs to and its position there."""
    rows = torch.arange(int(s["k"].shape[0]) if "k" in s else int(s["q"].shape[0]), device=DEV)
    seq = torch.bucketize(rows, s["cu"].long(), right=True) - 1
    live = rows < s["cu"][-1]
    seq = torch.where(live, seq, torch.zeros_like(seq))
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    return live, seq, rows - s["cu"].long()[seq], (s["length"].long() - new)[seq] + rows - s["cu"].long()[seq]


def _put(s):
    c, P = s["c"], s["c"]["page"]
    live, seq, _, at = _places(s)
    seq, at = seq[live], at[live]
    page, slot = s["table"].long()[seq, at // P], at % P
    k = _turn(s["k"], s["pos"], s["freq"], s["axis"], False, False) if c["rotary"] else s["k"].float()
    for x, rows in (("k", k), ("v", s["v"].float())):
        rows = rows[live]
        if c["fmt"] == "same":
            s[x + "_pool"][0, page, :, slot] = rows.to(_dtype(c))
        else:
            q, e = _quantise(rows, c["fmt"])
            s[x + "_pool"].view(torch.uint8)[0, page, :, slot] = q.view(torch.uint8)
            s[x + "_exp"][0, page, :, slot] = e


def _take(s, x, start, count):
    """[B][L][count][Hkv][d] in 32 bits: `count` tokens of every sequence from `start` on, those past its end unspecified."""
    c, P, pool, exp = s["c"], s["c"]["page"], s[x + "_pool"], s[x + "_exp"]
    at = start[:, None] + torch.arange(count, device=DEV)
    page = s["table"].long().gather(1, (at // P).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    slot = at % P
    q = pool.view(torch.uint8) if c["fmt"] == "e4m3" else pool                  # (8-bit floats are moved as bytes)
    q = q.permute(0, 1, 3, 2, 4)[:, page, slot]                               # [L][B][count][Hkv][d]
    q = q.view(torch.float8_e4m3fn) if c["fmt"] == "e4m3" else q
    e = exp.permute(0, 1, 3, 2)[:, page, slot] if exp is not None else None
    return _values(q, e).transpose(0, 1)


def _get(s):
    start = torch.zeros_like(s["length"]) if s["start"] is None else s["start"]
    count = s["out"][0].shape[2]
    live = (torch.arange(count, device=DEV) < (s["length"] - start)[:, None])[:, None, :, None, None]
    for out, x in zip(s["out"], ("k", "v")):
        out.copy_(torch.where(live, _take(s, x, start.long(), count).to(out.dtype), out))
    return s["out"]


def _attend(s):
    c = s["c"]
    B, Hq, Hkv, d, most, longest = c["B"], c["Hq"], c["Hkv"], c["d"], s["most"], s["longest"]
    G = Hq // Hkv
    live, seq, i, _ = _places(s)
    q = torch.zeros((B, most, Hq, d), device=DEV)
    q[seq[live], i[live]] = s["q"][live].float()
    zero = torch.zeros_like(s["length"]).long()
    k, v = [_take(s, x, zero, longest)[:, 0].transpose(1, 2) for x in ("k", "v")]                 # [B][Hkv][keys][d]
    j = torch.arange(longest, device=DEV)
    v = torch.where((j < s["length"][:, None])[:, None, :, None], v, torch.zeros_like(v))
    q = q.view(B, most, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * most, d)
    logits = torch.matmul(q, k.transpose(2, 3)) * (d ** -0.5)
    new = s["cu"][1:] - s["cu"][:-1]
    p = (s["length"] - new)[:, None] + torch.arange(most, device=DEV)                            # position of every query
    seen = (j < s["length"][:, None])[:, None].expand(B, most, longest)
    if c["causal"]:
        seen = seen & (j <= p[..., None])
    if c["window"]:
        seen = seen & (j > p[..., None] - c["window"])
    logits = logits.view(B, Hkv, G, most, longest).masked_fill(~seen[:, None, None], float("-inf"))
    top = logits.amax(-1, keepdim=True)
    weights = torch.exp(logits - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.view(B, Hkv, G * most, longest), v).view(B, Hkv, G, most, d) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, most, Hq, d)
    s["out"][live] = out[seq[live], i[live]].to(s["out"].dtype)
    return s["out"]


def run(state):
    s, c = state, state["c"]
    if own:
        from paper_2607_14695_b200 import binding as rb
        if c["kind"] == "rotary":
            return rb.reflex_rotary_axes(s["x"], s["y"], s["pos"], s["rotary"], inverse=c["inverse"])
        if c["kind"] == "attention":
            return rb.reflex_pages_attention(s["pages"], 0, s["batch"], s["q"], s["out"], causal=c["causal"], window=c["window"])
        if c["kind"] == "write":
            rb.reflex_pages_write(s["pages"], 0, s["batch"], s["k"], s["v"], rotary=s.get("rotary"), pos=s.get("pos"))
        return rb.reflex_pages_read(s["pages"], 0, s["batch"], s["out"][0], s["out"][1], start=s["start"])
    if c["kind"] == "rotary":
        s["y"].copy_(_turn(s["x"], s["pos"], s["freq"], s["axis"], c["adjacent"], c["inverse"]))
        return s["y"]
    if c["kind"] == "attention":
        return _attend(s)
    if c["kind"] == "write":
        _put(s)
    return _get(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rotary":
        return {"bytes": 2 * c["n"] * c["H"] * c["d"] * es + 4 * c["axes"] * c["n"], "flops": 3 * c["n"] * c["H"] * c["R"]}
    seqs, L = _sequences(c), c.get("L", 1)
    row = c["d"] * es if c["fmt"] == "same" else c["d"] + 1                   # a row in the pages
    new, held = sum(n for n, _ in seqs), sum(x for _, x in seqs)
    if c["kind"] == "write":            # rows read, pages written and read, rows written
        return {"bytes": 2 * new * c["Hkv"] * (2 * c["d"] * es + 2 * row) + (12 * new if c["rotary"] else 0), "flops": 3 * new * c["Hkv"] * c["d"] if c["rotary"] else 0}
    if c["kind"] == "read":
        return {"bytes": 2 * L * held * c["Hkv"] * (row + c["d"] * es), "flops": 0}
    pairs = keys = 0                    # (query, key) pairs and keys that the masks leave
    for n, length in seqs:
        first = length
        for p in range(length - n, length):
            lo, hi = (max(0, p - c["window"] + 1) if c["window"] else 0), (p + 1 if c["causal"] else length)
            pairs += max(0, hi - lo)
            first = min(first, lo)
        keys += length - first if n else 0
    return {"bytes": 2 * new * c["Hq"] * c["d"] * es + 2 * keys * c["Hkv"] * row, "flops": 4 * pairs * c["Hq"] * c["d"]}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def _exact_rotation(x, pos, freq, axis, adjacent, sign):
    x = x.double()
    R = 2 * len(freq)
    angle = torch.stack([pos[int(a)].double() * f for a, f in zip(axis, freq.double())], 1)
    turn = torch.polar(torch.ones_like(angle), sign * angle)[:, None]
    lo, hi = (x[..., 0:R:2], x[..., 1:R:2]) if adjacent else (x[..., :R // 2], x[..., R // 2:R])
    z = torch.complex(lo.contiguous(), hi.contiguous()) * turn
    rotated = torch.stack([z.real, z.imag], -1).flatten(-2) if adjacent else torch.cat([z.real, z.imag], -1)
    return torch.cat([rotated, x[..., R:]], -1)


def _exact_8_bits(x, fmt):
    """Every element to the nearest number of its row's grid, ties to the even one."""
    top = LARGEST[fmt][0]
    largest = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(largest / top))
    e = torch.where(largest > top * torch.exp2(e), e + 1, torch.where(largest <= top * torch.exp2(e - 1), e - 1, e))
    e = torch.where(largest > 0, e, torch.zeros_like(e)).clamp(min=E_MIN)
    u = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3) if fmt == "e4m3" else 1.0
    return torch.round(u / step) * step * torch.exp2(e)


def _exact_held(s, x, b, length, l=0):
    """Rows [0, length) of one sequence and layer as the pages hold them: [length][Hkv][d]."""
    P = s["c"]["page"]
    pages = s["table"][b, :-(-length // P)].long()
    rows = s[x + "_pool"][l][pages].double()
    if s[x + "_exp"] is not None:
        rows = rows * torch.exp2(s[x + "_exp"][l][pages].double() - 127)[..., None]
    return rows.transpose(1, 2).reshape(-1, *rows.shape[1:2], rows.shape[-1])[:length]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "rotary":
        return _exact_rotation(s["x"], s["pos"], s["freq"], s["axis"].tolist(), c["adjacent"], -1.0 if c["inverse"] else 1.0)
    seqs, cu = _sequences(c), s["cu"].tolist()
    if c["kind"] == "write":
        k = _exact_rotation(s["k"], s["pos"], s["freq"], s["axis"].tolist(), False, 1.0) if c["rotary"] else s["k"].double()
        out = [torch.zeros(o.shape, dtype=torch.float64, device=DEV) for o in s["out"]]
        for o, rows in zip(out, (k, s["v"].double())):
            if c["fmt"] != "same":
                rows = _exact_8_bits(rows, c["fmt"])
            for b, (n, _) in enumerate(seqs):
                o[b, 0, :n] = rows[cu[b]:cu[b + 1]]
        return out
    if c["kind"] == "read":
        out = [torch.zeros(o.shape, dtype=torch.float64, device=DEV) for o in s["out"]]
        for o, x in zip(out, ("k", "v")):
            for b, (_, length) in enumerate(seqs):
                for l in range(c["L"]):
                    if length:
                        o[b, l, :length] = _exact_held(s, x, b, length, l)
        return out
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    G = c["Hq"] // c["Hkv"]
    for b, (n, length) in enumerate(seqs):
        if not n:
            continue
        k, v = _exact_held(s, "k", b, length), _exact_held(s, "v", b, length)
        p, j = torch.arange(length - n, length, device=DEV)[:, None], torch.arange(length, device=DEV)[None]
        hidden = torch.zeros((n, length), dtype=torch.bool, device=DEV)
        if c["causal"]:
            hidden |= j > p
        if c["window"]:
            hidden |= j <= p - c["window"]
        for h in range(c["Hq"]):
            logits = (s["q"][cu[b]:cu[b + 1], h].double() @ k[:, h // G].T / c["d"] ** 0.5).masked_fill_(hidden, float("-inf"))
            weights = torch.softmax(logits, -1).nan_to_num_(0.0)
            out[cu[b]:cu[b + 1], h] = weights @ v[:, h // G]
    return out
