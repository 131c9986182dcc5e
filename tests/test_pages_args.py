"""What the calls of the paged prefix refuse before anything is launched, and the sizes they ask for (no GPU)."""
import ctypes

import pytest
import torch

from paper_2607_14695_b200 import binding as rb
from paper_2607_14695_b200 import build as rbuild

FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10004)        # never dereferenced


@pytest.fixture(scope="module")
def lib():
    rbuild.build()
    return rb.load()


def _desc(**kw):
    return rb.PagesDesc(**(dict(L=2, n_pages=10, page=32, Hq=8, Hkv=2, d=64, dtype=rb.DTYPE_BF16, format=rb.PAGE_INT8, max_seqs=4, max_rows=64) | kw))


def test_sizes(lib):
    size = lambda fn, **kw: getattr(lib, f"reflex_pages_{fn}_bytes")(ctypes.byref(_desc(**kw)))      # noqa: E731
    rows = 2 * 10 * 32 * 2
    assert size("pool") == rows * 64 and size("exp") == rows
    assert size("pool", format=rb.PAGE_SAME) == rows * 128 and size("exp", format=rb.PAGE_SAME) == 0
    assert size("pool", format=rb.PAGE_SAME, dtype=rb.DTYPE_F32) == rows * 256
    assert size("workspace") >= 256 and size("workspace", format=rb.PAGE_SAME) >= 256
    for bad in (dict(L=0), dict(n_pages=0), dict(page=48), dict(page=256), dict(Hq=3), dict(Hkv=0), dict(d=96), dict(dtype=2), dict(format=3), dict(format=-1),
                dict(max_seqs=0), dict(max_seqs=1025), dict(max_rows=0), dict(n_pages=1 << 30), dict(Hq=65536 * 2)):
        assert size("pool", **bad) == size("exp", **bad) == size("workspace", **bad) == 0, bad
    assert size("pool", n_pages=1 << 24, L=4) == 4 * (1 << 24) * 64 * 64                   # 64-bit sizes


def test_create(lib):
    out = ctypes.c_void_p()
    make = lambda d, k=FAKE, v=FAKE, ke=FAKE, ve=FAKE, ws=FAKE: lib.reflex_pages_create(ctypes.byref(d), k, v, ke, ve, ws, None, ctypes.byref(out))      # noqa: E731
    assert make(_desc(page=20)) == rb.ERR_SHAPE
    assert make(_desc(), k=None) == make(_desc(), v=None) == make(_desc(), ws=None) == rb.ERR_INVALID_ARG
    assert make(_desc(), ke=None) == make(_desc(), ve=None) == rb.ERR_INVALID_ARG
    assert make(_desc(format=rb.PAGE_SAME)) == rb.ERR_INVALID_ARG                        # exponents of pages that have none
    assert make(_desc(), k=ODD) == make(_desc(), v=ODD) == make(_desc(), ke=ODD) == make(_desc(), ve=ODD) == make(_desc(), ws=ctypes.c_void_p(0x10010)) == rb.ERR_ALIGN
    assert lib.reflex_pages_create(ctypes.byref(_desc()), FAKE, FAKE, FAKE, FAKE, FAKE, None, None) == rb.ERR_INVALID_ARG
    assert not out.value


def test_no_handle(lib):
    q = rb.PageBatchDesc(0x10000, 0x10000, 0x10000, 1, 1)
    assert lib.reflex_pages_write(None, 0, ctypes.byref(q), FAKE, 128, FAKE, 128, 1, None, None, None) == rb.ERR_INVALID_ARG
    assert lib.reflex_pages_read(None, 0, 1, ctypes.byref(q), None, FAKE, FAKE, 1, None) == rb.ERR_INVALID_ARG
    assert lib.reflex_pages_attention(None, 0, ctypes.byref(q), FAKE, FAKE, 1, 0.0, 0, 0, None) == rb.ERR_INVALID_ARG
    assert lib.reflex_pages_check_status(None, None) == lib.reflex_pages_destroy(None) == rb.ERR_INVALID_ARG


def test_rotary(lib):
    def call(x=FAKE, ldx=512, y=ctypes.c_void_p(0x20000), ldy=512, pos=FAKE, rot=rb.RotaryDesc(0x10000, 0x10000, 64, 3, 0), n=4, H=8, d=64, inverse=0, dtype=rb.DTYPE_BF16):
        return lib.reflex_rotary_axes(x, ldx, y, ldy, pos, ctypes.byref(rot) if rot else None, n, H, d, inverse, dtype, None)
    r = lambda **kw: rb.RotaryDesc(**(dict(freq=0x10000, axis=0x10000, R=64, axes=3, adjacent=0) | kw))      # noqa: E731
    assert call(n=0) == rb.OK
    for kw in (dict(x=None), dict(y=None), dict(pos=None), dict(rot=None), dict(rot=r(freq=None)), dict(rot=r(axis=None)), dict(rot=r(adjacent=2)), dict(inverse=2), dict(dtype=7),
               dict(y=FAKE, ldy=520)):
        assert call(**kw) == rb.ERR_INVALID_ARG, kw
    for kw in (dict(n=-1), dict(H=0), dict(d=40), dict(d=1040), dict(ldx=504), dict(ldy=511), dict(ldx=516), dict(rot=r(R=8)), dict(rot=r(R=72)), dict(rot=r(R=80)), dict(rot=r(axes=0)),
               dict(rot=r(axes=9))):
        assert call(**kw) == rb.ERR_SHAPE, kw
    for kw in (dict(x=ODD), dict(y=ODD), dict(pos=ctypes.c_void_p(0x10002)), dict(rot=r(freq=0x10002))):
        assert call(**kw) == rb.ERR_ALIGN, kw


def test_tensors_on_the_host_are_refused():
    x, pos = torch.zeros(2, 1, 32), torch.zeros(1, 2, dtype=torch.int32)
    rot = rb.Rotary(torch.ones(16), torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        rb.reflex_rotary_axes(x, x, pos, rot, stream=0)
