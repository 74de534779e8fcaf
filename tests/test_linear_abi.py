"""Refusals of the quantised linear layers, before anything is launched (no GPU: pointers are never dereferenced on the host)."""
import ctypes

import pytest
import torch

from paper_2509_09679_amd import binding as B

FAKE = 0x7F0000001000


def _desc(**kw):
    d = B.bq_linear()
    d.rows, d.inputs, d.outputs, d.experts, d.xbits, d.wbits = 5, 64, 48, 1, 8, 8
    d.dtype, d.scale_dtype, d.ld_x, d.ld_w, d.ld_y = B.BQ_F16, B.BQ_F32, 64, 64, 64
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _fwd(d, x=FAKE, xs=FAKE, w=FAKE, ws=FAKE, bias=None, y=FAKE):
    return B.lib().bq_linear_fwd(x, xs, w, ws, bias, y, ctypes.byref(d) if d is not None else None, None)


def _gfwd(d, offsets=FAKE, y=FAKE):
    return B.lib().bq_linear_grouped_fwd(FAKE, FAKE, FAKE, FAKE, None, offsets, y, ctypes.byref(d), None)


def _bwd(d, dy=FAKE, w=FAKE, ws=FAKE, dx=FAKE, work=FAKE, nbytes=1 << 40):
    return B.lib().bq_linear_bwd(dy, w, ws, dx, work, nbytes, ctypes.byref(d) if d is not None else None, None)


def _gbwd(d, offsets=FAKE, nbytes=1 << 40):
    return B.lib().bq_linear_grouped_bwd(FAKE, FAKE, FAKE, offsets, FAKE, FAKE, nbytes, ctypes.byref(d), None)


def test_descriptor_size_matches_header():
    assert ctypes.sizeof(B.bq_linear) == 64


def test_kinds_match_the_ctypes_prototypes():
    kind = {ctypes.c_void_p: "ps", ctypes.c_int32: "i", ctypes.c_size_t: "u", ctypes.c_int64: "u", ctypes.POINTER(B.bq_linear): "l"}
    for name, kinds in B._LINEAR_KINDS.items():
        types = getattr(B.lib(), name).argtypes
        assert len(types) == len(kinds) and all(k in kind[t] for k, t in zip(kinds, types)), name


@pytest.mark.parametrize("call", [_fwd, _gfwd, _bwd, _gbwd])
def test_bad_descriptors(call):
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(inputs=0), dict(inputs=131072, ld_x=1 << 20, ld_w=1 << 20), dict(outputs=0), dict(experts=0),
               dict(experts=4097), dict(ld_x=63), dict(ld_w=63), dict(ld_y=47), dict(ld_x=1 << 43), dict(ld_y=1 << 43), dict(ld_w=1 << 42),
               dict(rows=1 << 26, outputs=1 << 16, inputs=1 << 16, ld_x=1 << 16, ld_w=1 << 16, ld_y=1 << 16), dict(rows=(1 << 31) - 1, outputs=70000, inputs=70000, ld_x=70000, ld_w=70000, ld_y=70000)):
        assert call(_desc(**kw)) == 2, kw
    assert call(_desc(dtype=5)) == 3 and call(_desc(scale_dtype=B.BQ_BF16)) == 3
    assert call(_desc(wbits=3)) == 6 and call(_desc(wbits=16)) == 6
    assert call(_desc(rows=0)) == 0
    assert B.lib().bq_last_error() == b""


def test_forward_refusals():
    assert _fwd(None) == 1 and _fwd(_desc(xbits=2)) == 6
    assert _fwd(_desc(experts=2)) == 2 and _gfwd(_desc(experts=2), offsets=None) == 1
    for name in ("x", "xs", "w", "ws", "y"):
        assert _fwd(_desc(), **{name: None}) == 1, name
    assert _fwd(_desc(), xs=FAKE + 2) == _fwd(_desc(), ws=FAKE + 2) == _fwd(_desc(), y=FAKE + 1) == _fwd(_desc(), bias=FAKE + 1) == 4
    assert _gfwd(_desc(), offsets=FAKE + 2) == 4
    assert _fwd(_desc(outputs=(1 << 24) + 1, ld_y=1 << 25)) == 2
    assert _fwd(_desc(rows=0), x=None, xs=None, w=None, ws=None, y=None) == 0


def test_backward_refusals():
    assert _bwd(None) == 1 and _bwd(_desc(experts=2)) == 2 and _gbwd(_desc(), offsets=None) == 1
    for name in ("dy", "w", "ws", "dx", "work"):
        assert _bwd(_desc(), **{name: None}) == 1, name
    assert _bwd(_desc(), work=FAKE + 64) == _bwd(_desc(), dy=FAKE + 1) == _bwd(_desc(), dx=FAKE + 1) == _bwd(_desc(), ws=FAKE + 2) == 4
    assert _bwd(_desc(outputs=131072, ld_y=1 << 18)) == 2
    need = B.bq_linear_bwd_workspace_bytes(_desc())
    assert need > 0 and need % 256 == 0 and _bwd(_desc(), nbytes=need - 1) == 5
    assert b"needed" in B.lib().bq_last_error()
    assert B.bq_linear_bwd_workspace_bytes(_desc(wbits=5)) == 0 and B.bq_linear_bwd_workspace_bytes(_desc(rows=0)) > 0


def test_workspace_holds_what_it_is_for():
    for rows, n, k, e, dtype, planes in ((7, 100, 33, 1, B.BQ_F16, 2), (4096, 4096, 4096, 1, B.BQ_F32, 3), (100, 129, 64, 60, B.BQ_BF16, 2)):
        np = (n + 127) // 128 * 128
        d = _desc(rows=rows, outputs=n, inputs=k, experts=e, dtype=dtype, ld_x=k, ld_w=k, ld_y=n)
        assert B.bq_linear_bwd_workspace_bytes(d) >= 4 * rows + planes * rows * np + e * k * np


def test_rows_quant8_refusals():
    def call(x=FAKE, rows=3, cols=40, ld_x=40, dtype=B.BQ_F16, codes=FAKE, ld_codes=40, scales=FAKE, scale=B.BQ_F32):
        return B.lib().bq_rows_quant8(x, rows, cols, ld_x, dtype, codes, ld_codes, scales, scale, None)

    assert call(rows=0) == 0 and call(rows=0, x=None, codes=None, scales=None) == 0
    assert call(dtype=3) == call(scale=B.BQ_BF16) == 3
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 24) + 1, ld_x=1 << 25, ld_codes=1 << 25), dict(ld_x=39), dict(ld_codes=39),
               dict(ld_x=1 << 43)):
        assert call(**kw) == 2, kw
    assert call(x=None) == call(codes=None) == call(scales=None) == 1
    assert call(x=FAKE + 1) == call(scales=FAKE + 2) == 4


def test_descriptors_from_tensors():
    x, w, ws, y = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5), torch.zeros(7, 5, dtype=torch.bfloat16)
    d = B.make_linear(x, w, ws, y)
    assert (d.rows, d.inputs, d.outputs, d.experts, d.ld_x, d.ld_w, d.ld_y, d.dtype, d.scale_dtype) == (7, 32, 5, 1, 32, 32, 5, B.BQ_BF16, B.BQ_F32)
    d = B.make_linear(x[:, :16], torch.zeros(3, 5, 8, dtype=torch.int8), torch.zeros(3, 5), y, wbits=4)
    assert (d.inputs, d.experts, d.outputs, d.ld_x, d.ld_w) == (16, 3, 5, 32, 8)
    d = B.make_linear(x, torch.zeros(5, 16, dtype=torch.uint8), ws, y, xbits=8, wbits=4, inputs=32)
    assert d.ld_w == 16
    b = B.make_linear_bwd(y, torch.zeros(5, 12, dtype=torch.int8), ws, torch.zeros(7, 48, dtype=torch.bfloat16), wbits=2)
    assert (b.rows, b.inputs, b.outputs, b.ld_x, b.ld_y, b.wbits) == (7, 48, 5, 48, 5, 2)
    for bad in (lambda: B.make_linear(x, w[:, :30], ws, y), lambda: B.make_linear(x, w, ws[:4], y), lambda: B.make_linear(x, w, ws, y[:6]),
                lambda: B.make_linear(x, w, ws, y[:, :4]), lambda: B.make_linear(x.t().contiguous().t(), w, ws, y),
                lambda: B.make_linear(x[:1].expand(7, 32), w, ws, y), lambda: B.make_linear(x, torch.zeros(3, 10, 32, dtype=torch.int8)[:, :5], torch.zeros(3, 5), y),
                lambda: B.make_linear_bwd(y, w, ws, torch.zeros(7, 32)), lambda: B.make_linear_bwd(y, w, ws, torch.zeros(6, 32, dtype=torch.bfloat16)),
                lambda: B.make_linear_bwd(y[:, :4], w, ws, torch.zeros(7, 32, dtype=torch.bfloat16))):
        with pytest.raises(B.BqError):
            bad()


def test_a_changed_descriptor_is_looked_at_again(monkeypatch):
    monkeypatch.setattr(B, "_here", lambda: -1)
    x, w, ws, y, xs = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5), torch.zeros(7, 5), torch.zeros(7)
    d = B.make_linear(x, w, ws, y)
    B._check_fwd("t", d, x, xs, w, ws, None, y)
    d.rows = 8
    with pytest.raises(B.BqError):
        B._check_fwd("t", d, x, xs, w, ws, None, y)
    d.rows, d.dtype = 7, B.BQ_F16
    with pytest.raises(B.BqError):
        B._check_fwd("t", d, x, xs, w, ws, None, y)


def test_tensors_the_library_cannot_see(monkeypatch):
    # element types, extents and contiguity; CPU tensors taken for the current device's, nothing reaches the library
    monkeypatch.setattr(B, "_here", lambda: -1)
    x, w, ws, y = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5), torch.zeros(7, 5)
    xs, off = torch.zeros(7), torch.zeros(2, dtype=torch.int32)
    d = B.make_linear(x, w, ws, y)
    g = B.make_linear_bwd(y, w, ws, torch.zeros(7, 32))
    work = torch.zeros(10, dtype=torch.uint8)

    def fwd(x=x, xs=xs, w=w, ws=ws, b=None, y=y):
        B.bq_linear_fwd(x, xs, w, ws, b, y, d)

    for call, status in ((lambda: fwd(x=x.float()), 3), (lambda: fwd(xs=xs.half()), 3), (lambda: fwd(xs=xs[:6]), 2), (lambda: fwd(w=w[:4]), 2),
                         (lambda: fwd(ws=torch.zeros(10)[::2]), 2), (lambda: fwd(y=y.half()), 3), (lambda: fwd(y=y[:6]), 2),
                         (lambda: fwd(b=torch.zeros(4)), 2), (lambda: fwd(b=torch.zeros(5).half()), 3),
                         (lambda: fwd(x=torch.zeros(7, 40, dtype=torch.int8)[:, :32]), 2), (lambda: fwd(w=torch.zeros(5, 40, dtype=torch.int8)[:, :32]), 2),
                         (lambda: fwd(y=torch.zeros(7, 8)[:, :5]), 2), (lambda: B.bq_linear_bwd(torch.zeros(7, 6)[:, :5], w, ws, torch.zeros(7, 32), work, g), 2),
                         (lambda: B.bq_linear_grouped_fwd(x, xs, w, ws, None, off.long(), y, d), 3),
                         (lambda: B.bq_linear_grouped_fwd(x, xs, w, ws, None, off[:1], y, d), 2),
                         (lambda: B.bq_linear_bwd(y.half(), w, ws, torch.zeros(7, 32), work, g), 3),
                         (lambda: B.bq_linear_bwd(y, w, ws, torch.zeros(7, 31), work, g), 2),
                         (lambda: B.bq_linear_bwd(y, w, ws, torch.zeros(7, 32), work.int(), g), 3),
                         (lambda: B.bq_rows_quant8(torch.zeros(3, 8, dtype=torch.float64), x[:3, :8], torch.zeros(3)), 3),
                         (lambda: B.bq_rows_quant8(torch.zeros(3, 8), x[:3, :7], torch.zeros(3)), 2),
                         (lambda: B.bq_rows_quant8(torch.zeros(8, 3).t(), x[:3, :8], torch.zeros(3)), 2),
                         (lambda: B.bq_rows_quant8(torch.zeros(3, 8), x[:3, :8], torch.zeros(2)), 2)):
        with pytest.raises(B.BqError) as e:
            call()
        assert e.value.status == status, str(e.value)
    monkeypatch.setattr(B, "_here", lambda: 0)  # tensors of another device
    with pytest.raises(B.BqError, match="current device"):
        fwd()


def test_tensors_laid_out_otherwise_than_the_descriptor(monkeypatch):
    # all of these have the elements that the call needs, and would be read at the wrong places or behind their ends
    monkeypatch.setattr(B, "_here", lambda: -1)
    codes = lambda *s: torch.zeros(*s, dtype=torch.int8)  # noqa: E731
    x, w, ws, y, xs, off = codes(6, 32), codes(3, 4, 32), torch.zeros(3, 4), torch.zeros(6, 4), torch.zeros(6), torch.zeros(4, dtype=torch.int32)
    dx, work = torch.zeros(6, 32), torch.zeros(10, dtype=torch.uint8)
    wide = codes(6, 64)
    d, g = B.make_linear(x, w, ws, y), B.make_linear_bwd(y, w, ws, dx)
    p = B.make_linear(wide[:, :32], w, ws, y)  # rows of 32 that are 64 apart

    def fwd(x=x, w=w, b=None, y=y, d=d):
        B.bq_linear_grouped_fwd(x, xs, w, ws, b, off, y, d)

    def bwd(dy=y, w=w, dx=dx):
        B.bq_linear_grouped_bwd(dy, w, ws, off, dx, work, g)

    for call in (lambda: fwd(x=wide[:, ::2], d=p), lambda: fwd(x=wide[:3], d=p), lambda: fwd(x=x.reshape(-1), d=d), lambda: fwd(x=x.reshape(3, 64)),
                 lambda: fwd(w=codes(6, 4, 32)[::2]), lambda: fwd(w=codes(3, 32, 4).transpose(1, 2)), lambda: fwd(w=w.reshape(4, 3, 32)),
                 lambda: fwd(y=torch.zeros(4, 6).t()), lambda: fwd(b=torch.zeros(3, 8)[:, ::2]), lambda: bwd(dy=torch.zeros(6, 8)[:, ::2]),
                 lambda: bwd(w=codes(6, 4, 32)[1::2]), lambda: bwd(dx=torch.zeros(32, 6).t()), lambda: bwd(dx=dx.reshape(12, 16))):
        with pytest.raises(B.BqError) as e:
            call()
        assert e.value.status == 2, str(e.value)
    # strides of dimensions of one element do not matter, and the experts' weights may be one matrix
    one = B.make_linear(x[:1], w[:1, :1], ws[:1, :1], y[:1, :1])
    B._check_fwd("t", one, x[:1], xs, w[2:, 3:], ws[:1, :1], None, y[3:4, 2:3])
    B._check_fwd("t", p, wide[:, 32:], xs, w.reshape(12, 32), ws, torch.zeros(12), y)
    B._check_bwd("t", g, y, w.reshape(12, 32), ws, dx, work)
    B._check_bwd("t", g, y, w, ws, dx, work)
