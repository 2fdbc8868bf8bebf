"""Outputs of the norm at an input's address: what would lose a row or read it after it was written is refused
on the host, before any launch (no GPU needed)."""
import ctypes as C

import pytest

import paper_2607_20214_amd as E

INVALID = -1
X, R, W, S, Y, SC, DY, DW, WS = (C.c_void_p(1 << 20 | i << 16) for i in range(9))     # never dereferenced


def _desc(**kw):
    f = dict(rows=4, cols=64, dtype=E.BF16, y_dtype=E.BF16, eps=1e-6, ldx=64, ldr=64, lds=64, ldy=64)
    f.update(kw)
    return E._NormDesc(*f.values())


@pytest.mark.parametrize("kw,sum_,y", [
    (dict(), S, S),                                   # the sum would be lost
    (dict(), X, X),
    (dict(lds=72), X, Y), (dict(lds=72), R, Y),       # another row's values
    (dict(ldy=72), S, X), (dict(ldy=128), S, R),
    (dict(y_dtype=E.I8), S, X), (dict(y_dtype=E.I8), S, R), (dict(y_dtype=E.I8), S, S),
])
def test_forward(kw, sum_, y):
    d = _desc(**kw)
    assert E.load().elsaa_rms_norm_fwd(C.byref(d), X, R, W, sum_, y, SC, None) == INVALID
    assert E.load().elsaa_last_error().decode()


@pytest.mark.parametrize("kw,dx", [(dict(lds=72), X), (dict(lds=72), DY), (dict(lds=72), R)])
def test_backward(kw, dx):
    d = _desc(**kw)
    assert E.load().elsaa_rms_norm_bwd(C.byref(d), X, W, DY, R, dx, DW, WS, 1 << 30, None) == INVALID
    assert "stride" in E.load().elsaa_last_error().decode()
