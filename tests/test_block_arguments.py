"""Refusals of the layer norm, gated block and orthogonalising calls: found on the host, before anything is launched (no GPU needed)."""
import numpy as np
import pytest

from tests.helpers import mfet

A = 1 << 20  # an address that is never followed


def status(call, *args):
    m = mfet()
    with pytest.raises(m.MfetError) as e:
        call(*args)
    return e.value.status


def test_layer_norm_refusals():
    m = mfet()

    def args(**kw):
        v = dict(x=A, xt=m.F32, x_ld=64, rows=5, cols=64, w=A, b=A, eps=1e-5, y=A, yt=m.BF16, y_ld=64)
        v.update(kw)
        return list(v.values())

    def st(**kw):
        return status(m.mfet_layer_norm, *args(**kw))
    for kw in (dict(x=None), dict(y=None), dict(xt=3), dict(yt=m.MXFP4), dict(x_ld=63), dict(y_ld=63), dict(x_ld=1 << 31), dict(rows=-1),
               dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 30, x_ld=1 << 30, y_ld=1 << 30), dict(eps=-1.0), dict(eps=float("nan")),
               dict(xt=-1), dict(yt=1 << 32)):
        assert st(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(x=A + 2), dict(y=A + 1), dict(w=A + 2), dict(b=A + 1), dict(x=A + 1, xt=m.F16)):
        assert st(**kw) == m.ERR_ALIGNMENT, kw
    m.mfet_layer_norm(*args(rows=0))  # nothing to do: no launch, no GPU
    m.mfet_layer_norm(*args(rows=0, x=None, y=None))


def test_layer_norm_backward_refusals():
    m = mfet()

    def st(**kw):
        v = dict(x=A, xt=m.F32, x_ld=64, rows=5, cols=64, w=A, eps=1e-5, dy=A, dyt=m.BF16, dy_ld=64, dx=A, dx_ld=64, dw=A, db=A, ws=A, n=1 << 20)
        v.update(kw)
        return status(m.mfet_layer_norm_backward, *v.values())
    for kw in (dict(x=None), dict(dy=None), dict(dx=None), dict(xt=4), dict(dyt=3), dict(x_ld=63), dict(dy_ld=1), dict(dx_ld=63),
               dict(dx_ld=1 << 31), dict(rows=-1), dict(cols=0), dict(eps=float("nan")), dict(n=-1)):
        assert st(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(x=A + 2), dict(dy=A + 1), dict(dx=A + 2), dict(w=A + 2), dict(dw=A + 1), dict(db=A + 2), dict(ws=A + 2)):
        assert st(**kw) == m.ERR_ALIGNMENT, kw
    need = m.mfet_layer_norm_backward_bytes(5, 64)
    assert need > 0
    for kw in (dict(ws=None), dict(n=need - 1), dict(n=0), dict(ws=None, db=None)):
        assert st(**kw) == m.ERR_WORKSPACE, kw
    assert m.mfet_layer_norm_backward_bytes(-1, 64) == 0 and m.mfet_layer_norm_backward_bytes(5, 0) == 0
    assert m.mfet_layer_norm_backward_bytes(0, 64) == 0


def test_gated_refusals():
    m = mfet()

    def args(**kw):
        v = dict(x=A, t=m.BF16, x_ld=64, m=5, wg=A, wg_ld=64, wu=A, wu_ld=64, n=32, k=64, act=m.ACT_SILU, h=A, h_ld=32, ws=None, bytes=0, status=A)
        v.update(kw)
        return list(v.values())

    def st(**kw):
        return status(m.mfet_gated_linear, *args(**kw))
    for kw in (dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(t=m.F32), dict(t=m.INT4), dict(x_ld=63), dict(wg_ld=63),
               dict(wu_ld=63), dict(h_ld=31), dict(m=-1), dict(n=-1), dict(k=0), dict(k=1 << 30, x_ld=1 << 30, wg_ld=1 << 30, wu_ld=1 << 30),
               dict(m=1 << 31), dict(act=5), dict(act=-1), dict(bytes=-1), dict(m=(1 << 31) - 1, n=1 << 20, h_ld=1 << 20)):
        assert st(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(x=A + 1), dict(wg=A + 1), dict(wu=A + 1), dict(h=A + 1), dict(status=A + 2), dict(x=A + 2, ws=A + 8, bytes=1 << 20)):
        assert st(**kw) == m.ERR_ALIGNMENT, kw
    # rows that start on any address are copied, and that takes room
    for kw in (dict(x=A + 2), dict(x_ld=65), dict(wg_ld=65), dict(wu=A + 8), dict(x=A + 2, ws=A, bytes=5 * 128 - 1)):
        assert st(**kw) == m.ERR_WORKSPACE, kw
    m.mfet_gated_linear(*args(m=0))
    m.mfet_gated_linear(*args(n=0, h_ld=0))
    assert m.mfet_gated_linear_bytes(5, 32, 64) >= 5 * 128 + 2 * 32 * 128
    assert m.mfet_gated_linear_bytes(5, 32, 0) == 0 and m.mfet_gated_linear_bytes(-1, 32, 4) == 0


def test_gated_backward_refusals():
    m = mfet()

    def st(**kw):
        v = dict(x=A, t=m.BF16, x_ld=64, m=5, wg=A, wg_ld=64, wu=A, wu_ld=64, n=32, k=64, act=m.ACT_SILU, dh=A, dh_ld=32, dx=A, dx_ld=64,
                 dwg=A, dwg_ld=64, dwu=A, dwu_ld=64, ws=A, bytes=1 << 20, status=None)
        v.update(kw)
        return status(m.mfet_gated_linear_backward, *v.values())
    for kw in (dict(x=None), dict(wg=None), dict(wu=None), dict(dh=None), dict(t=m.F32), dict(x_ld=63), dict(wg_ld=1), dict(wu_ld=1), dict(dh_ld=31),
               dict(dx_ld=63), dict(dwg_ld=63), dict(dwu_ld=63), dict(m=-1), dict(k=0), dict(act=9), dict(dwg=None), dict(dwu=None)):
        assert st(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(x=A + 1), dict(wg=A + 1), dict(wu=A + 1), dict(dh=A + 1), dict(dx=A + 1), dict(dwg=A + 1), dict(dwu=A + 1), dict(ws=A + 8),
               dict(status=A + 1)):
        assert st(**kw) == m.ERR_ALIGNMENT, kw
    assert st(ws=None) == m.ERR_WORKSPACE and st(bytes=2 * 5 * 32 * 2 - 1) == m.ERR_WORKSPACE
    assert m.mfet_gated_linear_backward_bytes(5, 32, 64) > m.mfet_gated_linear_bytes(5, 32, 64)
    assert m.mfet_gated_linear_backward_bytes(5, -1, 64) == 0


def test_orthogonalize_refusals():
    m = mfet()

    def args(**kw):
        v = dict(g=A, t=m.F32, ld=64, rows=5, cols=64, c=None, steps=5, scale=1.0, out=A, ot=m.BF16, out_ld=64, ws=A, bytes=1 << 24, status=None)
        v.update(kw)
        return list(v.values())

    def st(**kw):
        return status(m.mfet_orthogonalize, *args(**kw))
    nan = float("nan")
    for kw in (dict(g=None), dict(out=None), dict(t=3), dict(ot=4), dict(ld=63), dict(out_ld=63), dict(rows=-1), dict(cols=-1, ld=0, out_ld=0),
               dict(steps=0), dict(steps=65), dict(steps=-1), dict(scale=nan), dict(scale=float("inf")), dict(c=[1.0, 2.0], steps=1),
               dict(c=[1.0, nan, 0.0], steps=1), dict(c=[1e6, 1e6, 1e6], steps=1), dict(c=[100.0, 0.0, 0.0] * 4, steps=4),
               dict(rows=(1 << 31) - 1, cols=(1 << 31) - 1, ld=(1 << 31) - 1, out_ld=(1 << 31) - 1), dict(bytes=-1)):
        assert st(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(g=A + 2), dict(out=A + 1), dict(ws=A + 8), dict(status=A + 2), dict(g=A + 1, t=m.BF16)):
        assert st(**kw) == m.ERR_ALIGNMENT, kw
    need = m.mfet_orthogonalize_bytes(5, 64)
    assert st(ws=None) == m.ERR_WORKSPACE and st(bytes=need - 1) == m.ERR_WORKSPACE
    m.mfet_orthogonalize(*args(rows=0))
    m.mfet_orthogonalize(*args(cols=0, c=np.array([[3.0, -4.0, 2.0]], np.float64), steps=1))
    assert m.mfet_orthogonalize_bytes(-1, 5) == 0


def test_argument_counts():
    m = mfet()
    for call in (m.mfet_layer_norm, m.mfet_layer_norm_backward, m.mfet_gated_linear, m.mfet_gated_linear_backward, m.mfet_orthogonalize):
        with pytest.raises(TypeError):
            call(A)
        with pytest.raises(TypeError):
            call(*[0] * 30)
