"""Refusals of the clipping, row and matrix calls: found on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from tests.helpers import mfet


def status(call, *args):
    m = mfet()
    with pytest.raises(m.MfetError) as e:
        call(*args)
    return e.value.status


def test_rows_refusals():
    m = mfet()
    A = 1 << 20  # an address that is never followed

    def desc(**kw):
        v = dict(data=A, rows=100, dim=64, dtype=m.MXFP4, loc=m.LOC_DEVICE, flags=0, seed=0, stride=0)
        v.update(kw)
        return m.TableDesc(v["data"], v["rows"], v["dim"], v["dtype"], v["loc"], v["flags"], v["seed"], v["stride"])

    for call in (m.mfet_rows_write, m.mfet_rows_read):
        def st(d, n=5, mem=A, dtype=m.F32, ld=64):
            return status(call, d, A, n, None, mem, dtype, ld)
        assert st(desc(data=None)) == m.ERR_INVALID_ARG
        assert st(desc(rows=0)) == m.ERR_INVALID_ARG
        assert st(desc(rows=1 << 63)) == m.ERR_INVALID_ARG
        assert st(desc(dim=0)) == m.ERR_INVALID_ARG
        assert st(desc(flags=1)) == m.ERR_INVALID_ARG
        assert st(desc(dtype=5)) == m.ERR_INVALID_ARG
        assert st(desc(loc=m.LOC_HOST)) == m.ERR_INVALID_ARG
        assert st(desc(), n=-1) == m.ERR_INVALID_ARG
        assert st(desc(), mem=None) == m.ERR_INVALID_ARG
        assert st(desc(), dtype=m.INT4) == m.ERR_INVALID_ARG
        assert st(desc(), ld=63) == m.ERR_INVALID_ARG
        assert st(desc(dim=60, dtype=m.MXFP4)) == m.ERR_UNSUPPORTED_DIM
        assert st(desc(dim=60, dtype=m.INT4)) == m.ERR_UNSUPPORTED_DIM
        assert st(desc(dim=60, dtype=m.F16)) == m.ERR_UNSUPPORTED_DIM
        assert st(desc(stride=40)) == m.ERR_INVALID_ARG
        assert st(desc(stride=56)) == m.ERR_ALIGNMENT
        assert st(desc(data=A + 8)) == m.ERR_ALIGNMENT
        assert st(desc(), mem=A + 2) == m.ERR_ALIGNMENT
        assert st(desc(), mem=A + 1, dtype=m.BF16) == m.ERR_ALIGNMENT
        call(desc(), A, 0, None, None, m.F32, 64)  # nothing to do: no launch, no GPU
    assert m.row_bytes(64, m.MXFP4) == 48 and m.row_bytes(32, m.MXFP4) == 32 and m.row_bytes(128, m.MXFP4) == 80
    assert m.row_bytes(40, m.MXFP4) == 32 and m.row_bytes(8, m.MXFP4) == 16


def test_grad_clip_refusals():
    m = mfet()
    A = 1 << 20

    def st(max_norm=1.0, norm=A, scratch=A, nbytes=1 << 20, **kw):
        v = dict(src=A, dst=A, rows=4, cols=8, ld=0, n_rows=None, dtype=m.F32, flags=0)
        v.update(kw)
        arr = (m.Grad * 1)(m.Grad(v["src"], v["dst"], v["rows"], v["cols"], v["ld"], v["n_rows"], v["dtype"], v["flags"]))
        return status(m.mfet_grad_clip, (arr, 1), max_norm, norm, scratch, nbytes)
    assert st(max_norm=-1.0) == m.ERR_INVALID_ARG
    assert st(max_norm=float("nan")) == m.ERR_INVALID_ARG
    assert st(src=None) == m.ERR_INVALID_ARG
    assert st(rows=-1) == m.ERR_INVALID_ARG
    assert st(cols=-1) == m.ERR_INVALID_ARG
    assert st(ld=7) == m.ERR_INVALID_ARG
    assert st(rows=1 << 40, cols=1 << 40) == m.ERR_INVALID_ARG
    assert st(dtype=m.INT4) == m.ERR_INVALID_ARG
    assert st(flags=1) == m.ERR_INVALID_ARG
    assert st(src=A + 2) == m.ERR_ALIGNMENT
    assert st(dst=A + 1, dtype=m.F16) == m.ERR_ALIGNMENT
    assert st(n_rows=A + 4) == m.ERR_ALIGNMENT
    assert st(norm=A + 2) == m.ERR_ALIGNMENT
    assert st(scratch=A + 4) == m.ERR_ALIGNMENT
    assert st(nbytes=0) == m.ERR_WORKSPACE
    assert st(scratch=None) == m.ERR_WORKSPACE
    assert status(m.mfet_grad_clip, (None, 1), 1.0, A, A, 1 << 20) == m.ERR_INVALID_ARG
    assert status(m.mfet_grad_clip, (None, -1), 1.0, A, A, 1 << 20) == m.ERR_INVALID_ARG
    assert m.mfet_grad_clip_bytes(-1) == 0 and m.mfet_grad_clip_bytes(1) > 0
    assert m.mfet_grad_clip_bytes(5000) > m.mfet_grad_clip_bytes(400)


def test_make_grads_refusals():
    import torch
    m = mfet()
    a = torch.zeros(4, 6)
    assert status(m.make_grads, [a], [a.half()]) == m.ERR_INVALID_ARG
    assert status(m.make_grads, [a], [a[:3]]) == m.ERR_INVALID_ARG
    assert status(m.make_grads, [a.t()], [a.t()]) == m.ERR_INVALID_ARG
    assert status(m.make_grads, [a.double()], [None]) == m.ERR_INVALID_ARG
    arr, n = m.make_grads([a, a[:, :5], a[0]], [None, a[:, :5], a[0]])
    assert n == 3 and (arr[0].rows, arr[0].cols, arr[0].ld) == (4, 6, 6) and arr[0].dst is None
    assert (arr[1].rows, arr[1].cols, arr[1].ld) == (4, 5, 6) and (arr[2].rows, arr[2].cols) == (1, 6)


def test_mx4_refusals():
    m = mfet()
    A = 1 << 20
    assert m.mfet_mx4_code_bytes(3, 33) == 3 * 2 * 16 and m.mfet_mx4_scale_bytes(129, 129) == 2 * 2 * 512
    assert m.mfet_mx4_code_bytes(-1, 5) == 0 and m.mfet_mx4_scale_bytes(5, 0) == 0 and m.mfet_mx4_linear_bytes(5, 0) == 0

    def q(x=A, dtype=m.F32, ld=64, rows=4, k=64, codes=A, scales=A):
        return status(m.mfet_mx4_quantize, x, dtype, ld, rows, k, codes, scales)
    assert q(x=None) == m.ERR_INVALID_ARG and q(codes=None) == m.ERR_INVALID_ARG and q(scales=None) == m.ERR_INVALID_ARG
    assert q(dtype=m.INT4) == m.ERR_INVALID_ARG and q(ld=63) == m.ERR_INVALID_ARG and q(rows=-1) == m.ERR_INVALID_ARG
    assert q(k=0) == m.ERR_INVALID_ARG
    assert q(x=A + 2) == m.ERR_ALIGNMENT and q(codes=A + 8) == m.ERR_ALIGNMENT and q(scales=A + 4) == m.ERR_ALIGNMENT
    m.mfet_mx4_quantize(None, m.F32, 64, 0, 64, None, None)

    def mm(a=A, asc=A, rows=200, w=A, wsc=A, n=64, k=64, bias=None, act=0, y=A, yd=m.F32, ld=64):
        return status(m.mfet_mx4_matmul, a, asc, rows, w, wsc, n, k, bias, act, y, yd, ld)
    for kw in (dict(a=None), dict(asc=None), dict(w=None), dict(wsc=None), dict(y=None), dict(rows=-1), dict(n=-1), dict(k=0),
               dict(act=2), dict(yd=m.INT4), dict(ld=63)):
        assert mm(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(a=A + 8), dict(asc=A + 8), dict(w=A + 4), dict(wsc=A + 1), dict(y=A + 2), dict(bias=A + 2)):
        assert mm(**kw) == m.ERR_ALIGNMENT, kw
    m.mfet_mx4_matmul(None, None, 0, None, None, 64, 64, None, 0, None, m.F32, 64)

    def li(x=A, xd=m.F32, xld=64, rows=200, w=A, wsc=A, n=64, k=64, bias=None, act=0, y=A, yd=m.F32, ld=64, scratch=A, nbytes=1 << 20):
        return status(m.mfet_mx4_linear, x, xd, xld, rows, w, wsc, n, k, bias, act, y, yd, ld, scratch, nbytes)
    for kw in (dict(x=None), dict(w=None), dict(wsc=None), dict(y=None), dict(rows=-1), dict(n=-1), dict(k=0), dict(act=2),
               dict(xd=m.INT4), dict(yd=m.INT4), dict(ld=63), dict(xld=63)):
        assert li(**kw) == m.ERR_INVALID_ARG, kw
    for kw in (dict(x=A + 2), dict(w=A + 4), dict(wsc=A + 1), dict(y=A + 2), dict(bias=A + 2), dict(scratch=A + 8)):
        assert li(**kw) == m.ERR_ALIGNMENT, kw
    assert li(scratch=None) == m.ERR_WORKSPACE and li(nbytes=100) == m.ERR_WORKSPACE
    m.mfet_mx4_linear(None, m.F32, 64, 0, None, None, 64, 64, None, 0, None, m.F32, 64, None, 0)


def test_struct_layout():
    m = mfet()
    assert C.sizeof(m.Grad) == 56 and m.Grad.n_rows.offset == 40 and m.Grad.dtype.offset == 48


def test_make_grads_refuses_rows_that_share_memory():
    """An expanded tensor's rows are one row in memory; as a stride of 0 it would be read as rows one behind the other."""
    import torch
    m = mfet()
    w = torch.zeros(4, 6, requires_grad=True)
    grad, = torch.autograd.grad((w.sum(0) * torch.arange(6.0)).sum(), w)
    assert grad.stride() == (0, 1)
    for t in (grad, torch.zeros(64).expand(10, 64), torch.zeros(1, 1).expand(5, 1), torch.zeros(20).as_strided((4, 6), (3, 1)),
              torch.zeros(1).expand(7)):
        assert status(m.make_grads, [t], [None]) == m.ERR_INVALID_ARG
        assert status(m.make_grads, [t], [t]) == m.ERR_INVALID_ARG
    for t in (torch.zeros(64).expand(1, 64), torch.zeros(0, 6), torch.zeros(4, 0), torch.zeros(()), torch.zeros(2, 3, 4), torch.zeros(5, 1)):
        arr, n = m.make_grads([t], [t])
        assert n == 1 and arr[0].rows * arr[0].cols == t.numel() and (arr[0].rows < 2 or arr[0].ld >= arr[0].cols)


def test_make_grads_looks_at_the_counts():
    """The library reads one 64-bit count per tensor, 8 bytes apart."""
    import torch
    m = mfet()
    a, b = torch.zeros(4, 6), torch.zeros(5, 3)
    for counts in (torch.zeros(2, dtype=torch.int32), torch.zeros(2), torch.zeros(1, dtype=torch.int64), torch.zeros(4, dtype=torch.int64)[::2],
                   torch.zeros(0, dtype=torch.int64), torch.zeros(1, dtype=torch.int64).expand(2), torch.zeros(2, dtype=torch.int64, device="meta")):
        assert status(m.make_grads, [a, b], [None, None], counts) == m.ERR_INVALID_ARG
    for counts in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int64), torch.zeros(2, 1, dtype=torch.int64)):
        arr, n = m.make_grads([a, b], [None, b], counts)
        assert n == 2 and [arr[i].n_rows for i in range(2)] == [counts.data_ptr(), counts.data_ptr() + 8]


def test_make_grads_wants_a_destination_for_every_tensor():
    """A list that ends early would drop the tensors behind its end from the norm."""
    import torch
    m = mfet()
    a, b = torch.zeros(4, 6), torch.zeros(5, 3)
    for src, dst in (([a, b], [a]), ([a], [a, b]), ([], [None]), ([a], [])):
        assert status(m.make_grads, src, dst) == m.ERR_INVALID_ARG
    assert m.make_grads([], [])[1] == 0


def test_make_grads_wants_a_destination_on_the_same_device():
    import torch
    m = mfet()
    a = torch.zeros(4, 6)
    assert status(m.make_grads, [a], [torch.zeros(4, 6, device="meta")]) == m.ERR_INVALID_ARG


def test_make_grads_keeps_what_its_addresses_point_at():
    """The list is kept from step to step: the memory behind it must not be handed to somebody else meanwhile."""
    import gc
    import weakref

    import torch
    m = mfet()

    def make():
        src, dst, counts = [torch.zeros(4, 6), torch.zeros(7)], [torch.zeros(4, 6), None], torch.zeros(2, dtype=torch.int64)
        return m.make_grads(src, dst, counts), [weakref.ref(t) for t in src + dst[:1] + [counts]]
    grads, held = make()
    gc.collect()
    assert all(r() is not None for r in held)
    del grads
    gc.collect()
    assert all(r() is None for r in held)


def test_lists_counts_and_status_words_are_aligned():
    """A kernel reads them as 64-bit and 32-bit words: an address between two words is refused like any other."""
    m = mfet()
    A = 1 << 20
    d = m.TableDesc(A, 100, 64, m.MXFP4, m.LOC_DEVICE, 0, 0, 0)
    for call in (m.mfet_rows_write, m.mfet_rows_read):
        for off in (1, 4):
            assert status(call, d, A + off, 5, None, A, m.F32, 64) == m.ERR_ALIGNMENT
            assert status(call, d, A, 5, A + off, A, m.F32, 64) == m.ERR_ALIGNMENT
        assert status(call, d, A, 5, None, A, m.F32, 64, A + 2) == m.ERR_ALIGNMENT
    assert status(m.mfet_mx4_matmul, A, A, 200, A, A, 64, 64, None, 0, A, m.F32, 64, A + 2) == m.ERR_ALIGNMENT
    assert status(m.mfet_mx4_linear, A, m.F32, 64, 200, A, A, 64, 64, None, 0, A, m.F32, 64, A, 1 << 20, A + 1) == m.ERR_ALIGNMENT
    assert status(m.mfet_mx4_linear, A, m.F32, 64, 2, A, A, 64, 64, None, 0, A, m.F32, 64, None, 0, A + 1) == m.ERR_ALIGNMENT


def test_descriptors_shorter_than_their_structure():
    """The library reads whole structures: what lends less memory than that is refused."""
    m = mfet()
    A = 1 << 20
    for call in (m.mfet_rows_write, m.mfet_rows_read):
        for short in (b"", bytes(47), bytearray(16)):
            assert status(call, short, A, 5, None, A, m.F32, 64) == m.ERR_INVALID_ARG
        assert status(call, None, A, 5, None, A, m.F32, 64) == m.ERR_INVALID_ARG
    one = (m.Grad * 1)(m.Grad(A, A, 4, 8, 0, None, m.F32, 0))
    for n in (2, 1000, 2**31 - 1):
        assert status(m.mfet_grad_clip, (one, n), 1.0, A, A, 1 << 20) == m.ERR_INVALID_ARG
    assert status(m.mfet_grad_clip, (bytes(55), 1), 1.0, A, A, 1 << 20) == m.ERR_INVALID_ARG


def test_integers_that_do_not_fit_their_argument():
    """2^32 is no dtype 0, and -1 bytes of scratch are not 2^64 - 1."""
    m = mfet()
    A, big = 1 << 20, 1 << 32
    d = m.TableDesc(A, 100, 64, m.MXFP4, m.LOC_DEVICE, 0, 0, 0)
    for wrong in (big, big + 2, -big, -1, 2**62):
        for call in (m.mfet_rows_write, m.mfet_rows_read):
            assert status(call, d, A, 5, None, A, wrong, 64) == m.ERR_INVALID_ARG
        assert status(m.mfet_mx4_quantize, A, wrong, 64, 4, 64, A, A) == m.ERR_INVALID_ARG
        assert status(m.mfet_mx4_matmul, A, A, 200, A, A, 64, 64, None, wrong, A, m.F32, 64) == m.ERR_INVALID_ARG
        assert status(m.mfet_mx4_matmul, A, A, 200, A, A, 64, 64, None, 0, A, wrong, 64) == m.ERR_INVALID_ARG
        for at in (1, 9, 11):
            args = [A, m.F32, 64, 200, A, A, 64, 64, None, 0, A, m.F32, 64, A, 1 << 20]
            args[at] = wrong
            assert status(m.mfet_mx4_linear, *args) == m.ERR_INVALID_ARG
        assert status(m.mfet_grad_clip, (None, -big + (wrong & 1)), 1.0, A, A, 1 << 20) == m.ERR_INVALID_ARG
    for nbytes in (-1, -2**63):
        one = (m.Grad * 1)(m.Grad(A, A, 4, 8, 0, None, m.F32, 0))
        assert status(m.mfet_grad_clip, (one, 1), 1.0, A, A, nbytes) == m.ERR_INVALID_ARG
        assert status(m.mfet_mx4_linear, A, m.F32, 64, 200, A, A, 64, 64, None, 0, A, m.F32, 64, A, nbytes) == m.ERR_INVALID_ARG
