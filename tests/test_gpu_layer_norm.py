"""Layer norm and its backward pass against the 64-bit definition (bounds of block_reference.norm, counted in roundings)."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu
EPS = 1e-5


def make(rows, cols, dtype, pad=0, shift=0, seed=0, size=1.0, centre=0.0):
    """A [rows, cols] view of a buffer whose rows are cols + pad apart and start `shift` elements behind a 16-byte boundary."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device="cuda")
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.randn(rows, cols, generator=g, device="cuda") * size + centre)
    return buf, view


def forward(x, w, b, y, eps=EPS, stream=None):
    m = mfet()
    s = torch.cuda.current_stream() if stream is None else stream
    m.mfet_layer_norm(x, m.dtype_of(x), x.stride(0), x.shape[0], x.shape[1], w, b, eps, y, m.dtype_of(y), y.stride(0), s.cuda_stream)


def backward(x, w, dy, dx, dw, db, eps=EPS, scratch=None):
    m = mfet()
    if scratch is None and (dw is not None or db is not None):  # whatever it held before does not matter
        scratch = torch.full((m.mfet_layer_norm_backward_bytes(*x.shape) // 4,), float("nan"), device="cuda")
    m.mfet_layer_norm_backward(x, m.dtype_of(x), x.stride(0), x.shape[0], x.shape[1], w, eps, dy, m.dtype_of(dy), dy.stride(0), dx,
                               dx.stride(0), dw, db, scratch, 0 if scratch is None else scratch.numel() * scratch.element_size(),
                               torch.cuda.current_stream().cuda_stream)


def check_forward(x, w, b, y, eps=EPS):
    want, bound = ref.norm(x.double(), None if w is None else w.double(), None if b is None else b.double(), eps)
    assert ref.within(y, want, bound + ref.rounding(want.abs() + bound, y.dtype))


def check_backward(x, w, dy, dx, dw, db, eps=EPS):
    wx, ww, wb, ex, ew, eb = ref.norm(x.double(), None if w is None else w.double(), None, eps, dy.double())
    assert ref.within(dx, wx, ex + ref.rounding(wx.abs() + ex, dx.dtype))
    if dw is not None:
        assert ref.within(dw, ww, ew + ref.rounding(ww, dw.dtype))
    if db is not None:
        assert ref.within(db, wb, eb + ref.rounding(wb, db.dtype))


COLS = [1, 2, 7, 8, 31, 255, 256, 257, 512, 513, 896, 1024, 1025, 1536, 1537, 2048, 2049, 2560, 3100, 4096, 4097, 5000, 6145, 8192, 8193, 16384, 16385, 20011]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("xt,yt,pad,shift", [("f32", "bf16", 0, 0), ("bf16", "f32", 3, 1), ("f16", "f16", 8, 0), ("f32", "f32", 1, 3), ("bf16", "bf16", 0, 5)])
def test_both_directions(cols, xt, yt, pad, shift):
    rows = 3 if cols > 4096 else 19
    xb, x = make(rows, cols, ref.DT[xt], pad, shift, 1)
    dyb, dy = make(rows, cols, ref.DT[yt], pad, shift, 2)
    w, b = torch.randn(cols, device="cuda") + 1, torch.randn(cols, device="cuda")
    yb, y = make(rows, cols, ref.DT[yt], pad, shift)
    dxb, dx = make(rows, cols, ref.DT[xt], pad, shift)
    dw, db = torch.full((cols,), 5.0, device="cuda"), torch.full((cols,), 5.0, device="cuda")
    before = x.clone(), dy.clone()
    forward(x, w, b, y)
    backward(x, w, dy, dx, dw, db)
    check_forward(x, w, b, y)
    check_backward(x, w, dy, dx, dw, db)
    assert torch.equal(x, before[0]) and torch.equal(dy, before[1])
    for buf, view in ((yb, y), (dxb, dx)):  # what lies between and around the rows is as it was
        view.fill_(7.0)
        assert bool((buf == 7.0).all())


@pytest.mark.parametrize("xt,yt", [("f32", "f32"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("pad", [0, 7])
def test_one_column_has_no_gradient(xt, yt, pad):
    """With one column x - mu and t - mean(t) are 0, whatever their size; with two equal ones and equal gradients, too."""
    for cols in (1, 2):
        rows = 333
        _, x = make(rows, cols, ref.DT[xt], pad, seed=1)
        _, dy = make(rows, cols, ref.DT[yt], pad, seed=2, size=37.0)
        if cols == 2:
            x[:, 1], dy[:, 1] = x[:, 0], dy[:, 0]
        w, b = torch.full((cols,), 1.3, device="cuda"), torch.full((cols,), 0.7, device="cuda")
        _, y = make(rows, cols, ref.DT[yt], pad)
        _, dx = make(rows, cols, ref.DT[xt], pad)
        forward(x, w, b, y)
        backward(x, w, dy, dx, None, None)
        assert torch.equal(y, b.to(y.dtype).expand(rows, cols))
        assert not dx.any()


@pytest.mark.parametrize("rows", [1, 2, 8, 9, 147, 5000, 20000])
@pytest.mark.parametrize("cols", [64, 1500])
def test_row_counts(rows, cols):
    _, x = make(rows, cols, torch.float32, seed=rows)
    _, dy = make(rows, cols, torch.bfloat16, seed=3, size=0.01)
    w, b = torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    forward(x, w, b, y)
    backward(x, w, dy, dx, dw, db)
    check_forward(x, w, b, y)
    check_backward(x, w, dy, dx, dw, db)


def test_no_rows():
    x = torch.empty(0, 16, device="cuda")
    dw, db = torch.ones(16, device="cuda"), torch.ones(16, device="cuda")
    backward(x, None, x, x, dw, db, scratch=torch.empty(4, device="cuda"))
    assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("cols", [40, 3000, 17000])
@pytest.mark.parametrize("w,dw,db", [(False, True, True), (True, False, True), (True, True, False), (False, False, False)])
def test_optional_arguments(cols, w, dw, db):
    _, x = make(11, cols, torch.float16)
    _, dy = make(11, cols, torch.float32, seed=5)
    w = torch.randn(cols, device="cuda") if w else None
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw, db = (torch.empty(cols, device="cuda") if v else None for v in (dw, db))
    forward(x, w, None, y)
    backward(x, w, dy, dx, dw, db)
    check_forward(x, w, None, y)
    check_backward(x, w, dy, dx, dw, db)


@pytest.mark.parametrize("cols", [33, 2000, 17000])
def test_rows_far_from_zero_and_of_any_scale(cols):
    for size, centre in ((1.0, 100.0), (1e-3, 10.0), (1e-15, 0.0), (1e15, 0.0), (1e-18, 1e-16)):
        for eps in (1e-5, 0.0):
            _, x = make(5, cols, torch.float32, size=size, centre=centre)
            _, dy = make(5, cols, torch.float32, seed=1)
            w, b = torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")
            y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
            forward(x, w, b, y, eps)
            backward(x, w, dy, dx, dw, db, eps)
            check_forward(x, w, b, y, eps)
            check_backward(x, w, dy, dx, dw, db, eps)


def test_constant_rows_and_values_that_are_not_finite():
    x = torch.randn(6, 300, device="cuda")
    x[1], x[2, 5], x[3, 7], x[4] = 2.5, float("nan"), float("inf"), 0.0
    w, b = torch.randn(300, device="cuda"), torch.randn(300, device="cuda")
    y = torch.empty_like(x)
    forward(x, w, b, y)
    assert torch.equal(y[1], b) and torch.equal(y[4], b)
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).all())  # the row alone
    ok = [0, 5]
    check_forward(x[ok], w, b, y[ok])
    dx, dy = torch.empty_like(x), torch.randn(6, 300, device="cuda")
    dw, db = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    backward(x, w, dy, dx, dw, db)
    assert bool(torch.isfinite(dx[[0, 1, 4, 5]]).all()) and bool(torch.isnan(dx[2]).all()) and bool(torch.isfinite(db).all())


def test_gradient_agrees_with_differences():
    """Of the 64-bit definition: <dx, v> against (f(x + h v) - f(x - h v)) / 2h, whose own error is h^2 of the third derivative."""
    _, x = make(9, 130, torch.float32)
    _, dy = make(9, 130, torch.float32, seed=1)
    w = torch.randn(130, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(130, device="cuda"), torch.empty(130, device="cuda")
    backward(x, w, dy, dx, dw, db)
    v = torch.randn(9, 130, dtype=torch.float64, device="cuda")
    h = 1e-4
    f = lambda p: (ref.norm(p, w.double(), None, EPS)[0] * dy.double()).sum()
    diff = float((f(x.double() + h * v) - f(x.double() - h * v)) / (2 * h))
    got = float((dx.double() * v).sum())
    assert abs(diff - got) < 1e-6 * float((dx.double() * v).abs().sum())


def test_rows_beyond_32_bits():
    """Rows 2^27 elements apart: the last ones start beyond 2^32 elements."""
    ld, rows, cols = 2**27, 34, 200
    big = torch.empty(ld * (rows - 1) + cols, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (rows, cols), (ld, 1))
    x.copy_(torch.randn(rows, cols, device="cuda"))
    y = torch.empty(rows, cols, device="cuda")
    forward(x, None, None, y)
    check_forward(x, None, None, y)
    dy = torch.randn(rows, cols, device="cuda")
    keep = x.double()
    dx = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    backward(x, None, dy, dx, None, None)
    check_backward(keep, None, dy, dx, None, None)


def test_same_bits_every_time_and_on_other_streams():
    _, x = make(3001, 896, torch.float32)
    _, dy = make(3001, 896, torch.bfloat16, seed=1)
    w = torch.randn(896, device="cuda")
    out = []
    for i in range(3):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty(896, device="cuda"), torch.empty(896, device="cuda")
            forward(x, w, None, y)
            backward(x, w, dy, dx, dw, db)
        s.synchronize()
        out.append((y, dx, dw, db))
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))


def test_captured_and_replayed_on_new_values():
    _, x = make(500, 640, torch.float32)
    _, dy = make(500, 640, torch.float32, seed=1)
    w, b = torch.randn(640, device="cuda"), torch.randn(640, device="cuda")
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(640, device="cuda"), torch.empty(640, device="cuda")
    ws = torch.empty(mfet().mfet_layer_norm_backward_bytes(500, 640), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        forward(x, w, b, y)
        backward(x, w, dy, dx, dw, db, scratch=ws)
    for _ in range(2):
        x.normal_()
        w.normal_()
        graph.replay()
        torch.cuda.synchronize()
        check_forward(x, w, b, y)
        check_backward(x, w, dy, dx, dw, db)
