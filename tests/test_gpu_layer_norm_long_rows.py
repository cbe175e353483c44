"""Layer norm of rows that no block holds: their mean is as good as that of shorter ones."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu
U = ref.U


def normal(x, w, b, eps, dtype):
    m = mfet()
    rows, cols = x.shape
    y = torch.empty(rows, cols, dtype=dtype, device="cuda")
    m.mfet_layer_norm(x, m.dtype_of(x), cols, rows, cols, w, b, eps, y, m.dtype_of(y), cols, torch.cuda.current_stream().cuda_stream)
    return y


def parts(x, eps):
    """(xh, r, bound of xh). A sum over a row has n = cols / 512 + 30 additions one after the other (512 threads, 8 neighbouring values each, then lanes and
    warps), each off by U of it. So the first mean is off by n U mean|x|; the differences d from it are off by U |d| and are of the size of the true ones and
    that; their mean, which is taken off again, by (n + 2) U of theirs. r is off by (n + 10) U of itself, and by what its variance has of the mean's error,
    which is taken out the same way."""
    cols = x.shape[1]
    n = cols / 512 + 30
    d = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    first = n * U * x.abs().mean(1, keepdim=True)
    off = r * (n + 4) * U * (d.abs().mean(1, keepdim=True) + first) + r * U * (d.abs() + first)
    rel = (n + 10) * U * (1 + 2 * (r * first) ** 2)
    return d * r, r, off + rel * (d * r).abs() + off * off


@pytest.mark.parametrize("cols", [16385, 20000, 2**20 + 3, 2**22])
@pytest.mark.parametrize("mean,spread", [(1.9, 0.0), (-1000.0, 1.0), (10.0, 1e-3), (0.0, 1.0)])
def test_rows_far_from_zero(cols, mean, spread):
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = mean + spread * torch.randn(3, cols, generator=g, device="cuda")
    xh, _, bound = parts(x.double(), 1e-5)
    y = normal(x, None, None, 1e-5, torch.float32)
    assert ref.within(y, xh, bound + 4 * U * xh.abs())
    x[1, 5] = float("inf")  # and nothing of it in the other rows
    y2 = normal(x, None, None, 1e-5, torch.float32)
    assert bool(torch.isnan(y2[1]).all()) and torch.equal(y2[::2], y[::2])


@pytest.mark.parametrize("cols,mean,spread", [(20011, -1000.0, 1.0), (2**20, 1.9, 0.0), (2**20, 0.5, 1.0)])
def test_gradients_of_rows_far_from_zero(cols, mean, spread):
    m = mfet()
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = mean + spread * torch.randn(5, cols, generator=g, device="cuda")
    dy, w = torch.randn(5, cols, generator=g, device="cuda"), 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    ws = torch.full((m.mfet_layer_norm_backward_bytes(5, cols),), 255, dtype=torch.uint8, device="cuda")
    m.mfet_layer_norm_backward(x, m.F32, cols, 5, cols, w, 1e-5, dy, m.F32, cols, dx, cols, dw, db, ws, ws.numel(), torch.cuda.current_stream().cuda_stream)
    xh, r, dxh = parts(x.double(), 1e-5)
    t, n = dy.double() * w.double(), cols / 512 + 30
    m0, m1 = t.mean(1, keepdim=True), (t * xh).mean(1, keepdim=True)
    want = r * (t - m0 - xh * m1)
    rel = dxh.amax(1, keepdim=True) + (n + 10) * U
    bound = r * (n * U * (t.abs().mean(1, keepdim=True) + xh.abs() * (t * xh).abs().mean(1, keepdim=True)) + dxh * m1.abs()
                 + (xh.abs() + dxh) * (t.abs() * dxh).mean(1, keepdim=True) + 6 * U * (t.abs() + m0.abs() + (xh * m1).abs())) + rel * want.abs()
    assert ref.within(dx, want, bound)
    assert ref.within(dw, (dy.double() * xh).sum(0), (dy.double().abs() * dxh).sum(0) + 16 * U * (dy.double() * xh).abs().sum(0))
    assert ref.within(db, dy.double().sum(0), 16 * U * dy.double().abs().sum(0))
