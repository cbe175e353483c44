"""The gated linear block and its backward pass against the 64-bit definition (bounds of block_reference.gated, counted in roundings)."""
import threading

import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu", "gelu", "sigmoid"]


def make(rows, cols, dtype, pad=0, shift=0, seed=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    buf = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device="cuda")
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.randn(rows, cols, generator=g, device="cuda") * size)
    return buf, view


class Block:
    """Operands and results of one size; pad and shift: how far rows are apart and from 16-byte boundaries."""

    def __init__(self, m, n, k, dtype="bf16", act="silu", pad=0, shift=0, seed=0, size=1.0):
        t = ref.DT[dtype]
        self.m, self.n, self.k, self.act, self.t = m, n, k, act, t
        self.x = make(m, k, t, pad, shift, seed, size)[1]
        self.wg = make(n, k, t, pad, shift, seed + 1, k**-0.5)[1]
        self.wu = make(n, k, t, pad, shift, seed + 2, k**-0.5)[1]
        self.dh = make(m, n, t, pad, shift, seed + 3, 0.5)[1]
        self.buf = [make(r, c, t, pad, shift) for r, c in ((m, n), (m, k), (n, k), (n, k))]
        self.h, self.dx, self.dwg, self.dwu = (v for _, v in self.buf)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        b = mfet()
        # whatever the scratch held before does not matter
        self.ws = torch.full((max(b.mfet_gated_linear_bytes(m, n, k), b.mfet_gated_linear_backward_bytes(m, n, k)),), 255, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None):
        b = mfet()
        s = torch.cuda.current_stream() if stream is None else stream
        b.mfet_gated_linear(self.x, b.dtype_of(self.x), self.x.stride(0), self.m, self.wg, self.wg.stride(0), self.wu, self.wu.stride(0), self.n,
                            self.k, ACTS.index(self.act), self.h, self.h.stride(0), self.ws, b.mfet_gated_linear_bytes(self.m, self.n, self.k),
                            self.status, s.cuda_stream)

    def backward(self, stream=None, dx=True, dw=True):
        b = mfet()
        s = torch.cuda.current_stream() if stream is None else stream
        b.mfet_gated_linear_backward(self.x, b.dtype_of(self.x), self.x.stride(0), self.m, self.wg, self.wg.stride(0), self.wu, self.wu.stride(0),
                                     self.n, self.k, ACTS.index(self.act), self.dh, self.dh.stride(0), self.dx if dx else None,
                                     self.dx.stride(0) if dx else 0, self.dwg if dw else None, self.dwg.stride(0) if dw else 0,
                                     self.dwu if dw else None, self.dwu.stride(0) if dw else 0, self.ws, self.ws.numel(), self.status,
                                     s.cuda_stream)

    def check_forward(self):
        h, bound = ref.gated(self.x.double(), self.wg.double(), self.wu.double(), self.act, self.t)
        assert ref.within(self.h, h, bound)
        assert int(self.status.item()) == 0

    def check_backward(self, dx=True, dw=True):
        wx, wg, wu, ex, eg, eu = ref.gated(self.x.double(), self.wg.double(), self.wu.double(), self.act, self.t, self.dh.double())
        if dx:
            assert ref.within(self.dx, wx, ex)
        if dw:
            assert ref.within(self.dwg, wg, eg)
            assert ref.within(self.dwu, wu, eu)
        assert int(self.status.item()) == 0


SIZES = [(1, 1, 1), (1, 896, 896), (2, 65, 17), (5, 128, 64), (8, 1000, 2048), (9, 40, 8), (63, 129, 65), (127, 127, 127), (128, 64, 192), (129, 33, 300), (256, 256, 256),
         (300, 700, 1075), (1000, 24, 40), (17, 2000, 100)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype,pad,shift", [("bf16", 0, 0), ("f16", 3, 1), ("f16", 8, 0), ("bf16", 1, 7)])
def test_both_directions(m, n, k, dtype, pad, shift):
    b = Block(m, n, k, dtype, "silu" if dtype == "bf16" else "gelu", pad, shift, seed=m)
    keep = [t.clone() for t in (b.x, b.wg, b.wu, b.dh)]
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()
    assert all(torch.equal(a, c) for a, c in zip(keep, (b.x, b.wg, b.wu, b.dh)))
    for buf, view in b.buf:  # what lies between and around the rows is as it was
        view.fill_(7.0)
        assert bool((buf == 7.0).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m", [3, 200])
def test_activations(act, dtype, m):
    b = Block(m, 150, 96, dtype, act, seed=4, size=3.0)  # gates from -10 to 10
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("m,n,k", [(2048, 2048, 512), (4099, 1030, 896), (700, 4096, 1500), (16384, 256, 128), (64, 16384, 64), (20000, 8, 16)])
def test_many_tiles(m, n, k):
    """More tiles than blocks, bands of tiles that end early, long sums."""
    b = Block(m, n, k, "bf16", "silu", seed=n)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("m,n,k", [(8192, 1024, 896), (5000, 1500, 700), (19000, 700, 260), (2500, 4000, 1000), (12000, 130, 2000)])
def test_both_gradients_in_one_launch(m, n, k):
    """More tiles of 256 x 256 than the GPU takes at a time, of products of different lengths."""
    b = Block(m, n, k, "bf16", "relu", seed=m)
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("m", [4, 300])
def test_gradients_one_by_one(m):
    for dx, dw in ((True, False), (False, True), (False, False)):
        b = Block(m, 90, 120, "f16")
        old = b.dx.clone(), b.dwg.clone()
        b.backward(dx=dx, dw=dw)
        b.check_backward(dx, dw)
        assert dx or torch.equal(b.dx, old[0])
        assert dw or torch.equal(b.dwg, old[1])


def test_no_rows_and_no_units():
    m = mfet()
    t = torch.full((6, 8), 3.0, dtype=torch.float16, device="cuda")
    w = torch.full((6, 8), 3.0, dtype=torch.float16, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    m.mfet_gated_linear_backward(None, 1, 5, 0, t, 8, t, 8, 6, 5, 0, None, 6, None, 0, t, 8, w, 8, None, 0, None, s)
    assert not bool(t[:, :5].any()) and not bool(w[:, :5].any()) and bool((t[:, 5:] == 3.0).all())
    t.fill_(3.0)
    m.mfet_gated_linear_backward(None, 1, 5, 6, None, 5, None, 5, 0, 5, 0, None, 0, t, 8, None, 0, None, 0, None, 0, None, s)
    assert not bool(t[:, :5].any()) and bool((t[:, 5:] == 3.0).all())


@pytest.mark.parametrize("m", [4, 200])
def test_values_that_are_not_finite_stay_in_their_row_and_column(m):
    b = Block(m, 70, 50, "bf16", "silu")
    b.x[2, 3] = float("nan")
    b.wg[5, 1] = float("inf")
    b.forward()
    bad = torch.isnan(b.h) | torch.isinf(b.h)
    rows, cols = torch.zeros(m, dtype=torch.bool, device="cuda"), torch.zeros(70, dtype=torch.bool, device="cuda")
    rows[2], cols[5] = True, True
    assert bool(torch.isnan(b.h[2]).all()) and not bool(bad[~rows][:, ~cols].any())
    b.wg[5, 1] = 0.0
    b.dh[1] = float("inf")
    b.backward()
    keep = torch.ones(m, dtype=torch.bool, device="cuda")
    keep[1:3] = False
    assert bool(torch.isfinite(b.dx[keep]).all()) and bool(torch.isnan(b.dx[2]).all())


@pytest.mark.parametrize("m", [5, 130])
def test_gates_at_the_ends_of_their_range(m):
    """e^-g leaves fp32's range on both sides."""
    for act in ACTS:
        b = Block(m, 64, 16, "bf16", act)
        b.x.fill_(1.0)
        b.wg.zero_()
        b.wu.fill_(0.0625)
        v = torch.tensor([-1e4, -200.0, -120.0, -89.0, -88.0, -30.0, -1e-3, 0.0, 1e-3, 30.0, 88.0, 89.0, 120.0, 200.0, 1e4], device="cuda")
        b.wg[:15, 0] = v.to(b.t)
        b.forward()
        b.check_forward()
        b.backward()
        assert bool(torch.isfinite(b.dx).all()) and bool(torch.isfinite(b.dwg).all())
        b.check_backward()


def test_gradient_agrees_with_differences():
    b = Block(40, 30, 20, "f16", "gelu")
    b.backward()
    wx, _, _, ex, _, _ = ref.gated(b.x.double(), b.wg.double(), b.wu.double(), b.act, b.t, b.dh.double())
    v, h = torch.randn(40, 20, dtype=torch.float64, device="cuda"), 1e-4
    f = lambda p: (ref.gated(p, b.wg.double(), b.wu.double(), b.act, b.t)[0] * b.dh.double()).sum()
    diff = float((f(b.x.double() + h * v) - f(b.x.double() - h * v)) / (2 * h))
    assert abs(diff - float((b.dx.double() * v).sum())) < float((ex * v.abs()).sum()) + 1e-6 * float((wx * v).abs().sum())


@pytest.mark.parametrize("m", [1, 3])
def test_rows_beyond_32_bits(m):
    """Rows of x and the weights 2^28 elements apart: most start beyond 2^32 bytes, the last ones beyond 2^32 elements."""
    ld, n, k = 2**28, 18, 24
    big = torch.zeros(ld * (n - 1) + k, dtype=torch.bfloat16, device="cuda")
    b = Block(m, n, k)
    wide = torch.as_strided(big, (n, k), (ld, 1))
    wide.copy_(b.wg)
    b.wg = wide
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()
    b2 = Block(n, m, k)
    wide.copy_(b2.x)
    b2.x = wide
    b2.forward()
    b2.check_forward()
    b2.backward()
    b2.check_backward()


@pytest.mark.parametrize("m,n,k", [(6, 512, 896), (700, 333, 500)])
def test_same_bits_every_time_and_on_other_streams(m, n, k):
    b = Block(m, n, k)
    out = []
    for _ in range(4):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        b.forward(s)
        b.backward(s)
        s.synchronize()
        out.append([t.clone() for t in (b.h, b.dx, b.dwg, b.dwu)])
        torch.cuda.synchronize()
    assert all(torch.equal(a, c) for o in out[1:] for a, c in zip(o, out[0]))


def test_two_threads_on_two_streams():
    blocks = [Block(400, 300, 200, seed=1), Block(3, 500, 700, seed=2)]
    errors = []
    torch.cuda.synchronize()

    def work(b):
        s = torch.cuda.Stream()
        try:
            for _ in range(50):
                b.forward(s)
                b.backward(s)
            s.synchronize()
        except Exception as e:  # handed to the test's own thread
            errors.append(e)
    threads = [threading.Thread(target=work, args=(b,)) for b in blocks]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors, errors[0]
    for b in blocks:
        b.check_forward()
        b.check_backward()


@pytest.mark.parametrize("m,n,k,pad", [(7, 256, 512, 0), (300, 200, 260, 3), (2048, 512, 640, 0)])
def test_captured_and_replayed_on_new_values(m, n, k, pad):
    b = Block(m, n, k, pad=pad)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward()
        b.backward()
    for _ in range(2):
        b.x.normal_()
        b.dh.normal_()
        graph.replay()
        torch.cuda.synchronize()
        b.check_forward()
        b.check_backward()
