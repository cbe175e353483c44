"""The orthogonalised update against the 64-bit definition (bound of block_reference.orthogonalize_bound, by Frobenius norm)."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu


def update(rows, cols, dtype=torch.float32, pad=0, shift=0, seed=0, size=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=dtype, device="cuda")
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    r = min(3, rows, cols)
    noise = torch.randn(rows, cols, generator=g, device="cuda")
    shared = torch.randn(rows, r, generator=g, device="cuda") @ torch.randn(r, cols, generator=g, device="cuda")
    view.copy_(size * (noise + 2 * shared))
    return buf, view


def call(g, out, coefficients=None, steps=5, scale=1.0, scratch=None, stream=None):
    m = mfet()
    rows, cols = g.shape
    if scratch is None:  # whatever it held before does not matter
        scratch = torch.full((m.mfet_orthogonalize_bytes(rows, cols),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    s = torch.cuda.current_stream() if stream is None else stream
    m.mfet_orthogonalize(g, m.dtype_of(g), g.stride(0), rows, cols, coefficients, steps, scale, out, m.dtype_of(out), out.stride(0), scratch,
                         scratch.numel(), status, s.cuda_stream)
    return status


def check(g, out, coefficients=None, steps=5, scale=1.0):
    steps = [ref.USUAL] * steps if coefficients is None else [tuple(float(v) for v in c) for c in coefficients]
    want = ref.orthogonalize(g.double(), steps, scale)
    off = float(torch.linalg.vector_norm(out.double() - want))
    bound = ref.orthogonalize_bound(want, g, steps, scale, out.dtype)
    assert off <= bound, (off, bound)


SIZES = [(1, 1), (1, 50), (50, 1), (2, 3), (16, 16), (48, 192), (192, 48), (64, 64), (65, 129), (128, 128), (129, 1000), (257, 256), (300, 301),
         (700, 300), (512, 1100), (900, 896)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("src,dst,pad,shift", [("f32", "f32", 0, 0), ("bf16", "bf16", 0, 0), ("f16", "f32", 3, 1), ("bf16", "f16", 5, 3)])
def test_against_the_definition(rows, cols, src, dst, pad, shift):
    _, g = update(rows, cols, ref.DT[src], pad, shift, seed=rows)
    buf, out = update(rows, cols, ref.DT[dst], pad, shift)
    keep = g.clone()
    status = call(g, out)
    check(g, out)
    assert int(status.item()) == 0 and torch.equal(g, keep)
    out.fill_(7.0)
    assert bool((buf == 7.0).all())


@pytest.mark.parametrize("rows,cols", [(2048, 1024), (1000, 3000), (2100, 2100)])
def test_large(rows, cols):
    _, g = update(rows, cols, torch.bfloat16)
    out = torch.empty(rows, cols, device="cuda")
    call(g, out)
    check(g, out)


@pytest.mark.parametrize("steps", [1, 2, 3, 6])
def test_steps_and_scale(steps):
    _, g = update(100, 260)
    out = torch.empty_like(g)
    call(g, out, steps=steps, scale=-0.3)
    check(g, out, steps=steps, scale=-0.3)
    call(g, out, steps=steps, scale=0.0)
    assert not bool(out.any())


@pytest.mark.parametrize("rows,cols", [(60, 90), (400, 150)])
def test_coefficients_of_every_step(rows, cols):
    """A schedule that converges: the result is the nearest matrix with orthonormal rows or columns. Its last steps leave singular values at 1,
    where the slope is 0, so what is left is the last steps' own rounding and what has not converged (the smallest singular value of the
    updates here, 0.02 of the norm and more, is inside 2^-20 of 1 after these steps)."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    m = torch.randn(rows, cols, generator=g, device="cuda")
    u, s, vh = torch.linalg.svd(m.double(), full_matrices=False)
    s = 1.0 + torch.rand(s.shape, generator=g, device="cuda", dtype=torch.float64)
    m = ((u * s) @ vh).float()
    schedule = [[3.4445, -4.775, 2.0315]] * 3 + [[1.875, -1.25, 0.375]] * 9
    out = torch.empty_like(m)
    call(m, out, schedule, len(schedule))
    check(m, out, schedule)
    assert float((out.double() - u @ vh).abs().max()) < 2.0**-17


def test_scale_of_the_update_does_not_matter():
    _, g = update(80, 120, size=1.0)
    out = [torch.empty_like(g) for _ in range(5)]
    for o, e in zip(out, (0, 60, -60, 100, -126)):
        call(g * 2.0**e, o)
        check(g * 2.0**e, o)
    assert all(torch.equal(o, out[0]) for o in out[1:4])  # powers of two change no bit
    top = g / g.abs().max() * 3e38  # squares far outside fp32
    call(top, out[0])
    check(top, out[0])


@pytest.mark.parametrize("rows,cols", [(40, 300), (300, 40)])
def test_zeros_and_values_that_are_not_finite(rows, cols):
    g = torch.zeros(rows, cols, device="cuda")
    out = torch.full_like(g, 3.0)
    call(g, out)
    assert not bool(out.any())
    for bad in (float("nan"), float("inf"), float("-inf")):
        _, g = update(rows, cols)
        g = g.clone()
        g[3, 5] = bad
        call(g, out)
        assert bool(torch.isnan(out).all())
    _, g = update(rows, cols)
    call(g, out)
    check(g, out)


@pytest.mark.parametrize("rows,cols", [(200, 500), (700, 640)])
def test_update_without_some_directions(rows, cols):
    """Rows and columns of zeros, and a matrix of rank 2."""
    _, g = update(rows, cols)
    g = g.clone()
    g[5:50], g[:, 7:20] = 0.0, 0.0
    out = torch.empty_like(g)
    call(g, out)
    check(g, out)
    assert not bool(out[5:50].any()) and not bool(out[:, 7:20].any())
    low = torch.randn(rows, 2, device="cuda") @ torch.randn(2, cols, device="cuda")
    call(low, out)
    check(low, out)


def test_rows_beyond_32_bits():
    ld, rows, cols = 2**28, 18, 40
    big = torch.zeros(ld * (rows - 1) + cols, dtype=torch.bfloat16, device="cuda")
    g = torch.as_strided(big, (rows, cols), (ld, 1))
    g.copy_(torch.randn(rows, cols, device="cuda"))
    out = torch.empty(rows, cols, device="cuda")
    call(g, out)
    check(g, out)
    small = g.contiguous()
    want = out.to(torch.bfloat16)
    call(small, g)
    assert torch.equal(g, want)


def test_same_bits_every_time_and_on_other_streams():
    _, g = update(500, 400)
    out = []
    for _ in range(4):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            o = torch.empty_like(g)
            call(g, o, stream=s)
        s.synchronize()
        out.append(o)
    assert all(torch.equal(o, out[0]) for o in out[1:])


def test_captured_and_replayed_on_new_values():
    _, g = update(260, 300)
    g = g.clone()
    out = torch.empty_like(g)
    m = mfet()
    ws = torch.empty(m.mfet_orthogonalize_bytes(260, 300), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.mfet_orthogonalize(g, 0, 300, 260, 300, [3.0, -3.0, 1.0] * 4, 4, 1.0, out, 0, 300, ws, ws.numel(), status,
                             torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        g.normal_()
        graph.replay()
        torch.cuda.synchronize()
        check(g, out, [(3.0, -3.0, 1.0)] * 4)
    assert int(status.item()) == 0
