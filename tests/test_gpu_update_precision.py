"""The orthogonalised update is about as near to the definition as an iteration in fp32, in every form that its sizes choose: one launch of one and of
several blocks, tiles of 64 and of 128 columns, pairs, symmetric products by half, one and two tiles in tensor memory."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet
from tests.test_gpu_orthogonalize import call, update

pytestmark = pytest.mark.gpu


def plain(g, steps):
    """The iteration in fp32, products included."""
    old = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        size = torch.linalg.vector_norm(g.double()).float()
        return ref.orthogonalize(g.float() / size, [ref.USUAL] * steps)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = old


SIZES = [(1, 60), (5, 300), (48, 192), (192, 48), (128, 128), (100, 1000), (128, 2048), (1500, 90), (129, 129), (300, 500), (512, 512), (900, 896), (1024, 896),
         (256, 4096), (1300, 1200), (1700, 1600), (2048, 2048), (2300, 3000)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("steps", [1, 5])
def test_as_near_as_an_iteration_in_fp32(rows, cols, steps):
    """At most twice as far off as the plain iteration, by the median of five updates, and one last rounding: two iterations that both round in fp32, but add
    up in other orders, differ by chance alone.

    A sum of one instruction of the tensor cores (products over a short side of at most 16) is truncated once: half a step of fp32, 2^-24, on average, where
    rounding to nearest has none, and nothing smaller than a step can be put back. Over A (twice, in A A), A A and B X, one step is off by
    2^-24 (|b| |A X| + 3 |c| |A A X| + |b A X + c A A X|) by that. That is added for them; after five steps it is as much of the result as the other errors."""
    off, by = [], []
    for seed in range(5):
        _, g = update(rows, cols, seed=seed)
        want = ref.orthogonalize(g.double(), [ref.USUAL] * steps)
        out = torch.empty_like(g)
        assert int(call(g, out, steps=steps).item()) == 0
        size = float(torch.linalg.vector_norm(want))
        off.append(float(torch.linalg.vector_norm(out.double() - want)) / size)
        by.append(float(torch.linalg.vector_norm(plain(g, steps).double() - want)) / size)
        short = 0.0
        if min(rows, cols) <= 16 and steps == 1:
            bax, caax = (ref.orthogonalize(g.double(), [c]) for c in ((0.0, ref.USUAL[1], 0.0), (0.0, 0.0, ref.USUAL[2])))
            norm = torch.linalg.vector_norm
            short = 2.0**-24 * float(norm(bax) + 3 * norm(caax) + norm(bax + caax)) / size
    print("%d x %d, %d steps: %.2e, in fp32 %.2e" % (rows, cols, steps, sorted(off)[2], sorted(by)[2]))
    assert sorted(off)[2] <= 2 * sorted(by)[2] + 2.0**-24 + short


@pytest.mark.parametrize("rows,cols", [(64, 8192), (8200, 60), (300, 4097), (500, 40000), (40001, 129), (1000, 20000), (64, 2**17 + 9), (2**20, 64), (1, 2**22),
                                       (2048, 16384), (4500, 5000)])
@pytest.mark.parametrize("steps", [1, 5])
def test_long_sides(rows, cols, steps):
    """The same where the sums over the long side (and over a short one of more than 4096) are long."""
    test_as_near_as_an_iteration_in_fp32(rows, cols, steps)


@pytest.mark.parametrize("rows,cols", [(100, 70000), (66000, 300), (1500, 66000)])
def test_long_sides_in_16_bits(rows, cols):
    test_results_in_16_bits_element_by_element(rows, cols, "f16")


@pytest.mark.parametrize("rows,cols", [(1700, 1600), (3000, 2300), (2300, 3000)])
@pytest.mark.parametrize("dst", ["bf16", "f16"])
def test_results_in_16_bits_element_by_element(rows, cols, dst):
    """Half a step of the type, and four times the largest error of an element of the plain iteration in fp32."""
    _, g = update(rows, cols, torch.bfloat16, pad=8)
    want = ref.orthogonalize(g.double(), [ref.USUAL] * 5)
    out = torch.empty(rows, cols, dtype=ref.DT[dst], device="cuda")
    status = call(g, out)
    near = 4 * float((plain(g, 5).double() - want).abs().max())
    assert ref.within(out, want, near + ref.rounding(want.abs() + near, out.dtype))
    assert int(status.item()) == 0
    again = torch.empty_like(out)
    call(g, again)
    assert torch.equal(out, again)
