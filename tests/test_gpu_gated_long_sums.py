"""The gradients of the gated block's weights are sums over the rows: of many rows, they are off by little more than their last rounding."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu
PART = 2**14  # rows that the tensor cores add up without a rounding to nearest


@pytest.mark.parametrize("m,n,k", [(2**20 + 5, 64, 64), (2**17 + 77, 384, 512), (66000, 100, 5000), (2**17, 1024, 2048), (70000, 700, 300), (2**16 + 1, 8, 8),
                                   (2**21, 40, 9), (65600, 16400, 8)])
@pytest.mark.parametrize("dtype,signs", [("f16", False), ("bf16", True)])
def test_sums_over_many_rows(m, n, k, dtype, signs):
    """Every unit's gate and up weights pick one feature, features and gradients have five bits, no activation: G = U = x, and dG = dU = dh x has ten
    bits, exact in fp32 and fp16; in bf16 (eight bits) it is rounded once, to nearest, which is done here too. What is left is the sum over the rows and one rounding.

    A part's sum is truncated once in 16 rows, by a step of fp32 (2^-23) of what it holds, and the 16 products beside it lose as much together: 2^-22 (2^14 /
    16 + 8) of the sum of the absolute values. The parts, one after the other: 2^-24 each."""
    b, t = mfet(), ref.DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(m)

    def five_bits(rows, cols, unit):
        v = torch.randint(1, 32, (rows, cols), generator=g, device="cuda", dtype=torch.int16).to(t) * unit
        return v * (torch.randint(0, 2, (rows, cols), generator=g, device="cuda", dtype=torch.int16) * 2 - 1).to(t) if signs else v
    x, dh = five_bits(m, k, 1 / 16), five_bits(m, n, 2.0**-11)
    pick = torch.arange(n, device="cuda") % k
    wg, wu = (torch.zeros(n, k, dtype=t, device="cuda") for _ in range(2))
    wg[range(n), pick] = wu[range(n), pick] = 1.0
    dx = torch.empty_like(x)
    dwg, dwu = (torch.full((n, k), 7.0, dtype=t, device="cuda") for _ in range(2))
    ws = torch.full((b.mfet_gated_linear_backward_bytes(m, n, k),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = []
    for _ in range(2):
        b.mfet_gated_linear_backward(x, b.dtype_of(x), k, m, wg, k, wu, k, n, k, b.ACT_NONE, dh, n, dx, k, dwg, k, dwu, k, ws, ws.numel(), status,
                                     torch.cuda.current_stream().cuda_stream)
        out.append((dwg.clone(), dwu.clone()))
    assert int(status.item()) == 0 and all(torch.equal(p, q) for p, q in zip(*out))
    want, size = torch.zeros(n, k, dtype=torch.float64, device="cuda"), torch.zeros(n, k, dtype=torch.float64, device="cuda")
    for i in range(0, m, 2**16):
        xs = x[i:i + 2**16].double()
        d = (dh[i:i + 2**16].double() * xs[:, pick]).to(t).double()
        want += d.T @ xs
        size += d.abs().T @ xs.abs()
        wide = torch.zeros_like(xs).index_add_(1, pick, 2 * d)
        far = torch.zeros_like(xs).index_add_(1, pick, 2 * d.abs()) * (2 * n / 16 + 8) * 2.0**-22
        assert ref.within(dx[i:i + 2**16], wide, far + ref.rounding(wide.abs() + far, t))
    bound = size * ((PART / 16 + 8) * 2.0**-22 + (m / PART + 4) * 2.0**-24)
    bound = bound + ref.rounding(want.abs() + bound, t)
    assert ref.within(dwg, want, bound) and ref.within(dwu, want, bound)
