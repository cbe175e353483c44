"""The slopes of the activations, unit by unit: every gradient is one product, so that nothing hides what a slope is off by."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu


def slope(act, g):
    s, c = torch.sigmoid(g), torch.sigmoid(-g)
    return s * c if act == "sigmoid" else s * (1 + g * c)


@pytest.mark.parametrize("m", [128, 9000])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_slopes_of_saturated_gates(dtype, act, m):
    """Unit j has the gate g_j (exact in its type) and the up value 1; row j alone has a gradient, 4096 of unit j. So dw_gate[j] is 4096 times the slope at
    g_j, rounded to the type as dG, and dx[j] is that times the unit's gate weight (one product, one more rounding).

    e^-g is off by 2^-22 of itself and by the rounding of its argument, 20 / ln 2 * 2^-24 * ln 2 = 2^-19.7; the quotient by 2^-22, the products by 2^-24
    each: 2^-18 together. silu's slope has a zero at -1.28: there the same is meant of 1 + |g|, not of the sum."""
    t, n, k = ref.DT[dtype], 128, 16
    b = mfet()
    g = torch.cat([torch.linspace(-20, 20, 96), torch.linspace(8, 18, 32)]).to("cuda", t)
    x, wg, wu = (torch.zeros(r, k, dtype=t, device="cuda") for r in (m, n, n))
    x[:, 0], wg[:, 0], wu[:, 1] = 1.0, g, 1.0
    x[:, 1] = 1.0
    dh = torch.zeros(m, n, dtype=t, device="cuda")
    dh[range(n), range(n)] = 4096.0
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    ws = torch.full((b.mfet_gated_linear_backward_bytes(m, n, k),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.mfet_gated_linear_backward(x, b.dtype_of(x), k, m, wg, k, wu, k, n, k, b.ACT_SIGMOID if act == "sigmoid" else b.ACT_SILU, dh, n, dx, k, dwg, k,
                                 dwu, k, ws, ws.numel(), status, torch.cuda.current_stream().cuda_stream)
    v = g.double()
    s = torch.sigmoid(v)
    size = slope(act, v).abs() if act == "sigmoid" else s * (1 + v.abs() * torch.sigmoid(-v))
    want, bound = 4096 * slope(act, v), 4096 * size * 2.0**-18
    bound = bound + ref.rounding(want.abs() + bound, t)
    assert ref.within(dwg[:, 0], want, bound)
    a = s if act == "sigmoid" else v * s
    want, wide = 4096 * a, 4096 * a.abs() * 2.0**-18
    # silu's value at 16 and more times 4096 is beyond fp16's last step (65504 + 16): its rounding is an infinity, which is what is wanted there
    want = torch.where(torch.isinf(want.to(t)), want.to(t).double(), want)
    assert ref.within(dwu[:, 0], want, wide + ref.rounding(4096 * a.abs() + wide, t))
    assert int(status.item()) == 0
