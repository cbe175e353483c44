"""The orthogonalised update with schedules whose polynomials have their largest value inside the range of the singular values: what bounds an iterate
decides under which power of two its fp16 words are kept, and which schedules are refused."""
import pytest
import torch

from tests import block_reference as ref
from tests.helpers import mfet

SMALL = [0.0, 1e-20, -1e-20, 1e-12, 1e-7, 1e-3]  # the fifth power's coefficient beside a cubic that turns inside the range


@pytest.mark.parametrize("c", SMALL)
def test_a_schedule_that_grows_inside_its_range_is_refused(c):
    """Step 1 takes 1 to 100. Step 2 has 1e5 * 100 * (1 - 100^2 / (3 * 60^2)) = 0.7e6 at 100, below 2^20, but 2 / 3 * 1e5 * 60 = 4e6 at 60 (the fifth
    power changes either by less than a hundredth of itself for the coefficients up to 1e-7, and only adds for 1e-3)."""
    m = mfet()
    with pytest.raises(m.MfetError) as e:
        m.mfet_orthogonalize(None, m.F32, 5, 0, 5, [[100.0, 0.0, 0.0], [1e5, -1e5 / (3 * 3600), c]], 2, 1.0, None, m.F32, 5, None, 0)
    assert e.value.status == m.ERR_INVALID_ARG
    # twenty times less grows to 2e5 (c = 1e-3, 100^5 = 1e10 times that, stays beyond)
    if c < 1e-3:
        m.mfet_orthogonalize(None, m.F32, 5, 0, 5, [[100.0, 0.0, 0.0], [5e3, -5e3 / (3 * 3600), c]], 2, 1.0, None, m.F32, 5, None, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [3, 130])
@pytest.mark.parametrize("c", SMALL)
def test_an_iterate_that_is_largest_inside_the_range(c, d):
    """Singular values of at most sqrt(3) after the first step, and of 1 where the matrix has three equal ones: step 2's cubic has its largest value, 1, at 1
    and is 0 at sqrt(3)."""
    m = mfet()
    schedule = [[3.0**0.5, 0.0, 0.0], [1.5, -0.5, c], [1.0, 0.0, 0.0]]
    g = torch.zeros(d, d, device="cuda")
    g[0, 0] = g[1, 1] = g[2, 2] = 0.25
    out = torch.empty(d, d, device="cuda")
    ws = torch.full((m.mfet_orthogonalize_bytes(d, d),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    m.mfet_orthogonalize(g, m.F32, d, d, d, schedule, 3, 1.0, out, m.F32, d, ws, ws.numel(), status, torch.cuda.current_stream().cuda_stream)
    steps = [tuple(torch.tensor(v, dtype=torch.float32).tolist()) for v in schedule]
    want = ref.orthogonalize(g.double(), steps)
    off = float(torch.linalg.vector_norm(out.double() - want))
    assert off <= ref.orthogonalize_bound(want, g, steps, 1.0, out.dtype)
    assert int(status.item()) == 0
