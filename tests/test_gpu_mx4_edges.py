"""The MXFP4 product at the edges of its result, and from a thread that has not used the GPU before."""
import threading

import numpy as np
import pytest
import torch

from tests import lowbit_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu


def operands(m_, n, k):
    rng = np.random.default_rng(n)
    out = []
    for rows in (m_, n):
        codes, scales, vals = ref.mx4_operand(rng.standard_normal((rows, k)))
        out.append((torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), vals))
    return out


def matmul(x, w, m_, n, k, y, stream):
    mfet().mfet_mx4_matmul(x[0], x[1], m_, w[0], w[1], n, k, None, 0, y, mfet().dtype_of(y), y.stride(0), None, stream)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,ld", [(1001, 1008), (1001, 1016), (62, 64), (33, 40), (128, 136), (1, 8)])
def test_what_lies_between_rows_is_not_written(dtype, n, ld):
    x, w = operands(150, n, 96)
    y = torch.full((150, ld), 7.0, device="cuda").to(dtype)
    matmul(x, w, 150, n, 96, y, torch.cuda.current_stream().cuda_stream)
    want = x[2] @ w[2].T
    half = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}[dtype]
    assert ref.within(y[:, :n], want, (96 / 32 + 8) * 2.0**-23 * (np.abs(x[2]) @ np.abs(w[2]).T) + half * np.abs(want))
    assert bool((y[:, n:] == 7.0).all())


def test_first_call_of_a_thread():
    x, w = operands(150, 64, 96)
    y = torch.zeros(150, 64, device="cuda")
    torch.cuda.synchronize()
    errors = []

    def work():
        try:
            matmul(x, w, 150, 64, 96, y, None)
        except Exception as e:  # handed to the test's own thread
            errors.append(e)
    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not errors, errors[0]
    want = x[2] @ w[2].T
    assert ref.within(y, want, (96 / 32 + 8) * 2.0**-23 * (np.abs(x[2]) @ np.abs(w[2]).T))
