"""The one-launch linear layer from several threads and with long rows, and operands near the ends of the format.

Tolerance of test_gpu_mx4.py: |err| <= (k / 32 + 8) * 2^-23 * sum |a| |w|."""
import threading

import numpy as np
import pytest
import torch

from tests import lowbit_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu


def operand(x64):
    codes, scales, vals = ref.mx4_operand(x64)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), vals


def check(y, a, w):
    assert ref.within(y, a @ w.T, (a.shape[1] / 32 + 8) * 2.0**-23 * (np.abs(a) @ np.abs(w).T))


class Linear:
    def __init__(self, rng, m_, n, k, x_size=0.04, w_size=None):
        m = mfet()
        self.args = (m_, n, k)
        x = np.clip(rng.standard_normal((m_, k)), -1.5, 1.5) * x_size
        w = np.clip(rng.standard_normal((n, k)), -1.5, 1.5) * (k**-0.5 if w_size is None else w_size)
        self.x = torch.from_numpy(x.astype(np.float32)).cuda()
        self.wc, self.ws, self.w = operand(w.astype(np.float32).astype(np.float64))
        self.a = ref.mx4_operand(self.x.double().cpu().numpy())[2]
        self.y = torch.zeros(m_, n, device="cuda")
        self.scratch = torch.empty(m.mfet_mx4_linear_bytes(m_, k), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def __call__(self, stream=None):
        m_, n, k = self.args
        s = torch.cuda.current_stream() if stream is None else stream
        mfet().mfet_mx4_linear(self.x, 0, k, m_, self.wc, self.ws, n, k, None, 0, self.y, 0, n, self.scratch, self.scratch.numel(),
                               self.status, s.cuda_stream)
        return self.y


@pytest.mark.parametrize("m_,k", [(8, 5200), (8, 7777), (5, 10_000), (4, 20_000), (1, 80_000), (8, 10_400)])
def test_few_long_rows(m_, k):
    call = Linear(np.random.default_rng(k), m_, 33, k)
    check(call(), call.a, call.w)
    assert int(call.status.item()) == 0


def test_threads_with_rows_of_different_lengths():
    """Every thread's launch has the shared memory that its own rows need."""
    rng = np.random.default_rng(1)
    calls = [Linear(rng, 8, 16, k) for k in (5200, 6400, 8000, 10_000)]
    want = [c().clone() for c in calls]
    torch.cuda.synchronize()
    errors = []

    def work(c):
        s = torch.cuda.Stream()
        try:
            for _ in range(1500):
                c(s)
            s.synchronize()
        except Exception as e:  # handed to the test's own thread
            errors.append(e)

    for c in calls:
        c.y.zero_()
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors[0]
    assert all(torch.equal(c.y, w) for c, w in zip(calls, want))


@pytest.mark.parametrize("m_", [1, 2, 3, 8, 9, 200])
@pytest.mark.parametrize("x_size,w_size", [(1e-30, 2e38), (2e38, 1e-30), (1e-38, 2e38), (2e38, 1e-38), (1e-20, 1e-15)])
def test_products_of_large_and_small_operands(m_, x_size, w_size):
    """Every product and sum is far inside fp32's range, although one factor is not."""
    call = Linear(np.random.default_rng(m_), m_, 70, 300, x_size, w_size)
    check(call(), call.a, call.w)
