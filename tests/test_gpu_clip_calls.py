"""Gradient clipping in the forms of a training step: next to other work, in place, the norm alone, constant and extreme values.

Tolerances as in test_gpu_grad_clip.py: the norm is its fp64 value rounded to fp32 (1e-7 relative), an fp32 gradient is g times the fp32
coefficient (1.3e-7 relative, 1e-45 absolute), a 16-bit one that product rounded once more."""
import math

import numpy as np
import pytest
import torch

from tests.helpers import mfet
from tests.lowbit_reference import within

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
REL, ABS = 1.3e-7, 1e-45


class Clip:
    """One list of gradients with its buffers."""

    def __init__(self, src, dst, counts=None):
        m = mfet()
        self.grads = m.make_grads(src, dst, counts)
        self.scratch = torch.full((m.mfet_grad_clip_bytes(len(src)),), 0xFF, dtype=torch.uint8, device="cuda")
        self.norm = torch.full((1,), -1.0, device="cuda")

    def __call__(self, max_norm, stream=None):
        s = torch.cuda.current_stream() if stream is None else stream
        mfet().mfet_grad_clip(self.grads, max_norm, self.norm, self.scratch, self.scratch.numel(), s.cuda_stream)
        return self.norm


def f64(t):
    return t.double().cpu().numpy()


def test_one_launch_calls_next_to_a_busy_stream():
    """The blocks of the one-launch form's cluster start when the SMs have room: results are those of a quiet GPU."""
    torch.manual_seed(0)
    xs = [torch.randn(n, device="cuda") * 0.01 for n in (5, 4000, 65536, 120_000)]
    ys = [torch.empty_like(x) for x in xs]
    calls = [Clip([x], [y]) for x, y in zip(xs, ys)]
    quiet = []
    for c, y in zip(calls, ys):
        c(0.05)
        quiet.append((c.norm.clone(), y.clone()))
    torch.cuda.synchronize()
    a = torch.randn(4096, 4096, device="cuda").bfloat16()
    busy, s = torch.cuda.Stream(), torch.cuda.Stream()
    for rep in range(100):
        with torch.cuda.stream(busy):
            a @ a
        for c, y in zip(calls, ys):
            with torch.cuda.stream(s):
                y.zero_()
            c(0.05, s)
        if rep % 10 == 9:
            s.synchronize()
            assert all(torch.equal(c.norm, n) and torch.equal(y, q) for c, y, (n, q) in zip(calls, ys, quiet))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 4096, 131_071, 400_003])
def test_in_place_above_and_below_the_limit(n, dtype):
    torch.manual_seed(n)
    keep = (torch.randn(n + 3, device="cuda") * 0.01).to(DTYPES[dtype])
    for shift in (0, 1):
        x = keep.clone()
        v = x[shift:shift + n]
        total = math.sqrt(math.fsum(np.square(f64(v)).tolist()))
        for limit in (total / 3, total * 3):
            v.copy_(keep[shift:shift + n])
            got = float(Clip([v], [v])(limit).item())
            assert abs(got - total) <= 1e-7 * total
            want = f64(keep[shift:shift + n]) * min(1.0, float(np.float32(limit)) / total)
            assert within(v, want, ABS + REL * np.abs(want))
            assert torch.equal(x[:shift], keep[:shift]) and torch.equal(x[shift + n:], keep[shift + n:])


def device_us(call, reps=20):
    for _ in range(3):
        call()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(reps):
        call()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) * 1e3 / reps


def test_the_norm_alone_costs_one_pass():
    """It reads every gradient once; clipping reads twice and writes once."""
    x = torch.randn(150_000_000, device="cuda", dtype=torch.bfloat16)
    y = torch.empty_like(x)
    full, norm = Clip([x], [y]), Clip([x], [None])
    full(0.1)
    norm(0.1)
    assert torch.equal(full.norm, norm.norm)
    assert device_us(lambda: norm(0.1)) < 0.75 * device_us(lambda: full(0.1))


@pytest.mark.parametrize("dtype,value", [("f16", 0.01398468), ("bf16", 0.0123), ("f32", 0.1), ("f32", 0.013984681), ("f16", 3e-7), ("f32", 7e-23)])
@pytest.mark.parametrize("n", [8000, 300_007, 5_000_000])
def test_equal_values_do_not_add_up_their_roundings(n, dtype, value):
    x = torch.full((n,), value, device="cuda").to(DTYPES[dtype])
    total = float(x[:1].double().item()) * math.sqrt(n)
    got = float(Clip([x], [None])(1.0).item())
    assert abs(got - total) <= 1e-7 * total


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("limit", [1.0, 1e-10, 1e-30])
def test_coefficients_below_fp32(dtype, limit):
    """Gradients near the largest values: the coefficient has no normal fp32 value, g * coef has."""
    torch.manual_seed(5)
    x = (torch.randn(20_000, device="cuda", dtype=torch.float64).clamp(-3, 3) * 1e38).float().to(DTYPES[dtype])
    y = torch.empty_like(x)
    total = math.sqrt(math.fsum(np.square(f64(x)).tolist()))
    Clip([x], [y])(limit)
    want = f64(x) * (float(np.float32(limit)) / total)
    assert within(y, want, ABS + REL * np.abs(want))


def test_more_than_2_to_the_32_elements():
    n = 2**32 + 100_003
    x = torch.full((n,), 0.01, device="cuda", dtype=torch.bfloat16)
    x[-5:] = 100.0
    v = float(x[0].double().item())
    total = math.sqrt((n - 5) * v * v + 5 * 100.0**2)
    c = Clip([x], [x])
    c(total / 4)  # in place, by a power of two
    assert abs(float(c.norm.item()) - total) <= 1e-7 * total
    assert float(x[-1].item()) == 25.0 and float(x[0].double().item()) == v / 4 and bool((x[:-5] == x[0]).all())
