"""Global gradient norm and clipping against the 64-bit formula.

Tolerances: squares and sums are fp64, so the norm's only error of note is its rounding to fp32 (2^-24 relative; 1e-7 allowed).
A clipped fp32 element is g * fp32(coef): two roundings, 2^-23 relative (1.2e-7; 1.3e-7 allowed, plus 1e-45 for subnormal
results). A 16-bit element is that product rounded once more: it has to lie between the roundings of the two ends of the fp32 interval."""
import math

import numpy as np
import pytest
import torch

from tests.helpers import mfet
from tests.lowbit_reference import within

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
REL, ABS = 1.3e-7, 1e-45


def stream():
    return torch.cuda.current_stream().cuda_stream


def clip(src, dst, max_norm, counts=None):
    m = mfet()
    g = m.make_grads(src, dst, counts)
    nbytes = m.mfet_grad_clip_bytes(len(src))
    scratch = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")  # needs no initialisation
    norm = torch.full((1,), -1.0, device="cuda")
    m.mfet_grad_clip(g, max_norm, norm, scratch, nbytes, stream())
    return float(norm.item())


def reference(tensors, max_norm):
    total = math.sqrt(math.fsum(float(np.square(t).sum()) for t in tensors))
    return total, (max_norm / total if total > max_norm else 1.0)


def check(got, want64):
    assert within(got, want64, ABS + REL * np.abs(want64))


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("sizes", [[1], [3, 1, 5], [8192], [8191, 8193, 16384, 16385], [100_003, 7, 40_000], [3_000_001]])
def test_dense_tensors_at_any_address(dtype, sizes):
    """The tensors lie one behind the other, so that most of them start at odd addresses."""
    torch.manual_seed(sum(sizes))
    flat = (torch.randn(sum(sizes) + 3, device="cuda") * 0.01).to(DTYPES[dtype])
    for shift in (0, 1, 3):
        views = list(flat[shift:shift + sum(sizes)].split(sizes))
        total, coef = reference([f64(v) for v in views], 0.005)
        for out_shift in (shift, (shift + 1) % 4):
            out = torch.full((sum(sizes) + 8,), 5.0, dtype=flat.dtype, device="cuda")
            dst = list(out[out_shift:out_shift + sum(sizes)].split(sizes))
            assert abs(clip(views, dst, 0.005) - total) <= 1e-7 * total
            for v, d in zip(views, dst):
                check(d, f64(v) * coef)
            assert (out[:out_shift] == 5).all() and (out[out_shift + sum(sizes):] == 5).all()


def test_in_place_mixed_types_and_tensors_that_only_count():
    torch.manual_seed(1)
    src = [torch.randn(1000, 33, device="cuda"), (torch.randn(64, 128, device="cuda")).half(), torch.randn(7, device="cuda").bfloat16(),
           torch.randn(5000, device="cuda")]
    keep = [f64(t) for t in src]
    total, coef = reference(keep, 3.0)
    got = clip(src, src[:3] + [None], 3.0)
    assert abs(got - total) <= 1e-7 * total and coef < 1
    for t, k in zip(src[:3], keep):
        check(t, k * coef)
    assert np.array_equal(f64(src[3]), keep[3])
    keep = [f64(t) for t in src]
    clip(src, src, 1e9)  # below the limit: nothing changes
    assert all(np.array_equal(f64(t), k) for t, k in zip(src, keep))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_with_counts_on_the_device(dtype):
    torch.manual_seed(2)
    caps, dims = [4000, 100, 1, 2500, 30], [32, 136, 8, 72, 1]
    counts = torch.tensor([1234, 0, 1, 9999, -5], dtype=torch.int64, device="cuda")
    used = [1234, 0, 1, 2500, 0]
    src = [(torch.randn(c, d, device="cuda") * 0.01).to(DTYPES[dtype]) for c, d in zip(caps, dims)]
    for s, u in zip(src, used):
        s[u:] = float("nan")  # what lies beyond the count is not read
    dst = [torch.full_like(s, 4.0) for s in src]
    total, coef = reference([f64(s[:u]) for s, u in zip(src, used)], 0.1)
    assert abs(clip(src, dst, 0.1, counts) - total) <= 1e-7 * total
    for s, d, u in zip(src, dst, used):
        check(d[:u], f64(s[:u]) * coef)
        assert (d[u:] == 4.0).all()


@pytest.mark.parametrize("cols,ld", [(1, 3), (5, 6), (33, 64), (128, 136)])
def test_rows_apart(cols, ld):
    torch.manual_seed(3)
    buf = torch.randn(700, ld, device="cuda")
    keep = f64(buf)
    src = buf[:, :cols]
    total, coef = reference([keep[:, :cols]], 2.0)
    assert abs(clip([src], [src], 2.0) - total) <= 1e-7 * total
    check(buf[:, :cols], keep[:, :cols] * coef)
    assert np.array_equal(f64(buf[:, cols:]), keep[:, cols:])


@pytest.mark.parametrize("n", [47, 48, 49, 448, 449, 1000])
def test_many_tensors(n):
    rng = np.random.default_rng(n)
    sizes = [int(v) for v in rng.integers(0, 300, n)]
    flat = torch.randn(sum(sizes), device="cuda")
    out = torch.zeros_like(flat)
    total, coef = reference([f64(flat)], 1.5)
    assert abs(clip(list(flat.split(sizes)), list(out.split(sizes)), 1.5) - total) <= 1e-7 * total
    check(out, f64(flat) * coef)
    assert abs(clip(list(flat.split(sizes)), [None] * n, 1.5) - total) <= 1e-7 * total  # the norm alone
    last_only = [None] * (n - 1) + [out[:sizes[-1]]]
    out.zero_()
    assert abs(clip(list(flat.split(sizes)), last_only, 1.5) - total) <= 1e-7 * total
    check(out[:sizes[-1]], f64(flat[sum(sizes) - sizes[-1]:]) * coef)


def test_no_tensors_empty_tensors_and_the_limits_ends():
    x = torch.randn(100, device="cuda")
    assert clip([], [], 1.0) == 0.0
    assert clip([x[:0]], [x[:0]], 1.0) == 0.0
    y = torch.empty_like(x)
    n = float(np.float32(np.linalg.norm(f64(x))))
    assert abs(clip([x], [y], math.inf) - n) <= 2e-7 * n and torch.equal(x, y)
    clip([x], [y], 0.0)
    assert (y == 0).all()
    z = torch.zeros(100, device="cuda")
    assert clip([z], [y], 0.0) == 0.0 and (y == 0).all()


@pytest.mark.parametrize("size", [1e30, 1e-30, 3e38, 1e-44])
def test_squares_outside_fp32(size):
    x = (torch.randn(5000, device="cuda", dtype=torch.float64).clamp(-1, 1) * size).float()
    total, _ = reference([f64(x)], 1.0)
    y = torch.empty_like(x)
    with np.errstate(over="ignore"):
        limit = float(np.float32(total / 4))  # no fp32 value for the largest size: no limit then
    got = clip([x], [y], limit)
    if total < 3.4e38:
        assert abs(got - total) <= 1e-7 * total + 1e-45
    else:
        assert got == math.inf  # the norm itself has no fp32 value; the gradients are clipped all the same
    if size > 1e-40:
        check(y, f64(x) * min(1.0, limit / total))


def test_nan_and_infinity_pass_through():
    for bad in (float("nan"), float("inf"), float("-inf")):
        x = torch.randn(40_000, device="cuda")
        x[12345] = bad
        y = torch.zeros_like(x)
        n = clip([x], [y], 1.0)
        assert math.isnan(n) if math.isnan(bad) else n == math.inf
        assert torch.equal(x.view(torch.int32), y.view(torch.int32))


def test_equal_inputs_give_equal_bits_and_two_streams():
    m = mfet()
    x = torch.randn(2_000_000, device="cuda")
    outs = []
    for _ in range(3):
        y = torch.empty_like(x)
        n = clip([x], [y], 1.0)
        outs.append((n, y))
    assert all(o[0] == outs[0][0] and torch.equal(o[1], outs[0][1]) for o in outs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, norm = torch.empty_like(x), torch.zeros(1, device="cuda")
    nb = m.mfet_grad_clip_bytes(1)
    scratch = torch.empty(nb, dtype=torch.uint8, device="cuda")
    m.mfet_grad_clip(m.make_grads([x], [y]), 1.0, norm, scratch, nb, s.cuda_stream)
    s.synchronize()
    assert torch.equal(y, outs[0][1])
