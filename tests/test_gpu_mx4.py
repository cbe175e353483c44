"""MXFP4 operands and their product against the 64-bit definition.

Codes and scale bytes are bit-exact. A product of two codes under their scales is exact, so y differs from the 64-bit result by the
rounding of fp32 sums alone. At worst every partial sum of 32 products loses a unit in the last place of the largest partial
sum there can be, the sum of all magnitudes: |err| <= (k / 32 + 8) * 2^-23 * sum |a| |w|, plus 2^-23 of the result for the bias
addition. A 16-bit y has to lie between the roundings of that interval's two ends."""
import numpy as np
import pytest
import torch

from tests import lowbit_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": 0, "f16": 1, "bf16": 2}


def stream():
    return torch.cuda.current_stream().cuda_stream


def features(rng, m, k, dtype):
    x = (rng.standard_normal((m, k)) * 0.04).astype(np.float32)
    x[2:: 5] *= 50.0
    x[1:: 9, : k // 2] = 0.0
    return torch.from_numpy(x).to(DTYPES[dtype]).cuda()


def operand(x64):
    codes, scales, vals = ref.mx4_operand(x64)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), vals


def check(y, a, w, bias, relu):
    k = a.shape[1]
    full = a @ w.T + (0.0 if bias is None else bias)
    mass = np.abs(a) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    want = np.maximum(full, 0) if relu else full
    assert ref.within(y, want, (k / 32 + 8) * 2.0**-23 * mass + 2.0**-23 * np.abs(want))


def padded(x, pad, shift, fill):
    n, k = x.shape
    buf = torch.full((n * (k + pad) + shift + 8,), fill, dtype=x.dtype, device="cuda")
    view = buf[shift:shift + n * (k + pad)].view(n, k + pad)
    view[:, :k] = x
    return buf, view


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 32), (3, 33), (128, 128), (129, 100), (130, 1075), (500, 896), (7, 2048)])
def test_quantise_is_bit_exact(rows, k, dtype):
    m = mfet()
    x = features(np.random.default_rng(rows + k), rows, k, dtype)
    for pad, shift in ((0, 0), (3, 1), (-k % 8 + 8, 0)):
        _, view = padded(x, pad, shift, 99.0)
        codes = torch.full((m.mfet_mx4_code_bytes(rows, k) + 16,), 0xAB, dtype=torch.uint8, device="cuda")
        scales = torch.full((m.mfet_mx4_scale_bytes(rows, k) + 16,), 0xAB, dtype=torch.uint8, device="cuda")
        m.mfet_mx4_quantize(view, CODE[dtype], k + pad, rows, k, codes, scales, stream())
        want_c, want_s, _ = ref.mx4_operand(x.double().cpu().numpy())
        assert np.array_equal(codes[:-16].cpu().numpy(), want_c.reshape(-1))
        blocks = -(-k // 32)
        got = ref.untile_scales(scales[:-16].cpu().numpy(), rows, blocks + -blocks % 4)
        assert np.array_equal(got, ref.untile_scales(want_s, rows, blocks + -blocks % 4))  # with the zeros behind the last block
        assert (codes[-16:] == 0xAB).all() and (scales[-16:] == 0xAB).all()


SHAPES = [(1, 1, 1), (1, 16, 32), (9, 128, 64), (32, 128, 256), (33, 127, 65), (64, 129, 127), (65, 1, 128), (100, 300, 129),
          (128, 128, 192), (129, 256, 255), (500, 777, 1075), (200, 64, 257), (640, 1000, 896), (1000, 130, 2048), (17, 2048, 31),
          (300, 96, 4100),
          # enough tiles for pairs of blocks: odd rows, columns and depths, a second block without rows
          (2305, 1030, 257), (1300, 2000, 1000), (5000, 640, 129), (2561, 1000, 2048), (9345, 300, 33), (130, 9500, 700)]


@pytest.mark.parametrize("m_,n,k", SHAPES)
def test_product(m_, n, k):
    m = mfet()
    rng = np.random.default_rng(m_ * 7 + n * 3 + k)
    ac, asc, a = operand(features(rng, m_, k, "f32").double().cpu().numpy())
    wc, wsc, w = operand(rng.standard_normal((n, k)) / np.sqrt(k))
    bias = rng.standard_normal(n).astype(np.float32)
    for ytype, pad, act, b in (("f32", 0, 0, None), ("bf16", 5, 1, bias), ("f16", 1, 0, bias)):
        buf, y = padded(torch.full((m_, n), 3.0, dtype=DTYPES[ytype], device="cuda"), pad, 1, 3.0)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        d_b = None if b is None else torch.from_numpy(b).cuda()
        m.mfet_mx4_matmul(ac, asc, m_, wc, wsc, n, k, d_b, act, y, CODE[ytype], n + pad, status, stream())
        assert int(status.item()) == 0
        check(y[:, :n], a, w, b, act == 1)
        y[:, :n] = 3.0
        assert (buf == 3.0).all()  # nothing between the rows or beyond them


@pytest.mark.parametrize("m_", [1, 2, 3, 4, 5, 7, 8, 9, 31, 200])
@pytest.mark.parametrize("n,k,xtype,ytype", [(1024, 896, "f32", "f32"), (1000, 2048, "bf16", "bf16"), (77, 1075, "f16", "f32"),
                                             (1, 1, "f32", "f16"), (9, 33, "bf16", "f32"), (130, 1025, "f32", "f32")])
def test_linear(m_, n, k, xtype, ytype):
    m = mfet()
    rng = np.random.default_rng(m_ * 11 + n + k)
    x = features(rng, m_, k, xtype)
    wc, wsc, w = operand(rng.standard_normal((n, k)) / np.sqrt(k))
    bias = rng.standard_normal(n).astype(np.float32)
    a = ref.mx4_operand(x.double().cpu().numpy())[2]
    for pad, shift, act, b in ((0, 0, 1, bias), (5, 1, 0, None), (8, 0, 0, bias)):
        _, view = padded(x, pad, shift, 99.0)
        buf, y = padded(torch.full((m_, n), 3.0, dtype=DTYPES[ytype], device="cuda"), pad, shift, 3.0)
        nbytes = m.mfet_mx4_linear_bytes(m_, k)
        scratch = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        d_b = None if b is None else torch.from_numpy(b).cuda()
        m.mfet_mx4_linear(view, CODE[xtype], k + pad, m_, wc, wsc, n, k, d_b, act, y, CODE[ytype], n + pad, scratch, nbytes, status,
                          stream())
        assert int(status.item()) == 0
        check(y[:, :n], a, w, b, act == 1)
        y[:, :n] = 3.0
        assert (buf == 3.0).all()


@pytest.mark.parametrize("m_", [3, 40, 300])
def test_nan_blocks_reach_their_row_and_column_alone(m_):
    m = mfet()
    rng = np.random.default_rng(m_)
    n, k = 200, 300
    x = features(rng, m_, k, "f32")
    x[1, 290], x[2, 0] = float("nan"), float("inf")
    w = rng.standard_normal((n, k)) / np.sqrt(k)
    w[150, 64] = np.inf
    wc, wsc, wv = operand(w)
    y = torch.zeros(m_, n, device="cuda")
    nbytes = m.mfet_mx4_linear_bytes(m_, k)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    m.mfet_mx4_linear(x, 0, k, m_, wc, wsc, n, k, None, 1, y, 0, n, scratch, nbytes, None, stream())
    nan = np.zeros((m_, n), bool)
    nan[1:3] = True
    nan[:, 150] = True
    assert np.array_equal(np.isnan(y.cpu().numpy()), nan)  # through the ReLU as well


def test_repeated_calls_give_equal_bits_and_another_stream():
    m = mfet()
    rng = np.random.default_rng(0)
    n, k = 1024, 896
    wc, wsc, _ = operand(rng.standard_normal((n, k)) / np.sqrt(k))
    for m_ in (5, 3000):
        x = features(rng, m_, k, "f32")
        nbytes = m.mfet_mx4_linear_bytes(m_, k)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        ys = []
        for s in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.current_stream()):
            torch.cuda.synchronize()
            y = torch.zeros(m_, n, device="cuda")
            torch.cuda.synchronize()
            for _ in range(4):  # back to back on the same scratch
                m.mfet_mx4_linear(x, 0, k, m_, wc, wsc, n, k, None, 0, y, 0, n, scratch, nbytes, None, s.cuda_stream)
            s.synchronize()
            ys.append(y)
        assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


def test_few_rows_beyond_the_one_launch_forms_work():
    """The largest product that one launch takes, and the next larger ones that go through the scratch."""
    m = mfet()
    rng = np.random.default_rng(77)
    for m_, n, k in ((8, 4096, 1024), (8, 4100, 1024), (3, 9000, 1000), (1, 40000, 900)):
        x = features(rng, m_, k, "f32")
        wc, wsc, w = operand(rng.standard_normal((n, k)) / np.sqrt(k))
        y = torch.zeros(m_, n, device="cuda")
        nbytes = m.mfet_mx4_linear_bytes(m_, k)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        m.mfet_mx4_linear(x, 0, k, m_, wc, wsc, n, k, None, 0, y, 0, n, scratch, nbytes, None, stream())
        check(y, ref.mx4_operand(x.double().cpu().numpy())[2], w, None, False)
