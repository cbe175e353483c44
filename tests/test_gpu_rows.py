"""Rows written into a table in its format and read back: bit-exact against the 64-bit definition."""
import numpy as np
import pytest
import torch

from tests import lowbit_reference as ref
from tests.helpers import mfet

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": 0, "f16": 1, "bf16": 2}


def values(rng, n, dim, dtype):
    x = (rng.standard_normal((n, dim)) * 0.01).astype(np.float32)
    if n:
        x[:: 7] *= 300.0
        x[3:: 11] = 0.0
    return torch.from_numpy(x).to(DTYPES[dtype]).cuda()


def stream():
    return torch.cuda.current_stream().cuda_stream


def desc(m, table, rows, dim, dtype, stride=0):
    return m.TableDesc(table.data_ptr(), rows, dim, dtype, m.LOC_DEVICE, 0, 0, stride)


def strided_copy(x, pad, shift):
    """x with `pad` elements between rows, its first element `shift` elements off the allocation's start."""
    n, dim = x.shape
    buf = torch.full((n * (dim + pad) + shift + 8,), 7.0, dtype=x.dtype, device="cuda")
    view = buf[shift:shift + n * (dim + pad)].view(n, dim + pad)
    view[:, :dim] = x
    return buf, view


@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [8, 24, 32, 40, 64, 72, 128, 136, 256, 264, 520])
def test_mxfp4_rows_are_bit_exact(dim, src):
    m = mfet()
    rng = np.random.default_rng(dim)
    for n, pad, shift, extra in ((1, 0, 0, 0), (5, 3, 1, 16), (333, 8, 0, 0), (1000, 0, 0, 32)):
        rows, rb = 2 * n + 3, m.row_bytes(dim, m.MXFP4)
        assert rb == ref.mx4_row_bytes(dim)
        stride = rb + extra
        table = torch.full((rows, stride), 0xAB, dtype=torch.uint8, device="cuda")
        d = desc(m, table, rows, dim, m.MXFP4, stride if extra else 0)
        x = values(rng, n, dim, src)
        at = torch.from_numpy(rng.permutation(rows)[:n]).cuda()
        _, view = strided_copy(x, pad, shift)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        m.mfet_rows_write(d, at, n, None, view, CODE[src], dim + pad, status, stream())
        want = np.full((rows, stride), 0xAB, np.uint8)
        want[at.cpu().numpy(), :rb] = ref.mx4_rows(x.double().cpu().numpy())
        assert np.array_equal(table.cpu().numpy(), want)
        for out in ("f32", "bf16", "f16"):
            back = torch.cat((at, torch.tensor([-1, at[0].item()], device="cuda")))
            buf, got = strided_copy(torch.full((n + 2, dim), 3.0, dtype=DTYPES[out], device="cuda"), pad, shift)
            keep = buf.clone()
            m.mfet_rows_read(d, back, n + 2, None, got, CODE[out], dim + pad, status, stream())
            codes, scales = ref.mx4_encode(x.double().cpu().numpy())
            full = np.concatenate([ref.mx4_decode(codes, scales), np.zeros((1, dim)), ref.mx4_decode(codes[:1], scales[:1])])
            assert torch.equal(got[:, :dim].cpu(), torch.from_numpy(full).to(DTYPES[out]))
            got[:, :dim] = 3.0
            assert torch.equal(buf, keep)  # nothing between or beyond the rows was written
        assert int(status.item()) == 0


def test_mxfp4_ties_powers_of_two_subnormals_and_extremes():
    """Every half-way point, block maxima at and next to powers of two, subnormal and largest fp32 values."""
    m = mfet()
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.999, 0.0, -0.0, 6.0, -5.0, -0.25, -2.5, 4.0])
    blocks = [np.concatenate([ties, -ties])]
    one_up, one_down = np.nextafter(np.float32(1), np.float32(2)), np.nextafter(np.float32(1), np.float32(0))
    for e in (-149, -148, -127, -126, -125, -124, -100, -24, -3, -1, 0, 1, 2, 60, 125, 126, 127):
        for f in (1.0, float(one_up), float(one_down), 1.5, 1.99):
            top = min(f * 2.0 ** e, float(np.finfo(np.float32).max))
            blocks.append(np.concatenate([[top, -top, top / 2, top / 3, top / 8, top / 17, 0.0, -top / 5], ties[:8] * top / 8, np.zeros(16)]))
    x = np.stack(blocks).astype(np.float32)
    n = x.shape[0]
    table = torch.zeros(n, m.row_bytes(32, m.MXFP4), dtype=torch.uint8, device="cuda")
    d = desc(m, table, n, 32, m.MXFP4)
    m.mfet_rows_write(d, None, n, None, torch.from_numpy(x).cuda(), 0, 32, None, stream())
    assert np.array_equal(table.cpu().numpy(), ref.mx4_rows(x.astype(np.float64)))
    out = torch.empty(n, 32, device="cuda")
    m.mfet_rows_read(d, None, n, None, out, 0, 32, None, stream())
    assert np.array_equal(out.cpu().numpy(), ref.mx4_decode(*ref.mx4_encode(x.astype(np.float64))).astype(np.float32))


@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
def test_blocks_with_nan_or_infinity_read_as_nan_and_leave_the_others_alone(src):
    m = mfet()
    x = values(np.random.default_rng(3), 8, 96, src)
    x[1, 5], x[2, 40], x[3, 95] = float("nan"), float("inf"), float("-inf")
    for dtype in (m.MXFP4, m.INT4):
        table = torch.zeros(8, m.row_bytes(96, dtype), dtype=torch.uint8, device="cuda")
        d = desc(m, table, 8, 96, dtype)
        m.mfet_rows_write(d, None, 8, None, x, CODE[src], 96, None, stream())
        out = torch.empty(8, 96, device="cuda")
        m.mfet_rows_read(d, None, 8, None, out, 0, 96, None, stream())
        nan = np.zeros((8, 96), bool)
        for r, c in ((1, 0), (2, 1), (3, 2)):
            nan[r, c * 32:(c + 1) * 32 if dtype == m.MXFP4 else None] = True
            if dtype == m.INT4:
                nan[r] = True
        assert np.array_equal(np.isnan(out.cpu().numpy()), nan)


@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 128, 264, 520])
def test_int4_rows_are_bit_exact(dim, src):
    m = mfet()
    rng = np.random.default_rng(100 + dim)
    n = 700
    x = values(rng, n, dim, src)
    x[5] = 0.125                        # a constant row: scale 0
    x[6] = 1000.0 + x[6]                # far from zero for its width
    x[7, 0] = 60000.0
    table = torch.full((n, m.row_bytes(dim, m.INT4)), 0xAB, dtype=torch.uint8, device="cuda")
    d = desc(m, table, n, dim, m.INT4)
    m.mfet_rows_write(d, None, n, None, x, CODE[src], dim, None, stream())
    want, fine = ref.int4_rows(x.float().cpu().numpy())
    assert fine.all()
    assert np.array_equal(table.cpu().numpy(), want)
    out = torch.empty(n, dim, device="cuda")
    m.mfet_rows_read(d, None, n, None, out, 0, dim, None, stream())
    scale = want[:, dim // 2:dim // 2 + 2].copy().view(np.float16).astype(np.float64)
    bias = want[:, dim // 2 + 2:dim // 2 + 4].copy().view(np.float16).astype(np.float64)
    codes = np.stack([want[:, :dim // 2] & 15, want[:, :dim // 2] >> 4], axis=2).reshape(n, dim)
    assert np.array_equal(out.cpu().numpy(), (codes * scale + bias).astype(np.float32))  # fma: one rounding


def test_int4_rows_near_half_way_quotients():
    """Quotients on and one ulp beside k + 1/2: the code is that of the double-precision quotient."""
    m = mfet()
    rng = np.random.default_rng(9)
    n, dim = 4000, 32
    lo = rng.standard_normal(n).astype(np.float16).astype(np.float32)
    scale = (2.0 ** rng.integers(-8, 3, n) * (1 + rng.integers(0, 1024, n) / 1024)).astype(np.float32)
    k = rng.integers(0, 15, (n, dim)) + 0.5
    x = (lo[:, None].astype(np.float64) + k * scale[:, None]).astype(np.float32)
    x = np.where(rng.random((n, dim)) < 0.5, np.nextafter(x, np.float32(np.inf)), x).astype(np.float32)
    x[:, 0], x[:, 1] = lo, lo + 15 * scale
    table = torch.zeros(n, m.row_bytes(dim, m.INT4), dtype=torch.uint8, device="cuda")
    m.mfet_rows_write(desc(m, table, n, dim, m.INT4), None, n, None, torch.from_numpy(x).cuda(), 0, dim, None, stream())
    assert np.array_equal(table.cpu().numpy(), ref.int4_rows(x)[0])


@pytest.mark.parametrize("table_dtype,dim", [("f32", 12), ("f32", 64), ("f16", 40), ("bf16", 136)])
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
def test_plain_tables_round_to_nearest(table_dtype, dim, src):
    m = mfet()
    n = 77
    x = values(np.random.default_rng(1), n, dim, src)
    table = torch.zeros(n, dim, dtype=DTYPES[table_dtype], device="cuda")
    d = desc(m, table, n, dim, CODE[table_dtype])
    at = torch.randperm(n, device="cuda")
    m.mfet_rows_write(d, at, n, None, x, CODE[src], dim, None, stream())
    assert torch.equal(table[at], x.to(table.dtype))
    out = torch.empty(n, dim, dtype=DTYPES[src], device="cuda")
    m.mfet_rows_read(d, at, n, None, out, CODE[src], dim, None, stream())
    assert torch.equal(out, x.to(table.dtype).to(out.dtype))


def test_counts_on_the_device_missing_rows_and_rows_past_the_table():
    m = mfet()
    n, dim, rows = 50, 64, 100
    x = values(np.random.default_rng(2), n, dim, "f32")
    for count, used in ((0, 0), (-3, 0), (17, 17), (50, 50), (51, 50), (2**40, 50)):
        table = torch.full((rows, m.row_bytes(dim, m.MXFP4)), 1, dtype=torch.uint8, device="cuda")
        d = desc(m, table, rows, dim, m.MXFP4)
        c = torch.tensor([count], dtype=torch.int64, device="cuda")
        m.mfet_rows_write(d, None, n, c, x, 0, dim, None, stream())
        want = np.full(tuple(table.shape), 1, np.uint8)
        want[:used] = ref.mx4_rows(x[:used].double().cpu().numpy())
        assert np.array_equal(table.cpu().numpy(), want)
        out = torch.full((n, dim), 9.0, device="cuda")
        m.mfet_rows_read(d, None, n, c, out, 0, dim, None, stream())
        assert (out[used:] == 9.0).all() and (used == 0 or not (out[:used] == 9.0).any())
    at = torch.arange(n, dtype=torch.int64, device="cuda")
    at[3], at[8], at[20] = -1, rows, 2**62
    table = torch.full((rows, m.row_bytes(dim, m.MXFP4)), 1, dtype=torch.uint8, device="cuda")
    d = desc(m, table, rows, dim, m.MXFP4)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    m.mfet_rows_write(d, at, n, None, x, 0, dim, status, stream())
    ok = [i for i in range(n) if i not in (3, 8, 20)]
    want = np.full(tuple(table.shape), 1, np.uint8)
    want[ok] = ref.mx4_rows(x[ok].double().cpu().numpy())
    assert np.array_equal(table.cpu().numpy(), want) and int(status.item()) == m.DEV_ROW_RANGE
    out = torch.full((n, dim), 9.0, device="cuda")
    m.mfet_rows_read(d, at, n, None, out, 0, dim, None, stream())  # without a status word
    assert (out[[3, 8, 20]] == 0).all()
    only_missing = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    status.zero_()
    m.mfet_rows_read(d, only_missing, n, None, out, 0, dim, status, stream())
    assert (out == 0).all() and int(status.item()) == 0


def test_rows_beyond_four_gigabytes():
    m = mfet()
    dim, rows = 64, 100_000_000  # 4.8 GB
    table = torch.zeros(rows * m.row_bytes(dim, m.MXFP4), dtype=torch.uint8, device="cuda")
    d = desc(m, table, rows, dim, m.MXFP4)
    x = values(np.random.default_rng(4), 64, dim, "f32")
    at = torch.arange(rows - 64, rows, dtype=torch.int64, device="cuda")
    m.mfet_rows_write(d, at, 64, None, x, 0, dim, None, stream())
    assert np.array_equal(table.view(rows, -1)[-64:].cpu().numpy(), ref.mx4_rows(x.double().cpu().numpy()))
    assert int(table.view(rows, -1)[:-64].max()) == 0
    out = torch.empty(64, dim, device="cuda")
    m.mfet_rows_read(d, at, 64, None, out, 0, dim, None, stream())
    assert np.array_equal(out.cpu().numpy(), ref.mx4_decode(*ref.mx4_encode(x.double().cpu().numpy())).astype(np.float32))


def test_another_stream():
    m = mfet()
    n, dim = 20000, 64
    x = values(np.random.default_rng(5), n, dim, "f32")
    table = torch.zeros(n, m.row_bytes(dim, m.MXFP4), dtype=torch.uint8, device="cuda")
    out = torch.empty(n, dim, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    d = desc(m, table, n, dim, m.MXFP4)
    m.mfet_rows_write(d, None, n, None, x, 0, dim, None, s.cuda_stream)
    m.mfet_rows_read(d, None, n, None, out, 0, dim, None, s.cuda_stream)
    s.synchronize()
    assert np.array_equal(out.cpu().numpy(), ref.mx4_decode(*ref.mx4_encode(x.double().cpu().numpy())).astype(np.float32))
