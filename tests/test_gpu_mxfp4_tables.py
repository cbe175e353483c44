"""MXFP4 tables in the look-up path: rows written by mfet_rows_write, pooled by mfet_embedding_bag_forward (device tables, host tables behind
the dedup and the hot-row cache, facets of other formats beside them), against the 64-bit definition.

Tolerance: the pooled values of the library's other formats, |gpu - ref| <= 1e-6 + 1e-5 |ref|, at the same scale (values around 0.01)."""
import numpy as np
import pytest
import torch

from tests import lowbit_reference as ref
from tests.helpers import assert_close, mfet

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def batch(rng, B, F, rows, longest):
    lens = rng.integers(0, longest + 1, B * F)
    lens[::5] = 0
    off = np.zeros(B * F + 1, np.int64)
    np.cumsum(lens, out=off[1:])
    n = int(off[-1])
    ids = rng.integers(0, rows, max(n, 1)).astype(np.uint64)
    return ids, off, rng.random(max(n, 1)).astype(np.float32)


def pooled(values, ids, off, w, B, f, pooling):
    out = np.zeros((B, values.shape[1]))
    for b in range(B):
        lo, hi = off[f * B + b], off[f * B + b + 1]
        if hi > lo:
            v = values[ids[lo:hi].astype(np.int64)]
            out[b] = (v * w[lo:hi, None]).sum(0) if pooling == 2 else v.mean(0) if pooling == 1 else v.sum(0)
    return out


@pytest.mark.parametrize("pooling", [0, 1, 2])
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 128, 136, 264, 520])
def test_pooled_rows(dim, pooling):
    m = mfet()
    rng = np.random.default_rng(dim * 3 + pooling)
    rows, B = 300, 150
    x = (rng.standard_normal((rows, dim)) * 0.01).astype(np.float32)
    table = torch.zeros(rows, m.row_bytes(dim, m.MXFP4) + 16, dtype=torch.uint8, device="cuda")  # rows further apart than they are long
    plain = torch.from_numpy((rng.standard_normal((rows, 64)) * 0.01).astype(np.float32)).cuda().half()
    d = m.TableDesc(table.data_ptr(), rows, dim, m.MXFP4, m.LOC_DEVICE, 0, 0, table.shape[1])
    int4 = torch.zeros(rows, m.row_bytes(64, m.INT4), dtype=torch.uint8, device="cuda")
    d4 = m.TableDesc(int4.data_ptr(), rows, 64, m.INT4, m.LOC_DEVICE, 0, 0, 0)
    m.mfet_rows_write(d, None, rows, None, torch.from_numpy(x).cuda(), 0, dim, None, stream())
    m.mfet_rows_write(d4, None, rows, None, plain, m.F16, 64, None, stream())
    as_read = torch.empty(rows, 64, device="cuda")
    m.mfet_rows_read(d4, None, rows, None, as_read, 0, 64, None, stream())
    h = m.mfet_tables_create([d, m.TableDesc(plain.data_ptr(), rows, 64, m.F16, m.LOC_DEVICE, 0, 0, 0), d4])
    try:
        ids, off, w = batch(rng, B, 2, rows, 90)
        shape, keep = m.make_shape(B, 2, [0, 1, 0, 1], 0, True)
        out = torch.full((B, 2 * dim + 128), float("nan"), device="cuda")
        tables, pools = [0, 1, 2, 0], [pooling, 0, pooling, pooling]
        m.mfet_embedding_bag_forward(h, shape, torch.from_numpy(ids.view(np.int64)).cuda(), torch.from_numpy(off).cuda(),
                                     torch.from_numpy(w).cuda(), tables, pools, out, stream())
        torch.cuda.synchronize()
        assert m.mfet_query_status(h) == 0
        v = ref.mx4_decode(*ref.mx4_encode(x.astype(np.float64)))
        want = np.concatenate([pooled(v, ids, off, w, B, 0, pooling), pooled(plain.double().cpu().numpy(), ids, off, w, B, 1, 0),
                               pooled(as_read.double().cpu().numpy(), ids, off, w, B, 0, pooling), pooled(v, ids, off, w, B, 1, pooling)], axis=1)
        assert_close(out.cpu().numpy(), want, "pooled MXFP4 rows")
    finally:
        torch.cuda.synchronize()
        m.mfet_tables_destroy(h)


@pytest.mark.parametrize("dim", [32, 72, 264])
def test_host_table_behind_cache(dim):
    """The quantised table in pinned host memory, some of its rows in the HBM cache, the others fetched."""
    m = mfet()
    rng = np.random.default_rng(dim)
    rows, B = 500, 64
    x = (rng.standard_normal((rows, dim)) * 0.01).astype(np.float32)
    packed = ref.mx4_rows(x.astype(np.float64))
    host = torch.from_numpy(packed.copy()).pin_memory()
    h = m.mfet_tables_create([m.TableDesc(None, rows, dim, m.MXFP4, m.LOC_HOST, 0, 0, 0)])
    try:
        m.mfet_host_tables_register(h, 0, host.data_ptr(), host.numel(), 1)
        ids, off, w = batch(rng, B, 1, rows, 60)
        cap = int(off[-1]) + 64
        ws = torch.empty(m.mfet_workspace_bytes(h, cap), dtype=torch.uint8, device="cuda")
        m.mfet_set_workspace(h, ws, ws.numel(), cap)
        cached = np.arange(0, rows, 3, dtype=np.int64)
        mem = torch.empty(m.mfet_cache_bytes(h, 0, cached.size), dtype=torch.uint8, device="cuda")
        m.mfet_cache_build(h, 0, cached, mem, mem.numel(), stream())
        shape, keep = m.make_shape(B, 1, [0], 0, True)
        out = torch.full((B, dim), float("nan"), device="cuda")
        m.mfet_embedding_bag_forward(h, shape, torch.from_numpy(ids.view(np.int64)).cuda(), torch.from_numpy(off).cuda(),
                                     torch.from_numpy(w).cuda(), [0], [2], out, stream())
        torch.cuda.synchronize()
        assert m.mfet_query_status(h) == 0
        v = ref.mx4_decode(*ref.mx4_encode(x.astype(np.float64)))
        assert_close(out.cpu().numpy(), pooled(v, ids, off, w, B, 0, 2), "host MXFP4 rows")
    finally:
        torch.cuda.synchronize()
        m.mfet_tables_destroy(h)


def test_the_synthetic_generator_refuses_mxfp4():
    m = mfet()
    buf = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    with pytest.raises(m.MfetError) as e:
        m.mfet_table_fill(buf, 0, 10, 64, m.MXFP4, 0, 1, 0, stream())
    assert e.value.status == m.ERR_INVALID_ARG
    with pytest.raises(m.MfetError) as e:
        m.mfet_tables_create([m.TableDesc(buf.data_ptr(), 10, 60, m.MXFP4, m.LOC_DEVICE, 0, 0, 0)])
    assert e.value.status == m.ERR_UNSUPPORTED_DIM
