"""The example that runs look-up, layer norm, gated block, their backward passes, clipping and the orthogonalised update together: every
stage against its 64-bit definition on what the stage before it gave."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block_step.py")
    spec = importlib.util.spec_from_file_location("gated_block_step", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


def test_it_runs():
    losses = example().main(steps=4, verbose=False)
    assert len(losses) == 4 and np.isfinite(losses).all()


def test_gradients_and_updates():
    ex = example()
    b = ex.Block(seed=3)
    try:
        b.norm_w.normal_(1.0, 0.2)
        b.norm_b.normal_(0.0, 0.1)
        b.forward()
        b.backward()
        torch.cuda.synchronize()
        x, bound = ref.norm(b.pooled.double(), b.norm_w.double(), b.norm_b.double(), ex.EPS)
        assert ref.within(b.x, x, bound + ref.rounding(x.abs() + bound, b.x.dtype))
        w = [t.double() for t in b.w]
        h, bound = ref.gated(b.x.double(), w[0], w[1], "silu", torch.bfloat16)
        assert ref.within(b.h, h, bound)
        dx, dwg, dwu, ex_, eg, eu = ref.gated(b.x.double(), w[0], w[1], "silu", torch.bfloat16, b.d_h.double())
        assert ref.within(b.d_x, dx, ex_) and ref.within(b.d_w[0], dwg, eg) and ref.within(b.d_w[1], dwu, eu)
        dp, dnw, dnb, ep, ew, eb = ref.norm(b.pooled.double(), b.norm_w.double(), None, ex.EPS, b.d_x.double())
        assert ref.within(b.d_pooled, dp, ep + ref.rounding(dp.abs() + ep, torch.float32))
        assert ref.within(b.d_norm[0], dnw, ew + ref.rounding(dnw, torch.float32)) and ref.within(b.d_norm[1], dnb, eb + ref.rounding(dnb, torch.float32))
        # the rows' gradients: every look-up of a row adds its sample's columns
        col = 0
        for i, d in enumerate(ex.DIMS):
            n = ex.BATCH * ex.BAG
            f = ex.SLOT_FEATURE[i]
            rows = torch.empty(n, dtype=torch.int64, device="cuda")
            ex.m.mfet_hash_ids(b.h_tables, i, b.ids[f * n:(f + 1) * n].contiguous(), n, rows, torch.cuda.current_stream().cuda_stream)
            part = b.d_pooled[:, col:col + d].double().repeat_interleave(ex.BAG, 0)
            dense = torch.zeros(ex.ROWS, d, dtype=torch.float64, device="cuda").index_add_(0, rows, part)
            mass = torch.zeros(ex.ROWS, d, dtype=torch.float64, device="cuda").index_add_(0, rows, part.abs())
            got = torch.zeros(ex.ROWS, d, dtype=torch.float64, device="cuda")
            k = int(b.counts[i].item())
            got[b.rows[i][:k]] = b.d_rows[i][:k].double()
            assert ref.within(got, dense, 1e-6 + 1e-5 * mass)
            col += d
        before = [t.clone() for t in b.master]
        b.step()
        torch.cuda.synchronize()
        for i in range(2):
            want = ref.orthogonalize(b.d_w[i].double(), [ref.USUAL] * 5, ex.LR_BLOCK)
            off = float(torch.linalg.vector_norm(b.update[i].double() - want))
            assert off <= ref.orthogonalize_bound(want, b.d_w[i], [ref.USUAL] * 5, ex.LR_BLOCK, torch.float32)
            assert torch.equal(b.master[i], before[i] - b.update[i])
        assert int(b.status.item()) == 0
    finally:
        b.close()


def test_a_step_in_a_graph():
    """Captured on a stream of its own while an eager step runs on another: the same bits as eager calls give."""
    ex = example()
    a, b = ex.Block(seed=5), ex.Block(seed=5)
    try:
        for _ in range(2):  # so that buffers of the upper model exist
            a.forward(), b.forward()
        a.backward(), b.backward()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.backward()
        for t in b.d_w + b.d_norm + [b.d_x, b.d_pooled]:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        a.backward()
        torch.cuda.synchronize()
        for s, t in zip(a.d_w + a.d_norm + [a.d_x, a.d_pooled], b.d_w + b.d_norm + [b.d_x, b.d_pooled]):
            assert torch.equal(s, t)
        graph.reset()
    finally:
        a.close()
        b.close()
