"""Fine-tuning the tables that are being served, step by step, without the host learning a row count:

  look up and pool the MXFP4 tables             mfet_embedding_bag_forward
  first dense layer, MXFP4 weights              mfet_mx4_linear
  gradient of the pooled features               (torch: the upper model is the user's)
  gradient of the rows, one list per slot       mfet_embedding_bag_backward
  clip all lists and the bias's gradient        mfet_grad_clip
  master rows read, updated and written back    mfet_rows_read, mfet_rows_write (fp32 tables)
  ... and quantised into the served tables      mfet_rows_write (MXFP4 tables)

Run on a B200: python examples/finetune_step.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_05700_b200 import mfet as m  # noqa: E402

BATCH, FEATURES, ROWS, OUT = 512, 2, 4000, 48
DIMS = [32, 64, 32, 64]           # two facets per feature
SLOT_FEATURE = [0, 0, 1, 1]
LR, MAX_NORM, BAG = 50.0, 2e-3, 12


def operand(w):
    """MXFP4 operand of an fp32 matrix: (codes, scales)."""
    codes = torch.zeros(m.mfet_mx4_code_bytes(*w.shape), dtype=torch.uint8, device="cuda")
    scales = torch.zeros(m.mfet_mx4_scale_bytes(*w.shape), dtype=torch.uint8, device="cuda")
    m.mfet_mx4_quantize(w, m.F32, w.stride(0), w.shape[0], w.shape[1], codes, scales, torch.cuda.current_stream().cuda_stream)
    return codes, scales


def main(steps: int = 12, verbose: bool = True):
    torch.manual_seed(0)
    stream = torch.cuda.current_stream().cuda_stream
    width = sum(DIMS)

    # master tables in fp32, served tables in MXFP4, written from them
    master = [torch.randn(ROWS, d, device="cuda") * 0.01 for d in DIMS]
    served = [torch.zeros(ROWS, m.row_bytes(d, m.MXFP4), dtype=torch.uint8, device="cuda") for d in DIMS]
    master_desc = [m.TableDesc(t.data_ptr(), ROWS, d, m.F32, m.LOC_DEVICE, 0, 0, 0) for t, d in zip(master, DIMS)]
    served_desc = [m.TableDesc(t.data_ptr(), ROWS, d, m.MXFP4, m.LOC_DEVICE, 0, 0, 0) for t, d in zip(served, DIMS)]
    for t, d, desc in zip(master, DIMS, served_desc):
        m.mfet_rows_write(desc, None, ROWS, None, t, m.F32, d, None, stream)
    h = m.mfet_tables_create(served_desc)

    # one batch of look-ups, every bag BAG long; targets of a layer that the features cannot fit yet
    n = BATCH * BAG
    ids = torch.randint(0, 2**40, (FEATURES * n,), device="cuda")
    offsets = torch.arange(0, FEATURES * n + 1, BAG, dtype=torch.int64, device="cuda")
    target = torch.randn(BATCH, OUT, device="cuda") * 0.05
    w = torch.randn(OUT, width, device="cuda") / width**0.5
    bias = torch.zeros(OUT, device="cuda")
    w_codes, w_scales = operand(w)
    shape, keep = m.make_shape(BATCH, FEATURES, SLOT_FEATURE)
    tables, pooling = list(range(len(DIMS))), [m.POOL_SUM] * len(DIMS)

    # buffers that every step reuses
    ws = torch.empty(m.mfet_workspace_bytes(h, n), dtype=torch.uint8, device="cuda")
    m.mfet_set_workspace(h, ws, ws.numel(), n)
    pooled, y = torch.empty(BATCH, width, device="cuda"), torch.empty(BATCH, OUT, device="cuda")
    scratch = torch.empty(m.mfet_mx4_linear_bytes(BATCH, width), dtype=torch.uint8, device="cuda")
    rows = [torch.empty(n, dtype=torch.int64, device="cuda") for _ in DIMS]
    grads = [torch.zeros(n, d, device="cuda") for d in DIMS]
    values = [torch.empty(n, d, device="cuda") for d in DIMS]
    counts = torch.zeros(len(DIMS) + 1, dtype=torch.int64, device="cuda")
    counts[-1] = 1  # the bias's gradient is one row
    grad_bias, norm = torch.empty(1, OUT, device="cuda"), torch.empty(1, device="cuda")
    to_clip = m.make_grads(grads + [grad_bias], grads + [grad_bias], counts)
    clip_scratch = torch.empty(m.mfet_grad_clip_bytes(len(DIMS) + 1), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    losses, norms = [], []
    try:
        for step in range(steps):
            m.mfet_embedding_bag_forward(h, shape, ids, offsets, None, tables, pooling, pooled, stream)
            m.mfet_mx4_linear(pooled, m.F32, width, BATCH, w_codes, w_scales, OUT, width, bias, m.ACT_NONE, y, m.F32, OUT, scratch,
                              scratch.numel(), status, stream)
            diff = y - target
            losses.append((diff * diff).mean())
            grad_y = diff * (2.0 / diff.numel())
            grad_pooled = (grad_y @ w).contiguous()  # the quantiser counts as the identity
            torch.sum(grad_y, 0, out=grad_bias[0])
            for s in range(len(DIMS)):
                m.mfet_embedding_bag_backward(h, shape, ids, offsets, None, tables, pooling, grad_pooled, s, rows[s], grads[s],
                                              counts[s:s + 1], stream)
            m.mfet_grad_clip(to_clip, MAX_NORM, norm, clip_scratch, clip_scratch.numel(), stream)
            norms.append(norm.clone())
            bias.sub_(grad_bias[0], alpha=LR)
            for s, d in enumerate(DIMS):
                m.mfet_rows_read(master_desc[s], rows[s], n, counts[s:s + 1], values[s], m.F32, d, status, stream)
                values[s].sub_(grads[s], alpha=LR)  # rows beyond the count are not used
                m.mfet_rows_write(master_desc[s], rows[s], n, counts[s:s + 1], values[s], m.F32, d, status, stream)
                m.mfet_rows_write(served_desc[s], rows[s], n, counts[s:s + 1], values[s], m.F32, d, status, stream)
        torch.cuda.synchronize()
        assert m.mfet_query_status(h) == 0 and int(status.item()) == 0
    finally:
        torch.cuda.synchronize()
        m.mfet_tables_destroy(h)
    losses, norms = [float(v) for v in losses], [float(v) for v in norms]
    if verbose:
        for k, (a, b) in enumerate(zip(losses, norms)):
            print("step %2d  loss %.6f  gradient norm %.5f%s" % (k, a, b, "  (clipped)" if b > MAX_NORM else ""))
    return losses, norms, master, served


if __name__ == "__main__":
    main()
