"""A training step of a ranking model's first block on multi-faceted features:

  look up and pool the tables                   mfet_embedding_bag_forward   (fp32 features)
  normalise the features                        mfet_layer_norm              (to bf16)
  gated block                                   mfet_gated_linear
  head and loss                                 (torch: the upper model is the user's)
  gradient of the block and of its weights      mfet_gated_linear_backward
  ... of the features, norm weight and bias     mfet_layer_norm_backward     (to fp32)
  ... of the rows, one list per slot            mfet_embedding_bag_backward
  clip all of them together                     mfet_grad_clip
  orthogonalise the block's updates             mfet_orthogonalize
  write the rows back                           mfet_rows_read, mfet_rows_write

Run on a B200: python examples/gated_block_step.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_05700_b200 import mfet as m  # noqa: E402

BATCH, FEATURES, ROWS, UNITS, OUT, BAG = 512, 2, 4000, 160, 8, 6
DIMS = [32, 64, 32, 64]           # two facets per feature
SLOT_FEATURE = [0, 0, 1, 1]
WIDTH, EPS = sum(DIMS), 1e-5
LR_ROWS, LR_NORM, LR_BLOCK, MAX_NORM = 0.5, 0.05, 0.02, 1.0


class Block:
    """The tables, the block's weights and every buffer of a step, all kept from step to step."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.tables = [rand(ROWS, d) * 0.01 for d in DIMS]
        self.descs = [m.TableDesc(t.data_ptr(), ROWS, d, m.F32, m.LOC_DEVICE, 0, 0, 0) for t, d in zip(self.tables, DIMS)]
        self.h_tables = m.mfet_tables_create(self.descs)
        n = BATCH * BAG
        self.ids = torch.randint(0, 2**40, (FEATURES * n,), generator=g, device="cuda")
        self.offsets = torch.arange(0, FEATURES * n + 1, BAG, dtype=torch.int64, device="cuda")
        self.shape, self.keep = m.make_shape(BATCH, FEATURES, SLOT_FEATURE)
        self.slots, self.pooling = list(range(len(DIMS))), [m.POOL_SUM] * len(DIMS)
        self.ws = torch.empty(m.mfet_workspace_bytes(self.h_tables, n), dtype=torch.uint8, device="cuda")
        m.mfet_set_workspace(self.h_tables, self.ws, self.ws.numel(), n)
        bf = torch.bfloat16
        self.norm_w, self.norm_b = torch.ones(WIDTH, device="cuda"), torch.zeros(WIDTH, device="cuda")
        self.master = [rand(UNITS, WIDTH) / WIDTH**0.5 for _ in range(2)]   # gate and up
        self.w = [t.to(bf) for t in self.master]
        self.head = rand(OUT, UNITS) / UNITS**0.5
        self.target = rand(BATCH, OUT)
        empty = lambda *s, dtype=bf: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.pooled, self.x, self.h = empty(BATCH, WIDTH, dtype=torch.float32), empty(BATCH, WIDTH), empty(BATCH, UNITS)
        self.d_x, self.d_pooled = empty(BATCH, WIDTH), empty(BATCH, WIDTH, dtype=torch.float32)
        self.d_w = [empty(UNITS, WIDTH) for _ in range(2)]
        self.d_norm = [empty(WIDTH, dtype=torch.float32) for _ in range(2)]
        self.rows = [empty(n, dtype=torch.int64) for _ in DIMS]
        self.d_rows = [torch.zeros(n, d, device="cuda") for d in DIMS]
        self.values = [empty(n, d, dtype=torch.float32) for d in DIMS]
        dense = self.d_w + [t.view(1, -1) for t in self.d_norm]
        self.counts = torch.tensor([0] * len(DIMS) + [t.shape[0] for t in dense], dtype=torch.int64, device="cuda")
        self.grads = m.make_grads(self.d_rows + dense, self.d_rows + dense, self.counts)
        self.update = [empty(UNITS, WIDTH, dtype=torch.float32) for _ in range(2)]
        self.total, self.status = torch.empty(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        byte = lambda k: torch.empty(k, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.s_norm = byte(m.mfet_layer_norm_backward_bytes(BATCH, WIDTH))
        self.s_gated = byte(m.mfet_gated_linear_backward_bytes(BATCH, UNITS, WIDTH))
        self.s_clip = byte(m.mfet_grad_clip_bytes(len(DIMS) + len(dense)))
        self.s_orth = byte(m.mfet_orthogonalize_bytes(UNITS, WIDTH))

    def forward(self):
        s = torch.cuda.current_stream().cuda_stream
        m.mfet_embedding_bag_forward(self.h_tables, self.shape, self.ids, self.offsets, None, self.slots, self.pooling, self.pooled, s)
        m.mfet_layer_norm(self.pooled, m.F32, WIDTH, BATCH, WIDTH, self.norm_w, self.norm_b, EPS, self.x, m.BF16, WIDTH, s)
        m.mfet_gated_linear(self.x, m.BF16, WIDTH, BATCH, self.w[0], WIDTH, self.w[1], WIDTH, UNITS, WIDTH, m.ACT_SILU, self.h, UNITS, None, 0,
                            self.status, s)
        diff = self.h.float() @ self.head.T - self.target
        self.d_h = (diff * (2.0 / diff.numel()) @ self.head).to(torch.bfloat16)
        return (diff * diff).mean()

    def backward(self):
        s = torch.cuda.current_stream().cuda_stream
        m.mfet_gated_linear_backward(self.x, m.BF16, WIDTH, BATCH, self.w[0], WIDTH, self.w[1], WIDTH, UNITS, WIDTH, m.ACT_SILU, self.d_h, UNITS,
                                     self.d_x, WIDTH, self.d_w[0], WIDTH, self.d_w[1], WIDTH, self.s_gated, self.s_gated.numel(), self.status, s)
        m.mfet_layer_norm_backward(self.pooled, m.F32, WIDTH, BATCH, WIDTH, self.norm_w, EPS, self.d_x, m.BF16, WIDTH, self.d_pooled, WIDTH,
                                   self.d_norm[0], self.d_norm[1], self.s_norm, self.s_norm.numel(), s)
        for i in range(len(DIMS)):
            m.mfet_embedding_bag_backward(self.h_tables, self.shape, self.ids, self.offsets, None, self.slots, self.pooling, self.d_pooled, i,
                                          self.rows[i], self.d_rows[i], self.counts[i:i + 1], s)

    def step(self):
        s = torch.cuda.current_stream().cuda_stream
        m.mfet_grad_clip(self.grads, MAX_NORM, self.total, self.s_clip, self.s_clip.numel(), s)
        for i in range(2):  # the block's weights: updates of the same size in every direction
            m.mfet_orthogonalize(self.d_w[i], m.BF16, WIDTH, UNITS, WIDTH, None, 5, LR_BLOCK, self.update[i], m.F32, WIDTH, self.s_orth,
                                 self.s_orth.numel(), self.status, s)
            self.master[i].sub_(self.update[i])
            self.w[i].copy_(self.master[i])
        self.norm_w.sub_(self.d_norm[0], alpha=LR_NORM)
        self.norm_b.sub_(self.d_norm[1], alpha=LR_NORM)
        n = BATCH * BAG
        for i, d in enumerate(DIMS):
            m.mfet_rows_read(self.descs[i], self.rows[i], n, self.counts[i:i + 1], self.values[i], m.F32, d, self.status, s)
            self.values[i].sub_(self.d_rows[i], alpha=LR_ROWS)  # rows beyond the count are not used
            m.mfet_rows_write(self.descs[i], self.rows[i], n, self.counts[i:i + 1], self.values[i], m.F32, d, self.status, s)

    def close(self):
        torch.cuda.synchronize()
        m.mfet_tables_destroy(self.h_tables)


def main(steps: int = 10, verbose: bool = True):
    block = Block()
    losses = []
    try:
        for _ in range(steps):
            losses.append(block.forward())
            block.backward()
            block.step()
        torch.cuda.synchronize()
        assert m.mfet_query_status(block.h_tables) == 0 and int(block.status.item()) == 0
    finally:
        block.close()
    losses = [float(v) for v in losses]
    if verbose:
        for k, v in enumerate(losses):
            print("step %2d  loss %.6f" % (k, v))
    return losses


if __name__ == "__main__":
    main()
