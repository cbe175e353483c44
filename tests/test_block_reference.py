"""The 64-bit definitions that the GPU tests compare with: their gradients against differences and autograd (no GPU needed)."""
import pytest
import torch

from tests import block_reference as ref

H = 1e-6


def directional(f, point, direction):
    return (f(point + H * direction) - f(point - H * direction)) / (2 * H)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 40)])
def test_layer_norm_gradients(rows, cols):
    g = torch.Generator().manual_seed(rows)
    x, dy, dirx = (torch.randn(rows, cols, generator=g, dtype=torch.float64) for _ in range(3))
    w, b, dirw = (torch.randn(cols, generator=g, dtype=torch.float64) for _ in range(3))
    dx, dw, db = ref.norm(x, w, b, 1e-3, dy)[:3]
    loss = lambda x_, w_, b_: (ref.norm(x_, w_, b_, 1e-3)[0] * dy).sum()
    scale = float(dy.abs().sum() * (1 + w.abs().max())) + 1
    assert abs(directional(lambda p: loss(p, w, b), x, dirx) - (dx * dirx).sum()) < 1e-7 * scale * 30
    assert abs(directional(lambda p: loss(x, p, b), w, dirw) - (dw * dirw).sum()) < 1e-7 * scale
    assert abs(directional(lambda p: loss(x, w, p), b, dirw) - (db * dirw).sum()) < 1e-7 * scale


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu", "sigmoid"])
def test_gated_gradients(name):
    g = torch.Generator().manual_seed(7)
    x, wg, wu, dh = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((6, 5), (4, 5), (4, 5), (6, 4)))
    dx, dwg, dwu = ref.gated(x, wg, wu, name, torch.float32, dh)[:3]
    leaves = [t.clone().requires_grad_(True) for t in (x, wg, wu)]
    fn = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
          "sigmoid": torch.sigmoid}[name]
    ((fn(leaves[0] @ leaves[1].T) * (leaves[0] @ leaves[2].T)) * dh).sum().backward()
    for got, leaf in zip((dx, dwg, dwu), leaves):
        assert torch.allclose(got, leaf.grad, rtol=1e-11, atol=1e-11)
        d = torch.randn(got.shape, generator=g, dtype=torch.float64)
        at = [x, wg, wu]
        i = [k for k, l in enumerate(leaves) if l is leaf][0]
        loss = lambda p: (ref.gated(*[p if k == i else at[k] for k in range(3)], name, torch.float32)[0] * dh).sum()
        assert abs(directional(loss, at[i], d) - (got * d).sum()) < 1e-5 * (1 + got.abs().sum())


@pytest.mark.parametrize("name", ["silu", "gelu", "sigmoid"])
def test_slopes_have_the_stated_bounds(name):
    v = torch.linspace(-12, 12, 20001, dtype=torch.float64)
    _, s, curve = ref.act(name, v)
    assert float(s.abs().max()) < 1.13
    assert float(((s[1:] - s[:-1]) / (v[1] - v[0])).abs().max()) < curve * 1.001


@pytest.mark.parametrize("rows,cols", [(3, 7), (7, 3), (4, 4)])
def test_orthogonalize_acts_on_the_singular_values(rows, cols):
    g = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    u, s, vh = torch.linalg.svd(g, full_matrices=False)
    s = s / torch.linalg.vector_norm(g)
    steps = [(3.0, -4.0, 2.0), (1.875, -1.25, 0.375)]
    for a, b, c in steps:
        s = a * s + b * s**3 + c * s**5
    assert torch.allclose(ref.orthogonalize(g, steps, 0.5), 0.5 * (u * s) @ vh, rtol=1e-12, atol=1e-12)
