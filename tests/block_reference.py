"""Layer norm, the gated linear block and the orthogonalised update in 64 bits (torch double on the device of the arguments), with what
a kernel that computes in fp32 may be off by. Half a step of a type is HALF[dtype] relative to a value (at least TINY[dtype])."""
import math

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
U = 2.0**-24  # half a step of fp32
HALF = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
TINY = {torch.float32: 2.0**-149, torch.float16: 2.0**-25, torch.bfloat16: 2.0**-133}
USUAL = (3.4445, -4.775, 2.0315)


def rounding(v, dtype):
    return v.abs() * HALF[dtype] + TINY[dtype]


def norm(x, w, b, eps, dy=None):
    """(y, bound) or, with dy, (dx, dw, db, bounds of the three). x, dy: double; w, b: double or None.

    Every sum of a row is taken by at least 32 threads, of at most 32 values each when the row is held (else cols / 512), then across lanes and
    warps: `n` additions one after the other, each off by U of the partial sum."""
    cols = x.shape[1]
    n = max(32, cols / 512 + 8) + 5 + 16
    w = torch.ones_like(x[0]) if w is None else w
    b = torch.zeros_like(x[0]) if b is None else b
    mu = x.mean(1, keepdim=True)
    d = x - mu
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    xh = d * r
    off = r * n * U * x.abs().mean(1, keepdim=True)       # of the mean, in units of xh
    dxh = off * (1 + xh.abs()) + off * off * xh.abs() + (n + 10) * U * xh.abs()
    if dy is None:
        y = xh * w + b
        return y, dxh * w.abs() + 4 * U * (xh * w).abs() + 4 * U * b.abs()
    t = dy * w
    m0, m1 = t.mean(1, keepdim=True), (t * xh).mean(1, keepdim=True)
    dx = r * (t - m0 - xh * m1)
    rel = off + off * off + (n + 10) * U                   # of r
    bound = r * (n * U * (t.abs().mean(1, keepdim=True) + xh.abs() * (t * xh).abs().mean(1, keepdim=True)) + dxh * m1.abs()
                 + (xh.abs() + dxh) * (t.abs() * dxh).mean(1, keepdim=True) + 6 * U * (t.abs() + m0.abs() + (xh * m1).abs())) + rel * dx.abs()
    rows = x.shape[0]
    deep = min(rows, rows / 64 + 128) + 8                   # additions one after the other down a column
    return (dx, (dy * xh).sum(0), dy.sum(0), bound,
            (dy.abs() * dxh).sum(0) + deep * U * (dy * xh).abs().sum(0), deep * U * dy.abs().sum(0))


def act(name, g):
    """(act(g), act'(g), a bound of |act''|)"""
    if name == "none":
        return g, torch.ones_like(g), 0.0
    if name == "relu":
        return torch.where(g > 0, g, torch.where(g <= 0, torch.zeros_like(g), g)), (g > 0).to(g.dtype), 0.0
    if name == "gelu":
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 0.8
    s = torch.sigmoid(g)
    if name == "sigmoid":
        return s, s * (1 - s), 0.1
    return g * s, s * (1 + g * (1 - s)), 0.5


def product_bound(a, b, k):
    """Of a product on the tensor cores over k values: exact products, one truncation of fp32 (2^-23) per instruction of 16 values, and the few
    additions that join parts of k."""
    return (k / 16 + 8) * 2.0**-23 * (a.abs() @ b.abs())


def gated(x, wg, wu, name, dtype, dh=None):
    """(h, bound) or (dx, dwg, dwu, bounds): x, wg, wu, dh double, exactly values of dtype."""
    k = x.shape[1]
    g, u = x @ wg.T, x @ wu.T
    eg, eu = product_bound(x, wg.T, k), product_bound(x, wu.T, k)
    a, s, curve = act(name, g)
    ea = 1.13 * eg + 2.0**-17 * a.abs()                     # |act'| <= 1.13; the exponential's error
    if dh is None:
        h = a * u
        bound = ea * u.abs() + (a.abs() + ea) * eu
        return h, bound + rounding(h.abs() + bound, dtype)
    es = curve * eg + 2.0**-16
    if name == "none":
        es = torch.zeros_like(g)
    if name == "relu":
        es = (g.abs() <= eg).to(g.dtype)                     # the slope jumps at 0
    dg, du = dh * u * s, dh * a
    edg = dh.abs() * (eu * (s.abs() + es) + u.abs() * es)
    edg = edg + rounding(dg.abs() + edg, dtype) + 2 * U * dg.abs()
    edu = dh.abs() * ea
    edu = edu + rounding(du.abs() + edu, dtype) + 2 * U * du.abs()
    out = []
    m, n = dh.shape
    dx = dg @ wg + du @ wu
    bx = edg @ wg.abs() + edu @ wu.abs() + product_bound(dg.abs() + edg, wg, 2 * n) + product_bound(du.abs() + edu, wu, 2 * n)
    out.append((dx, bx))
    for d, e in ((dg, edg), (du, edu)):
        out.append((d.T @ x, e.T @ x.abs() + product_bound((d.abs() + e).T, x, m)))
    return tuple(v for v, _ in out) + tuple(b + rounding(v.abs() + b, dtype) for v, b in out)


def orthogonalize(g, coefficients, scale=1.0):
    """coefficients: (a, b, c) of every step."""
    size = torch.linalg.vector_norm(g)
    if not bool(torch.isfinite(size)):
        return torch.full_like(g, float("nan"))
    x = g / size if float(size) > 0 else torch.zeros_like(g)
    for a, b, c in coefficients:
        if g.shape[0] > g.shape[1]:
            p = x.T @ x
            x = a * x + x @ (b * p + c * (p @ p))
        else:
            p = x @ x.T
            x = a * x + (b * p + c * (p @ p)) @ x
    return scale * x


def orthogonalize_bound(x, g, coefficients, scale, dtype):
    """Of the error's Frobenius norm: what two-word matrices cost, what the sums cost, and the last rounding.

    An odd polynomial of the singular values passes an error on times at most the largest |slope| over their range (its divided differences are
    values of the slope), which for the usual coefficients is the slope a at 0. A step's own error from the words is taken as 2^-21 of the matrix
    (two words hold 2^-23 of a value, the product of the low words that is left out is 2^-22). One fp16 word would give 2^-12 instead.

    The sums: a product over K values truncates N = 3 K / 16 times, each time by 0.5 of a step of fp32 on average, all in one direction, with 0.58
    rms; a sum of K values that rounds to nearest is off by 0.29 sqrt(K) rms. So the same iteration in fp32, run here, is off by less by a
    factor of (0.5 N + 0.58 sqrt(N)) / (0.29 sqrt(K)) = 0.33 sqrt(K) + 0.87, if all of the truncations' common part counts (it only does in
    directions of large singular values); twice that, since one run is one sample."""
    grown = 1.0
    for a, _, _ in coefficients[1:]:
        grown = 1.0 + abs(a) * grown
    size = float(torch.linalg.vector_norm(x))
    length = max(g.shape)
    plain = float(torch.linalg.vector_norm(orthogonalize(g.float() / torch.linalg.vector_norm(g.double()).float(), coefficients, scale).double() - x)) \
        if size > 0 and math.isfinite(size) else 0.0
    return 2.0**-21 * grown * size + 2 * (0.33 * length**0.5 + 0.87) * plain + HALF[dtype] * size + TINY[dtype] * x.numel()**0.5


def within(got, want, bound):
    """Every element inside its bound; NaN where NaN is wanted."""
    got = got.double()
    nan = torch.isnan(want)
    bad = torch.where(nan, ~torch.isnan(got), ~((got - want).abs() <= bound) & (got != want))
    if bool(bad.any()):
        i = torch.nonzero(bad)[0].tolist()
        print("%d of %d outside; first at %s: got %r, want %r, bound %r" % (int(bad.sum()), bad.numel(), i, float(got[tuple(i)]), float(want[tuple(i)]),
                                                                        float(bound[tuple(i)]) if bound.dim() else float(bound)))
    return not bool(bad.any())
