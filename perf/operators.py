"""The operators around a fine-tuned, quantised embedding table, as they are measured.

Three operators, each in a plain form (elementary torch operations in 32 bits) and as the library's call:

  clip    the global 2-norm of many gradient tensors, and the gradients scaled so that it is at most max_norm
  rows    rows of values written into an MXFP4 table (quantised as they are written), and rows read back from it
  linear  act(quantised(x) @ w.T + bias) with MXFP4 operands: a first dense layer on pooled features

MXFP4: blocks of 32 values along a row share one scale 2^(e-127), held as the byte e; a value is a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale. A block's e is floor(log2(largest magnitude)) - 2 + 127, at least 0; values
are rounded to the nearest, ties to the even code, and saturate at 6 times the scale.
"""
import math

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}

# the most work that a drawn case may have (that of the largest listed ones)
MAX_CLIP, MAX_ROWS_ELEMS, MAX_TABLE_ROWS, MAX_M, MAX_K, MAX_N = 200_000_000, 2_000_000 * 64, 8_000_000, 16384, 2048, 2048


def listed():
    return [
        # the dense parameters of a very small model: one layer's weight and bias, where the launches are the cost
        {"name": "clip_one_layer", "op": "clip", "kind": "dense", "tensors": 2, "total": 17_000, "dtype": "f32", "spread": 3.0, "fill": 1.0, "dim": 0},
        # the sparse gradients of twelve facet tables (dims 32, 64 and 128 in turn, as many values as a batch of 8192
        # has look-ups for, of which 45 % are distinct rows; their number is known on the device alone)
        {"name": "clip_facets", "op": "clip", "kind": "rows", "tensors": 12, "total": 73_400_320, "dtype": "f32", "spread": 0.0, "fill": 0.45, "dim": 32},
        # the dense part of a ranking model: 300 tensors from a bias of a few values to matrices, in bf16, one after
        # the other in a bucket and hence at odd addresses
        {"name": "clip_dense_bf16", "op": "clip", "kind": "dense", "tensors": 300, "total": 199_999_967, "dtype": "bf16", "spread": 4.0, "fill": 1.0, "dim": 0},
        # one row refreshed between two requests
        {"name": "rows_one", "op": "rows", "n": 1, "dim": 64, "table_rows": 100_000, "src": "f32", "dst": "f32"},
        # the rows that one training step of a 128-column facet table touched
        {"name": "rows_step", "op": "rows", "n": 36_863, "dim": 128, "table_rows": 1_000_000, "src": "f32", "dst": "f32"},
        # a hot-row cache of two million rows refreshed from bf16 master rows
        {"name": "rows_refresh", "op": "rows", "n": 2_000_000, "dim": 64, "table_rows": 8_000_000, "src": "bf16", "dst": "bf16"},
        # rows whose width is not a multiple of the block, in fp16
        {"name": "rows_short_block", "op": "rows", "n": 100_003, "dim": 40, "table_rows": 500_000, "src": "f16", "dst": "f32"},
        # the first layer for one request: 896 pooled features
        {"name": "linear_one", "op": "linear", "m": 1, "k": 896, "n": 1024, "x": "f32", "y": "f32", "pad": 0, "bias": True, "relu": True},
        # a handful of candidates, odd output width, padded rows
        {"name": "linear_few", "op": "linear", "m": 7, "k": 2048, "n": 1000, "x": "f32", "y": "bf16", "pad": 5, "bias": True, "relu": False},
        # a batch of 500 with a width that ends inside a block
        {"name": "linear_ragged", "op": "linear", "m": 500, "k": 1075, "n": 777, "x": "bf16", "y": "f32", "pad": 3, "bias": False, "relu": True},
        # the multi-faceted batch: 8192 samples of 896 features, as the look-up writes them
        {"name": "linear_facets", "op": "linear", "m": 8192, "k": 896, "n": 1024, "x": "f32", "y": "bf16", "pad": 0, "bias": True, "relu": True},
        # the widest feature tensor: 16384 samples of 2048 features
        {"name": "linear_wide", "op": "linear", "m": 16384, "k": 2048, "n": 2048, "x": "bf16", "y": "bf16", "pad": 0, "bias": True, "relu": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["clip", "rows", "linear"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "clip":
        kind = rng.choice(["dense", "rows"])
        total = _log(rng, 1000, MAX_CLIP // 2 if dtype == "f32" else MAX_CLIP)
        if kind == "rows":
            return {"op": op, "kind": kind, "tensors": rng.randint(1, 24), "total": max(total, 100_000), "dtype": "f32" if total > 10_000_000 else dtype,
                    "spread": 0.0, "fill": round(rng.uniform(0.05, 1.0), 3), "dim": 8 * rng.randint(1, 32)}
        return {"op": op, "kind": kind, "tensors": min(_log(rng, 1, 400), total // 8), "total": total, "dtype": dtype, "spread": round(rng.uniform(0.5, 4.0), 2),
                "fill": 1.0, "dim": 0}
    if op == "rows":
        dim = 8 * _log(rng, 1, 32)
        n = _log(rng, 1, min(MAX_ROWS_ELEMS // dim, 2_000_000))
        return {"op": op, "n": n, "dim": dim, "table_rows": min(MAX_TABLE_ROWS, max(2 * n, _log(rng, 1000, MAX_TABLE_ROWS * 64 // dim))), "src": dtype,
                "dst": rng.choice(["f32", "f16", "bf16"])}
    return {"op": op, "m": _log(rng, 1, MAX_M), "k": _log(rng, 32, MAX_K), "n": _log(rng, 16, MAX_N), "x": dtype, "y": rng.choice(["f32", "f16", "bf16"]),
            "pad": rng.choice([0, 0, 8, rng.randint(1, 31)]), "bias": rng.random() < 0.7, "relu": rng.random() < 0.5}


# ---------------------------------------------------------------- MXFP4, plain ----

def _pow2(e):
    """2^e in fp32 for whole e in [-127, 127], from the bits."""
    return torch.where(e < -126, torch.full_like(e, 0x00400000), (e + 127) << 23).view(torch.float32)


def _encode(x):
    """(codes, scale bytes) of fp32 rows x [r, 32 b]: codes uint8 [r, 32 b], scales uint8 [r, b]."""
    b = x.reshape(x.shape[0], -1, 32)
    amax = b.abs().amax(dim=2)
    e = torch.clamp(torch.frexp(amax)[1] - 3, min=-127)  # amax = f * 2^k with f in [0.5, 1): floor(log2 amax) = k - 1
    e = torch.where(amax > 0, e, torch.full_like(e, -127))
    v = b.abs() * _pow2(-e)[:, :, None]
    code = (v > 0.25).to(torch.uint8) + (v >= 0.75).to(torch.uint8) + (v > 1.25).to(torch.uint8) + (v >= 1.75).to(torch.uint8) \
        + (v > 2.5).to(torch.uint8) + (v >= 3.5).to(torch.uint8) + (v > 5.0).to(torch.uint8)
    code = code + (b < 0).to(torch.uint8) * 8
    return code.reshape(x.shape), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """fp32 values of codes uint8 [r, c] under scales uint8 [r, ceil(c / 32)]."""
    lut = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float32, device=codes.device)
    s = _pow2(scales.to(torch.int32) - 127).repeat_interleave(32, dim=1)[:, :codes.shape[1]]
    return lut[codes.to(torch.int32)] * s


def _pad32(x):
    k = x.shape[1]
    return torch.nn.functional.pad(x, (0, -k % 32))


def _pack(codes):
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), dim=2).reshape(packed.shape[0], -1)


def _tile_scales(s):
    """Scale bytes [r, b] in the order that the product reads: 128 rows x 4 blocks are 512 bytes in a row, byte
    (r % 32) * 16 + (r / 32) * 4 + b of them; rows and blocks are filled up with zeros."""
    r, b = s.shape
    s = torch.nn.functional.pad(s, (0, -b % 4, 0, -r % 128))
    return s.reshape(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous().reshape(-1)


def _untile_scales(t, r, b):
    rp, bp = r + -r % 128, b + -b % 4
    return t.reshape(rp // 128, bp // 4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rp, bp)[:r, :b]


def _row_bytes(dim):
    return (dim // 2 + (dim + 31) // 32 + 15) // 16 * 16


# ---------------------------------------------------------------- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1_000_003 + 17)


def _clip_shapes(c):
    """(rows, columns) of every gradient tensor, the same for every seed."""
    t = c["tensors"]
    if c["kind"] == "rows":
        dims = [c["dim"] << (i % 3) for i in range(t)]
        return [(max(1, c["total"] // sum(dims)), d) for d in dims]
    w = [math.exp(-c["spread"] * ((i * 0.6180339887) % 1.0) * 2.0) for i in range(t)]  # sizes over a wide range
    left, sizes = c["total"], []
    for i in range(t):
        n = max(1, int(c["total"] * w[i] / sum(w))) if i + 1 < t else left
        n = max(1, min(n, left - (t - 1 - i)))
        sizes.append(n)
        left -= n
    return [(1, n) for n in sizes]


def _clip_counts(c):
    return [max(1, int(r * c["fill"]) - i) if c["kind"] == "rows" else r for i, (r, _) in enumerate(_clip_shapes(c))]


def _prepare_clip(c, g):
    shapes = _clip_shapes(c)
    total = sum(r * d for r, d in shapes)
    dt = DTYPES[c["dtype"]]
    # gradients of a loss averaged over a batch: small, a few hot rows far larger than the rest
    flat = torch.randn(total, generator=g, device="cuda", dtype=torch.float32)
    flat.mul_(0.01)
    flat[:: 1009] *= 20.0
    flat = flat.to(dt)
    out = torch.zeros(total, dtype=dt, device="cuda")
    counts = torch.tensor(_clip_counts(c), dtype=torch.int64, device="cuda")
    at = [0]
    for r, d in shapes:
        at.append(at[-1] + r * d)
    live = sum(n * d for n, (_, d) in zip(_clip_counts(c), shapes))
    max_norm = 0.3 * 0.01 * math.sqrt(live * (1 + 399 / 1009))  # the norm is about 3.3 times the limit
    return {"op": "clip", "shapes": shapes, "src": [flat[a:b].view(s) for a, b, s in zip(at, at[1:], shapes)],
            "dst": [out[a:b].view(s) for a, b, s in zip(at, at[1:], shapes)], "flat": out, "counts": counts if c["kind"] == "rows" else None,
            "norm": torch.zeros(1, device="cuda"), "max_norm": max_norm, "scratch": torch.empty(1 << 16, dtype=torch.uint8, device="cuda")}


def _prepare_rows(c, g):
    n, dim, rows = c["n"], c["dim"], c["table_rows"]
    nb = (dim + 31) // 32
    src = torch.randn(n, dim, generator=g, device="cuda", dtype=torch.float32) * 0.01
    src[:: 97] *= 50.0
    src[5:: 1003] = 0.0  # rows that nothing has touched yet
    src = src.to(DTYPES[c["src"]])
    table = torch.zeros(rows, _row_bytes(dim), dtype=torch.uint8, device="cuda")
    table[:, :dim // 2] = torch.randint(0, 256, (rows, dim // 2), generator=g, device="cuda", dtype=torch.uint8)
    table[:, dim // 2:dim // 2 + nb] = torch.randint(112, 125, (rows, nb), generator=g, device="cuda", dtype=torch.uint8)
    order = torch.randperm(rows, generator=g, device="cuda")
    slots = order[:n].sort().values                    # distinct rows, ascending: as the backward pass lists them
    back = torch.cat((slots, order[n:2 * n]))          # read: what was written and as many others, in any order
    back = back[torch.randperm(back.numel(), generator=g, device="cuda")].contiguous()
    back[7:: 501] = -1                                 # look-ups without a row read zeros
    return {"op": "rows", "dim": dim, "src": src, "table": table, "slots": slots, "back": back,
            "dst": torch.empty(back.numel(), dim, dtype=DTYPES[c["dst"]], device="cuda"), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _prepare_linear(c, g):
    m, k, n, pad = c["m"], c["k"], c["n"], c["pad"]
    nb = (k + 31) // 32
    # pooled features: sums of some tens of rows of size 0.01, some samples with much longer bags, some with none
    x = torch.randn(m, k + pad, generator=g, device="cuda", dtype=torch.float32) * 0.04
    x[3:: 29] *= 8.0
    x[11:: 64, : k // 2] = 0.0
    w = torch.randn(n, k, generator=g, device="cuda", dtype=torch.float32) / math.sqrt(k)
    codes, scales = _encode(_pad32(w))
    pb = (m + 127) // 128 * ((nb + 3) // 4) * 512
    return {"op": "linear", "x": x.to(DTYPES[c["x"]]), "m": m, "k": k, "n": n, "w": _pack(codes).contiguous(), "ws": _tile_scales(scales),
            "bias": torch.randn(n, generator=g, device="cuda") * 0.1 if c["bias"] else None, "relu": c["relu"],
            "y": torch.zeros(m, n + pad, dtype=DTYPES[c["y"]], device="cuda"),
            "scratch": torch.empty(m * nb * 16 + pb + 256, dtype=torch.uint8, device="cuda"), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    return {"clip": _prepare_clip, "rows": _prepare_rows, "linear": _prepare_linear}[case["op"]](case, _gen(seed))


# ---------------------------------------------------------------- one pass ----

def _clip_plain(s):
    counts = s["counts"]
    if counts is None:
        live = [t.float() for t in s["src"]]
    else:
        live = [torch.where((torch.arange(t.shape[0], device=t.device) < counts[i])[:, None], t.float(), 0.0) for i, t in enumerate(s["src"])]
    norm = torch.sqrt(sum((t * t).sum() for t in live))
    coef = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    [d.copy_(t * coef) for d, t in zip(s["dst"], live)]
    s["norm"].copy_(norm)


def _rows_plain(s):
    dim, nb, table = s["dim"], (s["dim"] + 31) // 32, s["table"]
    codes, scales = _encode(_pad32(s["src"].float()))
    table[s["slots"], :dim // 2] = _pack(codes)[:, :dim // 2]
    table[s["slots"], dim // 2:dim // 2 + nb] = scales
    row = table[s["back"].clamp(min=0)]
    got = _decode(_unpack(row[:, :dim // 2]), row[:, dim // 2:dim // 2 + nb])
    s["dst"].copy_(torch.where((s["back"] >= 0)[:, None], got, 0.0))


def _linear_plain(s):
    k, n = s["k"], s["n"]
    x = _decode(*_encode(_pad32(s["x"][:, :k].float())))
    w = _decode(_unpack(s["w"]), _untile_scales(s["ws"], n, (k + 31) // 32))
    y = x @ w.T
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["relu"]:
        y = torch.clamp(y, min=0)
    s["y"][:, :n].copy_(y)


def _run_own(s):
    from paper_2508_05700_b200 import mfet as m
    stream = torch.cuda.current_stream().cuda_stream
    if s["op"] == "clip":
        if "grads" not in s:  # the list of tensors, which a training program keeps
            s["grads"] = m.make_grads(s["src"], s["dst"], s["counts"])
        m.mfet_grad_clip(s["grads"], s["max_norm"], s["norm"], s["scratch"], s["scratch"].numel(), stream)
    elif s["op"] == "rows":
        if "desc" not in s:
            s["desc"] = m.TableDesc(s["table"].data_ptr(), s["table"].shape[0], s["dim"], m.MXFP4, m.LOC_DEVICE, 0, 0, 0)
        m.mfet_rows_write(s["desc"], s["slots"], s["slots"].numel(), None, s["src"], m.dtype_of(s["src"]), s["dim"], s["status"], stream)
        m.mfet_rows_read(s["desc"], s["back"], s["back"].numel(), None, s["dst"], m.dtype_of(s["dst"]), s["dim"], s["status"], stream)
    else:
        x, y = s["x"], s["y"]
        m.mfet_mx4_linear(x, m.dtype_of(x), x.stride(0), s["m"], s["w"], s["ws"], s["n"], s["k"], s["bias"], m.ACT_RELU if s["relu"] else m.ACT_NONE,
                          y, m.dtype_of(y), y.stride(0), s["scratch"], s["scratch"].numel(), s["status"], stream)


def run(state):
    if own:
        _run_own(state)
    else:
        {"clip": _clip_plain, "rows": _rows_plain, "linear": _linear_plain}[state["op"]](state)
    if state["op"] == "clip":
        return {"grads": state["flat"], "norm": state["norm"]}
    if state["op"] == "rows":
        return {"values": state["dst"], "status": state["status"]}
    return {"y": state["y"][:, :state["n"]], "status": state["status"]}


# ---------------------------------------------------------------- what it cannot do without ----

def work(case):
    if case["op"] == "clip":
        n = sum(r * d for r, (_, d) in zip(_clip_counts(case), _clip_shapes(case)))
        return {"bytes": 2.0 * n * SIZES[case["dtype"]], "flops": 3.0 * n}
    if case["op"] == "rows":
        n, dim = case["n"], case["dim"]
        back = min(2 * n, case["table_rows"])
        row = dim // 2 + (dim + 31) // 32
        return {"bytes": float(n * (dim * SIZES[case["src"]] + row + 8) + back * (dim * SIZES[case["dst"]] + row + 8)), "flops": 2.0 * n * dim + back * dim}
    m, k, n = case["m"], case["k"], case["n"]
    w = n * (k / 2 + k / 32)
    return {"bytes": m * k * SIZES[case["x"]] + w + m * n * SIZES[case["y"]] + (4.0 * n if case["bias"] else 0.0), "flops": 2.0 * m * k * n}


# ---------------------------------------------------------------- from the definition, in 64 bits ----

def _values64(x):
    """What MXFP4 makes of each row of x (fp64 [r, c]): per block of 32 the power of two, then the nearest level, by
    the spacing of the levels around the value."""
    r, c = x.shape
    b = torch.nn.functional.pad(x, (0, -c % 32)).reshape(r, -1, 32)
    top = b.abs().amax(dim=2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = torch.where(torch.exp2(e) > top, e - 1, e)             # log2 may have been rounded across a whole number
    e = torch.where(torch.exp2(e + 1) <= top, e + 1, e)
    scale = torch.exp2(torch.where(top > 0, torch.clamp(e - 2, min=-127.0), -127.0))
    a = b.abs() / scale
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(torch.float64)
    q = torch.clamp(torch.round(a / step) * step, max=6.0)     # torch.round: ties to even multiples = even codes
    return (torch.sign(b) * q * scale).reshape(r, -1)[:, :c]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        counts = _clip_counts(case)
        total = math.sqrt(math.fsum(float(t[:n].double().square().sum()) for t, n in zip(s["src"], counts)))
        coef = min(1.0, s["max_norm"] / total)
        flat = torch.cat([torch.cat((t[:n].double() * coef, torch.zeros_like(t[n:], dtype=torch.float64))).reshape(-1) for t, n in zip(s["src"], counts)])
        return {"grads": flat, "norm": torch.tensor([total], dtype=torch.float64)}
    if case["op"] == "rows":
        dim, nb = s["dim"], (s["dim"] + 31) // 32
        raw = s["table"]
        got = torch.zeros(s["back"].numel(), dim, dtype=torch.float64, device="cuda")
        where = torch.full((raw.shape[0],), -1, dtype=torch.int64, device="cuda")
        where[s["slots"]] = torch.arange(s["slots"].numel(), device="cuda")
        ok = s["back"] >= 0
        at = torch.where(ok, where[s["back"].clamp(min=0)], -1)
        new = torch.nonzero(at >= 0).reshape(-1)
        got[new] = _values64(s["src"].double())[at[new]]
        old = torch.nonzero(ok & (at < 0)).reshape(-1)
        row = raw[s["back"][old]]
        code = torch.empty(old.numel(), dim, dtype=torch.uint8, device="cuda")
        code[:, 0::2], code[:, 1::2] = row[:, :dim // 2] % 16, row[:, :dim // 2] // 16
        mag = (code % 8).double()
        mag = torch.where(mag < 4, mag / 2, torch.where(mag < 6, mag - 2, 2 * mag - 8))
        val = torch.where(code >= 8, -mag, mag)
        power = torch.exp2(row[:, dim // 2:dim // 2 + nb].double() - 127.0)
        got[old] = val * power[:, torch.arange(dim, device="cuda") // 32]
        return {"values": got, "status": None}
    k, n = s["k"], s["n"]
    g = _gen(seed)  # the weights' own values once more, in the order in which prepare() draws them
    torch.randn(s["m"], s["x"].shape[1], generator=g, device="cuda", dtype=torch.float32)
    w = torch.randn(n, k, generator=g, device="cuda", dtype=torch.float32) / math.sqrt(k)
    y = _values64(s["x"][:, :k].double()) @ _values64(w.double()).T
    if s["bias"] is not None:
        y = y + s["bias"].double()
    return {"y": torch.clamp(y, min=0) if s["relu"] else y, "status": None}
