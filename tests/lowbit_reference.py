"""Plain 64-bit definitions of what the row, matrix and clipping calls compute (numpy; nothing of the library)."""
import numpy as np

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx4_encode(x):
    """(codes [r, c], scale bytes [r, ceil(c / 32)]) of fp64 rows x."""
    x = np.asarray(x, np.float64)
    r, c = x.shape
    nb = -(-c // 32)
    b = np.pad(x, ((0, 0), (0, nb * 32 - c))).reshape(r, nb, 32)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[:, :, None], 0.0, b)
    amax = np.abs(b).max(axis=2)
    _, e = np.frexp(amax)  # amax = f * 2^e, 0.5 <= f < 1
    byte = np.where(amax > 0, np.maximum(e - 1 - 2 + 127, 0), 0)
    v = np.abs(b) / np.exp2(byte - 127.0)[:, :, None]
    d = np.abs(v[..., None] - LEVELS)
    near = d.min(axis=-1, keepdims=True)
    # of two equally near levels the one with the even code
    code = np.where(d == near, np.arange(8) + 100 * (np.arange(8) % 2), 1000).argmin(axis=-1)
    code = code + 8 * np.signbit(b)
    code = np.where(bad[:, :, None], 0, code).reshape(r, nb * 32)[:, :c]
    return code.astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def mx4_decode(codes, scales):
    codes = np.asarray(codes, np.int64)
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    with np.errstate(invalid="ignore"):
        return v * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def pack(codes):
    """Two codes per byte, the even element in the low nibble."""
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def mx4_row_bytes(dim):
    return (dim // 2 + -(-dim // 32) + 15) // 16 * 16


def mx4_rows(x):
    codes, scales = mx4_encode(x)
    r, dim = codes.shape
    out = np.zeros((r, mx4_row_bytes(dim)), np.uint8)
    out[:, :dim // 2] = pack(codes)
    out[:, dim // 2:dim // 2 + scales.shape[1]] = scales
    return out


def int4_rows(x32):
    """INT4 rows of fp32 rows: scale = fp16((max - min) / 15), bias = fp16(min), the quotient in double precision."""
    x32 = np.asarray(x32, np.float32)
    r, dim = x32.shape
    with np.errstate(all="ignore"):
        lo, hi = x32.min(axis=1), x32.max(axis=1)
        scale = ((hi - lo) / np.float32(15)).astype(np.float16)
        bias = lo.astype(np.float16)
        fine = np.isfinite(scale) & np.isfinite(bias)
        q = np.rint((x32.astype(np.float64) - bias.astype(np.float64)[:, None]) / scale.astype(np.float64)[:, None])
        code = np.where((fine & (scale > 0))[:, None], np.clip(np.nan_to_num(q), 0, 15), 0).astype(np.uint8)
    out = np.zeros((r, (dim // 2 + 4 + 15) // 16 * 16), np.uint8)
    out[:, :dim // 2] = pack(code)
    meta = np.stack([scale, bias], axis=1)
    meta[~fine] = np.float16(np.nan)
    out[:, dim // 2:dim // 2 + 4] = meta.view(np.uint8).reshape(r, 4)
    return out, fine


def tile_scales(s):
    """The scale bytes of an operand in the order of the product."""
    r, b = s.shape
    s = np.pad(s, ((0, -r % 128), (0, -b % 4)))
    return np.ascontiguousarray(s.reshape(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).transpose(0, 3, 2, 1, 4)).reshape(-1)


def untile_scales(t, r, b):
    rp, bp = r + -r % 128, b + -b % 4
    return t.reshape(rp // 128, bp // 4, 32, 4, 4).transpose(0, 3, 2, 1, 4).reshape(rp, bp)[:r, :b]


def mx4_operand(x):
    """(codes bytes [r, blocks * 16], tiled scale bytes, values) of fp64 rows x."""
    r, k = x.shape
    codes, scales = mx4_encode(np.pad(x, ((0, 0), (0, -k % 32))))
    return pack(codes), tile_scales(scales), mx4_decode(codes, scales)[:, :k]


def within(got, want64, tol64):
    """Whether every element of the torch tensor `got` lies between the roundings to its type of want - tol and want + tol:
    `tol` is what the fp32 arithmetic may be off, and the one rounding to the output type is held exactly."""
    import torch
    lo = torch.from_numpy(np.asarray(want64 - tol64, np.float64)).to(got.dtype)
    hi = torch.from_numpy(np.asarray(want64 + tol64, np.float64)).to(got.dtype)
    g = got.cpu()
    return bool(((g >= lo) & (g <= hi)).all())
