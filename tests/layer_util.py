"""Plain 64-bit definitions of the layer operators (numpy / torch on the CPU),
shared by their tests."""
import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"bf16": 0, "f16": 1, "f32": 2}
FORMATS = {"int8": 0, "e4m3": 1}
# unit roundoff, and half the smallest step near zero
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}

# every e4m3 code's value, from its sign, exponent and mantissa
E4M3 = np.array([(-1) ** (c >> 7) * ((c & 7) * 2.0 ** -9 if (c >> 3 & 15) == 0 else
                                     (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                 for c in range(256)])


def layout(rows, cols):
    groups = -(-cols // 32)
    pitch, spitch = 32 * groups, 4 * -(-groups // 4)
    return groups, pitch, spitch, rows * (pitch + spitch)


def encode(x, fmt):
    """(codes as bytes [rows][pitch], scale bytes [rows][groups]) of f64 values,
    one group at a time, the exponent by trying them in order."""
    rows, cols = x.shape
    groups, pitch, _, _ = layout(rows, cols)
    codes = np.zeros((rows, pitch), np.uint8)
    scales = np.zeros((rows, groups), np.uint8)
    top, hi = (127.0, 121) if fmt == "int8" else (448.0, 119)
    if fmt == "e4m3":
        grid = E4M3[:127]  # 0 .. 448
    for g in range(groups):
        part = x[:, 32 * g:32 * g + 32]
        a = np.abs(part).max(1)
        e = np.full(rows, -110)
        with np.errstate(invalid="ignore"):
            for _ in range(110 + hi):
                e = np.where((a > top * 2.0 ** e) & (e < hi), e + 1, e)
        bad = ~np.isfinite(a)
        v = np.clip(np.where(bad[:, None], 0, part) / 2.0 ** e[:, None], -top, top)
        if fmt == "int8":
            c = np.rint(v).astype(np.int64) & 255
        else:
            m = np.abs(v)
            lo = np.clip(np.searchsorted(grid, m, side="right") - 1, 0, 126)
            up = np.minimum(lo + 1, 126)
            d, u = m - grid[lo], grid[up] - m
            c = np.where((d < u) | ((d == u) & (lo % 2 == 0)) | (up == lo), lo, up)
            c = c | np.where(np.signbit(v), 128, 0)
        codes[:, 32 * g:32 * g + part.shape[1]] = c
        scales[:, g] = np.where(bad, 255, e + 127)
        codes[:, 32 * g:32 * g + part.shape[1]][bad] = 0
    return codes, scales


def decode(codes, scales, cols, fmt):
    """f64 values of codes and scale bytes."""
    v = codes.astype(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(s, 32, 1))[:, :cols]


def kept(x, fmt):
    """What a checkpoint of f64 values stands for."""
    c, s = encode(x, fmt)
    return decode(c, s, x.shape[1], fmt)


def as_type(v, dtype):
    """f64 values in the type, f16 saturating, back in f64."""
    if dtype == "f16":
        v = np.clip(v, -65504, 65504)
    return torch.from_numpy(v).to(DTYPES[dtype]).double().numpy()


def buffer(codes, scales, device="cuda"):
    """The checkpoint buffer of codes and scale bytes."""
    rows, groups = scales.shape
    s = np.full((rows, 4 * -(-groups // 4)), 0xEE, np.uint8)  # what is past the groups is not read
    s[:, :groups] = scales
    return torch.from_numpy(np.concatenate([codes.reshape(-1), s.reshape(-1)])).to(device)


def turned(u, cos, sin, rot, half, back=False):
    """Rot u (or its transpose) over the last axis; cos, sin [..., rot / 2]."""
    if back:
        sin = -sin
    a = slice(0, rot // 2) if half else slice(0, rot, 2)
    b = slice(rot // 2, rot) if half else slice(1, rot, 2)
    y = u.copy()
    y[..., a] = u[..., a] * cos - u[..., b] * sin
    y[..., b] = u[..., b] * cos + u[..., a] * sin
    return y


def spread(u, cos, sin, rot, half):
    """The sum of the magnitudes of what a rotated element is made of."""
    u, cos, sin = np.abs(u), np.abs(cos), np.abs(sin)
    a = slice(0, rot // 2) if half else slice(0, rot, 2)
    b = slice(rot // 2, rot) if half else slice(1, rot, 2)
    y = u.copy()
    y[..., a] = u[..., a] * cos + u[..., b] * sin
    y[..., b] = u[..., b] * cos + u[..., a] * sin
    return y
