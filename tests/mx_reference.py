"""Plain 64-bit implementation of the microscaled formats and of the operators on them, for the tests.  It shares no code with the
library; where a format rounds to 32 bits by definition, numpy's float32 does it."""
import numpy as np
import torch

MXFP4, NVFP4, MXINT8 = 0, 1, 2
BLOCK = {MXFP4: 32, NVFP4: 16, MXINT8: 32}
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(0x7F)])


def up(a, b):
    return -(-a // b) * b


def nearest_even(v, grid):
    """Indices into `grid` (ascending, codes by rank) of the nearest values, ties to the even index."""
    v = np.abs(np.asarray(v, dtype=np.float64))
    hi = np.clip(np.searchsorted(grid, v, side="left"), 1, len(grid) - 1)
    lo = hi - 1
    below, above = v - grid[lo], grid[hi] - v
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def quantize(x, fmt, largest=None):
    """x (rows, cols) float32 -> (elements as code numbers (rows, padded), scale bytes (rows, blocks))."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    b = BLOCK[fmt]
    pad = np.zeros((rows, up(cols, 32)), np.float32)
    pad[:, :cols] = x
    q = np.zeros(pad.shape, np.int16)
    s = np.zeros((rows, pad.shape[1] // b), np.uint8)
    if fmt == NVFP4:
        m = np.float32(largest)
        m = np.float32(2.0 ** -100) if m < np.float32(2.0 ** -100) else m
    with np.errstate(all="ignore"):
        for r in range(rows):
            for c in range(s.shape[1]):
                v = pad[r, c * b:(c + 1) * b]
                if not np.isfinite(v).all():
                    s[r, c] = 0x7F if fmt == NVFP4 else 0xFF
                    continue
                a = np.abs(v).max()
                if fmt == NVFP4:
                    t = a * (np.float32(448) / m)
                    code = 0x7F if np.isnan(t) else int(nearest_even(min(float(t), 448.0), E4M3))
                    s[r, c] = code
                    scale = np.float32(np.nan) if code == 0x7F else np.float32(E4M3[code])
                    z = v * ((np.float32(2688) / m) / scale) if scale > 0 else np.zeros(b, np.float32)
                else:
                    e = max((int(np.frexp(a)[1]) - 1 if a > 0 else -1000) - (2 if fmt == MXFP4 else 0), -127)
                    s[r, c] = e + 127
                    z = v.astype(np.float64) * 2.0 ** -e
                if fmt == MXINT8:
                    q[r, c * b:(c + 1) * b] = np.clip(np.rint(z * 64.0), -127, 127)
                else:
                    q[r, c * b:(c + 1) * b] = nearest_even(np.minimum(np.abs(z), 6.0), E2M1) + 8 * np.signbit(z)
    return q, s


def scale_values(s, fmt):
    """Scale bytes as 64-bit numbers, without NVFP4's tensor scale."""
    s = np.asarray(s)
    if fmt == NVFP4:
        return np.where(s == 0x7F, np.nan, E4M3[np.minimum(s, 0x7E)])
    return np.where(s == 0xFF, np.nan, 2.0 ** (s.astype(np.float64) - 127))


def values(q, s, fmt, cols=None):
    """What elements and scales stand for, in 64 bits, without NVFP4's tensor scale."""
    q = np.asarray(q)
    v = q / 64.0 if fmt == MXINT8 else E2M1[q & 7] * np.where(q & 8, -1.0, 1.0)
    with np.errstate(invalid="ignore"):
        return (v * np.repeat(scale_values(s, fmt), BLOCK[fmt], 1))[:, :cols]


def tensor_scale(largest):
    m = np.float32(largest)
    return np.float32(np.float32(2.0 ** -100) if m < np.float32(2.0 ** -100) else m) / np.float32(2688)


def pack(q, fmt):
    if fmt == MXINT8:
        return q.astype(np.int8)
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8)


def unpack(codes, fmt):
    if fmt == MXINT8:
        return codes.astype(np.int16)
    return np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1).astype(np.int16)


def scale_offset(fmt, r, c, scales_per_row):
    if fmt == MXINT8:
        return r * up(scales_per_row, 16) + c
    return (r // 128 * up(scales_per_row, 4) // 4 + c // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + c % 4


def lay_scales(s, fmt):
    rows, n = s.shape
    size = rows * up(n, 16) if fmt == MXINT8 else up(rows, 128) * up(n, 4)
    out = np.zeros(size, np.uint8)
    r, c = np.meshgrid(np.arange(rows), np.arange(n), indexing="ij")
    out[scale_offset(fmt, r, c, n)] = s
    return out


def device(x, fmt, largest=None):
    """A tensor quantized here, as device tensors (codes, scales) and as 64-bit values."""
    q, s = quantize(x, fmt, largest)
    return torch.from_numpy(pack(q, fmt)).cuda(), torch.from_numpy(lay_scales(s, fmt)).cuda(), values(q, s, fmt, np.shape(x)[1])


def act(x, kind):
    """(act(x), act'(x), z, the logistic function's value at z) in 64 bits; kind as the library's ACT_*."""
    x = np.asarray(x, dtype=np.float64)
    one = np.ones_like(x)
    if kind == 0:
        return x, one, one, one
    if kind == 1:
        return np.where(x > 0, x, 0.0), np.where(x > 0, 1.0, 0.0), one, one
    g = np.sqrt(8 / np.pi)
    z = x if kind == 2 else g * (x + 0.044715 * x ** 3)
    dz = one if kind == 2 else g * (1 + 3 * 0.044715 * x ** 2)
    with np.errstate(over="ignore"):
        s, n = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
        return x * s, s + np.nan_to_num(x * s * n * dz), z, s
