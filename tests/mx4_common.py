"""Microscaled 4-bit floating point in numpy: codes, scales and the values they stand for."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """(codes [rows][ldq] 0 .. 15, scales [rows][lds]) of x [rows][K], rounded to f32."""
    with np.errstate(over="ignore"):
        x = np.asarray(x).astype(np.float32).astype(np.float64)
    n, K = x.shape
    ldq, lds = (K + 63) // 64 * 64, (K + 255) // 256 * 8
    b = np.zeros((n, ldq))
    b[:, :K] = x
    b = b.reshape(n, ldq // 32, 32)
    amax = np.abs(b).max(2)
    bad = ~np.isfinite(amax)
    _, ex = np.frexp(np.where(bad | (amax == 0), 1.0, amax))
    e = np.where(amax == 0, -127, np.maximum(ex - 3, -127))
    v = np.where(bad[:, :, None], 0.0, b) * 2.0 ** -e[:, :, None].astype(np.float64)
    a = np.abs(v)
    d = np.abs(a[..., None] - VALUES)
    near = d.min(-1, keepdims=True) == d
    even = near & (np.arange(8) % 2 == 0)  # a tie lies between an even and an odd code
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1)) + 8 * np.signbit(v)
    code = np.where(bad[:, :, None], 0, code)
    sx = np.zeros((n, lds), np.uint8)
    sx[:, : ldq // 32] = np.where(bad, 255, e + 127)
    return code.reshape(n, ldq).astype(np.uint8), sx


def pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def unpack(xq):
    return np.stack([xq & 15, xq >> 4], -1).reshape(*xq.shape[:-1], -1)


def values(xq, sx):
    """[..][K] in f64; a scale of 255 makes its block NaN."""
    c = unpack(xq).astype(np.int64)
    s = sx[..., : c.shape[-1] // 32].astype(np.float64)
    s = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return (np.where(c >= 8, -1.0, 1.0) * VALUES[c % 8]) * np.repeat(s, 32, -1)
