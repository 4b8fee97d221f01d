"""MXFP4 matrices in 64 bits, written from their definition alone (numpy, CPU)."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate((GRID, -GRID))


def held_bytes(cols):
    return -(-cols // 32) * 16


def scale_bytes(rows, cols):
    return -(-rows // 128) * -(-cols // 128) * 512


def scale_at(rows, cols):
    """Where the scale byte of every block of [rows, ceil(cols / 32)] lies."""
    r, b = np.arange(rows)[:, None], np.arange(-(-cols // 32))[None]
    return (r // 128 * -(-cols // 128) + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4


def blocks(x):
    rows, cols = x.shape
    return np.pad(x, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)


def scale_exponents(top):
    """Smallest e >= -127 with top <= 6 * 2^e (255 - 127 where top is not finite)."""
    with np.errstate(invalid="ignore"):
        m, k = np.frexp(top)  # top = m 2^k, m in [0.5, 1); 6 * 2^e = 0.75 * 2^(e + 3)
        e = np.where(m <= 0.75, k - 3, k - 2)
        e = np.where(top == 0, -127, np.maximum(e, -127))
    return np.where(np.isfinite(top), e, 128)


def nearest(a):
    """Codes of magnitudes a <= 6, to nearest, ties to the even code."""
    d = np.abs(a[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    hit = d == best
    low = hit.argmax(-1)
    high = 7 - hit[..., ::-1].argmax(-1)
    return np.where((low != high) & (low % 2 == 1), high, low)


def quantised(x):
    """Codes [rows, 32 blocks] and scale bytes [rows, blocks] of [rows, cols] values."""
    g = blocks(np.asarray(x, np.float64))
    top = np.abs(g).max(-1)
    e = scale_exponents(top)
    bad = e == 128
    with np.errstate(invalid="ignore"):
        q = g / np.ldexp(1.0, np.where(bad, 0, e))[..., None]
    q = np.where(bad[..., None], 0.0, q)
    code = nearest(np.abs(q)) + 8 * np.signbit(q)
    return code.reshape(g.shape[0], -1).astype(np.uint8), (e + 127).astype(np.uint8)


def packed(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def values(code, byte):
    """[rows, 32 blocks] in 64 bits."""
    s = np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))
    return (VALUES[code.reshape(byte.shape + (32,))] * s[..., None]).reshape(code.shape)


def laid_out(byte, cols, fill=0):
    """Scale bytes [rows, blocks] in memory; blocks behind the rows' ends are zeros, rows that do not exist `fill`."""
    rows = byte.shape[0]
    out = np.full(scale_bytes(rows, cols), fill, np.uint8)
    pad = -byte.shape[1] % 4
    whole = np.pad(byte, ((0, 0), (0, pad)))
    out[scale_at(rows, whole.shape[1] * 32)] = whole
    return out
