"""The 8-bit moments of tests/optim_reference.py over all blocks of a long tensor at once (its loop over blocks takes 20 us each)."""
import numpy as np

from optim_reference import BLOCK, SPAN


def encode(x, kind, rnd=None):
    n, rows = x.size, -(-x.size // BLOCK)

    def blocks(a):
        out = np.zeros(rows * BLOCK, np.int64)
        out[:n] = a
        return out.reshape(rows, BLOCK)

    bits = x.astype(np.float32).view(np.uint32).astype(np.int64)
    if kind == "v":
        bits = np.where(x < 0, 0, bits)
    add = 0x7FFFF + ((bits >> 20) & 1) if rnd is None else rnd << 4
    mag, add = blocks(bits & 0x7FFFFFFF), blocks(add)
    top = mag.max(1, keepdims=True)
    exps = np.where(top >= 0x7F800000, 255, np.maximum((top + 0xFFFFF) >> 23, SPAN[kind] + 1))
    c = ((mag + add) >> 20) - 8 * (exps - SPAN[kind])
    c = np.maximum(c, 0) if kind == "m" else np.where(mag > 0, np.maximum(c, 1), 0)
    c = np.where(exps == 255, 0, c)
    assert c.max(initial=0) <= (127 if kind == "m" else 255)
    c = c.reshape(-1)[:n]
    return (c + np.where((bits >> 31 != 0) & (c > 0), 128, 0)).astype(np.uint8), exps.reshape(-1).astype(np.uint8)


def decode(codes, exps, kind):
    """In fp32, which holds every code's value."""
    e = np.maximum(exps.astype(np.int64), SPAN[kind] + 1).repeat(BLOCK)[:codes.size]
    c = codes.astype(np.int64)
    q = (c & 127 if kind == "m" else c) + 8 * (e - SPAN[kind])
    x = np.where((c & 127 if kind == "m" else c) > 0, (q << 20).astype(np.uint32).view(np.float32), np.float32(0))
    if kind == "m":
        x = np.where(c > 127, -x, x)
    return np.where(exps.repeat(BLOCK)[:codes.size] == 255, np.float32(np.nan), x).astype(np.float32)
