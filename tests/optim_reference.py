"""The optimizer step, its 8-bit moments and the gradient norm from their
definitions in include/flashrec.h, in numpy on the CPU: moments in fp32 with
each operation rounded (the definition fixes their bits), everything else in
64 bits.  Shares no code with the library."""
import math

import numpy as np

BLOCK = 256
U = 2.0 ** -24  # fp32 unit roundoff
MASK32, MASK64 = (1 << 32) - 1, (1 << 64) - 1
SPAN = {"m": 15, "v": 31}


def bf16_to_f32(bits):
    return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32)


def f32_to_bf16(x):
    """Bits of the nearest bf16, ties to even (finite values)."""
    b = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


# ---------------------------------------------------------------- random bits

def mix64(z):
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & MASK64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & MASK64
    return z ^ (z >> 31)


def random_bits(seed, step, tensor, index):
    """(for m, for v, for a weight): 16 bits each, of the elements `index` (uint64 array) of a tensor."""
    key = mix64((mix64((mix64(seed) + step) & MASK64) + tensor * 0x9E3779B97F4A7C15) & MASK64)
    lo, hi = key & MASK32, key >> 32
    i = np.asarray(index, np.uint64)
    p, low = i >> np.uint64(1), np.uint64(MASK32)
    u = ((p & low) * np.uint64(0x9E3779B1) + (np.uint64(lo) ^ (((p >> np.uint64(32)) * np.uint64(0x85EBCA77)) & low))) & low
    u ^= u >> np.uint64(16)
    u = (u * np.uint64(2891336453) + np.uint64(hi)) & low
    u ^= u >> np.uint64(15)
    odd = (i & np.uint64(1)).astype(bool)
    h = (u * np.where(odd, np.uint64(741103597), np.uint64(1597334677))) & low
    w = (u * np.uint64(747796405)) & low
    return ((h & np.uint64(0xFFFF)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64),
            np.where(odd, w & np.uint64(0xFFFF), w >> np.uint64(16)).astype(np.int64))


# ---------------------------------------------------------------- 8-bit moments

def _blocks(n):
    return [slice(a, min(a + BLOCK, n)) for a in range(0, n, BLOCK)]


def encode(x, kind, rnd=None):
    """(codes, exponents) of one tensor's moments; rnd: 16 random bits per element, None for the nearest."""
    bits = x.astype(np.float32).view(np.uint32).astype(np.int64)
    if kind == "v":
        bits = np.where(x < 0, 0, bits)
    mag = bits & 0x7FFFFFFF
    add = 0x7FFFF + ((mag >> 20) & 1) if rnd is None else rnd << 4
    codes, exps = np.zeros(x.size, np.uint8), np.zeros(-(-x.size // BLOCK), np.uint8)
    for k, s in enumerate(_blocks(x.size)):
        top = int(mag[s].max())
        if top >= 0x7F800000:
            exps[k] = 255
            continue
        e = max((top + 0xFFFFF) >> 23, SPAN[kind] + 1)
        exps[k] = e
        if e == 255:
            continue
        c = ((mag[s] + add[s]) >> 20) - 8 * (e - SPAN[kind])
        c = np.maximum(c, 0) if kind == "m" else np.where(mag[s] > 0, np.maximum(c, 1), 0)
        assert c.max() <= (127 if kind == "m" else 255)
        codes[s] = c + np.where((bits[s] >> 31 != 0) & (c > 0), 128, 0)
    return codes, exps


def decode(codes, exps, kind):
    """Values in 64 bits, from the meaning of a code: (1 + fraction / 8) 2^exponent."""
    out = np.zeros(codes.size)
    for k, s in enumerate(_blocks(codes.size)):
        e = int(exps[k])
        if e == 255:
            out[s] = math.nan
            continue
        c = codes[s].astype(np.int64)
        sign = np.where(c > 127, -1.0, 1.0) if kind == "m" else 1.0
        c = c & 127 if kind == "m" else c
        q = c + 8 * (max(e, SPAN[kind] + 1) - SPAN[kind])
        out[s] = np.where(c > 0, sign * (1 + (q % 8) / 8) * 2.0 ** (q // 8 - 127.0), 0.0)
    return out


# ---------------------------------------------------------------- the step

class Numbers:
    def __init__(self, lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=3, seed=7):
        self.lr, self.beta1, self.beta2, self.eps = lr, beta1, beta2, eps
        self.weight_decay, self.step, self.seed = weight_decay, step, seed


def moments(h, m, v, grad, scale=1.0):
    """New moments in fp32, bit for bit."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = grad.astype(f) * f(scale)
        m2 = m.astype(f) * f(h.beta1) + g * f(1 - h.beta1)
        v2 = v.astype(f) * f(h.beta2) + (g * g) * f(1 - h.beta2)
    return m2, v2


def step64(h, p, m, v, grad, scale=1.0, lr_scale=1.0, decay_scale=1.0):
    """(p, m, v, bounds on their fp32 errors) in 64 bits.

    The bounds count roundings, u = 2^-24 each, of the operation in fp32: the constants beta, 1 - beta, lr, ... have one of
    their own, a product adds one, a sum one of its result.  m: beta1, product, sum; 1 - beta1, scale's product, product, sum:
    at most 4 u of each term.  v: scale's product counts twice in g g: 6 u of each term.  The direction d = m / below: below
    has half of v's, the square root's, v_fix's and its product's, the sum's, eps's: 9 u; the quotient and m_fix and its
    product: 3 more; so (4 + 9 + 3) u of what m's terms give, one more to round.  Then decay (constant, its tensor factor, its
    product: 4 u with the sum), lr (constant, tensor factor: 3 u with the product), and p's own rounding."""
    g = grad.astype(np.float64) * scale
    m64, v64, p64 = (x.astype(np.float64) for x in (m, v, p))
    m2 = h.beta1 * m64 + (1 - h.beta1) * g
    v2 = h.beta2 * v64 + (1 - h.beta2) * g * g
    m_fix, v_fix = 1 / (1 - h.beta1 ** h.step), 1 / (1 - h.beta2 ** h.step)
    below = np.sqrt(v2 * v_fix) + h.eps
    terms = h.beta1 * np.abs(m64) + (1 - h.beta1) * np.abs(g)
    lr, decay = h.lr * lr_scale, h.weight_decay * decay_scale
    p2 = p64 - lr * (m2 * m_fix / below + decay * p64)
    tiny = 2.0 ** -149
    p_err = U * np.abs(p2) + lr * (20 * U * terms * m_fix / below + 7 * U * decay * np.abs(p64)) + 4 * tiny
    # (a product below 2^-126 is off by 2^-150 at most: v's square root then by half of that over itself, under eps)
    return p2, m2, v2, 1.01 * p_err, 1.01 * 4 * U * terms + 4 * tiny, 1.01 * 6 * U * v2 + 4 * tiny


def norm64(grads, max_norm, grad_scale):
    """(norm, scale, nonfinite) of a list of arrays, sums exact."""
    bad, parts = 0, []
    for g in grads:
        x = g.astype(np.float64)
        ok = np.isfinite(x)
        bad += int((~ok).sum())
        parts.append(x[ok] ** 2)
    total = math.fsum(np.concatenate(parts).tolist()) if parts else 0.0
    norm = grad_scale * math.sqrt(total)
    scale = 0.0 if bad else grad_scale * (max_norm / norm if norm > max_norm else 1.0)
    return norm, scale, bad
