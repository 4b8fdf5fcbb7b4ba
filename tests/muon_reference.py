"""The orthogonalised update's definition in 64 bits (include/flashrec.h), in numpy."""
import numpy as np

USUAL = ((3.4445, -4.7750, 2.0315),) * 5
# A rounding to fp16 is off by 2^-11 at most.  An iteration has three, of X, of X X^T and of the polynomial in it, each of a
# relative size of one in what it enters and passed on with a gain of about one (the parts that would grow go in unrounded):
# the worst case adds them up.
ROUNDING = 3 * 2.0 ** -11
# Two fp16 numbers hold what one leaves to 2^-11 of that, and the product of the second ones, left out, is as small.
SPLIT_ROUNDING = 3 * 2 * 2.0 ** -22


def orthogonal(g, coefficients=USUAL):
    x = np.asarray(g, dtype=np.float64)
    with np.errstate(all="ignore"):
        top = np.abs(x).max() if x.size else 0.0
        if top == 0.0:
            return np.zeros_like(x)
        x = x / top
        x = x / np.sqrt((x * x).sum())
        tall = x.shape[0] > x.shape[1]
        if tall:
            x = x.T
        for a, b, c in coefficients:
            s = x @ x.T
            x = a * x + (b * s + c * (s @ s)) @ x
    return x.T if tall else x


def bound(coefficients=USUAL, split=False, shape=(0, 0)):
    """Of |error| / |O|, 2-norms over all elements.  split: products of both halves; the tensor cores add 16 products at a time,
    each sum off by 2^-23 at most (it may be cut off), in the three products of an iteration."""
    each = SPLIT_ROUNDING + 3 * (3 * (max(shape) // 16 + 8)) * 2.0 ** -23 if split else ROUNDING
    return each * len(coefficients)


def matrix(rng, rows, cols, kind="half"):
    """Matrices as gradients are: noise and a part of low rank, rows of different sizes; or one of the hard spectra."""
    g = rng.normal(size=(rows, cols))
    r = max(1, min(rows, cols) // 16)
    low = rng.normal(size=(rows, r)) @ rng.normal(size=(r, cols)) / np.sqrt(r)
    if kind == "half":
        g = (g + low) * np.exp(0.3 * rng.normal(size=(rows, 1)))
    elif kind == "lowrank":
        g = low
    elif kind == "decay":
        k = min(rows, cols)
        g = (rng.normal(size=(rows, k)) * np.exp(-6.0 * np.arange(k) / k)) @ rng.normal(size=(k, cols))
    elif kind == "spiky":
        g = g * np.exp(1.5 * rng.normal(size=(rows, 1)))
    return (g * 1e-3).astype(np.float32)
