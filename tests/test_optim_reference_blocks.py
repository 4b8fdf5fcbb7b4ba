"""tests/optim_reference_blocks.py gives what tests/optim_reference.py gives (no GPU)."""
import numpy as np
import pytest

import optim_reference as ref
import optim_reference_blocks as blocks


@pytest.mark.parametrize("rounding", ["nearest", "random"])
@pytest.mark.parametrize("spread", [0.0, 3.0, 15.0, 45.0])
@pytest.mark.parametrize("kind", ["m", "v"])
def test_equal_block_by_block(kind, spread, rounding):
    r = np.random.default_rng(int(spread) + len(rounding))
    for n in (0, 1, 255, 256, 257, 5000):
        x = np.clip(r.normal(size=n) * np.exp(r.normal(size=n) * spread), -1e38, 1e38).astype(np.float32)
        x[::5] = 0
        if n > 1000:
            x[256:512] = 0
            x[600], x[900], x[1300], x[1600], x[1999] = 1e-42, np.nan, np.inf, 3.3e38, -np.inf
        if kind == "v":
            x = np.abs(x)
            x[3:4] = -1.0
        rnd = ref.random_bits(9, 2, 1, np.arange(n))[0 if kind == "m" else 1] if rounding == "random" else None
        want, got = ref.encode(x, kind, rnd), blocks.encode(x, kind, rnd)
        for a, b in zip(want, got):
            assert a.dtype == b.dtype and np.array_equal(a, b)
        assert np.array_equal(blocks.decode(*got, kind).astype(np.float64), ref.decode(*want, kind), equal_nan=True)


@pytest.mark.parametrize("kind", ["m", "v"])
def test_every_code_under_every_exponent(kind):
    codes, exps = np.tile(np.arange(256, dtype=np.uint8), 256), np.arange(256, dtype=np.uint8)
    assert np.array_equal(blocks.decode(codes, exps, kind).astype(np.float64), ref.decode(codes, exps, kind), equal_nan=True)
