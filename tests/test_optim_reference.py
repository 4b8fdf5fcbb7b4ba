"""The CPU reference of the optimizer step is itself right (no GPU): against
closed forms, brute force over all codes, and statistics of the random bits."""
import math

import numpy as np
import pytest

import optim_reference as ref


@pytest.mark.parametrize("kind", ["m", "v"])
def test_nearest_code_is_the_nearest_value(kind):
    r = np.random.default_rng(1)
    x = np.abs(r.normal(size=256) * np.exp(r.normal(size=256) * 4)).astype(np.float32)
    codes, exps = ref.encode(x, kind)
    top = 128 if kind == "m" else 256
    values = ref.decode(np.arange(top, dtype=np.uint8), np.repeat(exps, 1), kind)
    got = ref.decode(codes, exps, kind)
    for a, b in zip(x.astype(np.float64), got):
        best = np.abs(values - a).min()
        if a < values[1]:
            assert b in (0.0, values[1]) if kind == "m" else b == values[1]
        else:
            assert abs(b - a) == best


@pytest.mark.parametrize("kind", ["m", "v"])
def test_largest_element_of_a_block_keeps_its_precision(kind):
    for e in list(range(-120, 127, 13)) + [126]:
        for f in (1.0, 1.5, 1.874, 1.876, 1.95):
            x = np.zeros(256, np.float32)
            x[3] = np.float32(f) * np.float32(2.0) ** e
            codes, exps = ref.encode(x, kind)
            value = ref.decode(codes, exps, kind)
            assert abs(value[3] - x[3]) <= x[3] / 16 and not value[:3].any()


def test_moments_and_step_of_known_numbers():
    h = ref.Numbers(lr=0.1, beta1=0.5, beta2=0.75, eps=1e-12, weight_decay=0.0, step=1)
    m, v = ref.moments(h, np.zeros(2), np.zeros(2), np.array([4.0, -2.0], np.float32), 0.5)
    assert m.tolist() == [1.0, -0.5] and v.tolist() == [1.0, 0.25]
    p = ref.step64(h, np.array([1.0, 1.0]), np.zeros(2), np.zeros(2), np.array([4.0, -2.0]), 0.5)[0]
    assert np.allclose(p, [0.9, 1.1], atol=1e-11)  # a first step goes by lr against the gradient's sign
    h.weight_decay = 0.5
    p = ref.step64(h, np.array([1.0, 1.0]), np.zeros(2), np.zeros(2), np.array([4.0, -2.0]), 0.5, 2.0, 0.5)[0]
    assert np.allclose(p, [1 - 0.2 * 1.25, 1 - 0.2 * -0.75], atol=1e-11)


def test_norm_of_known_numbers():
    gs = [np.array([3.0, np.nan], np.float32), np.array([4.0], np.float32)]
    assert ref.norm64(gs, 1.0, 1.0) == (5.0, 0.0, 1)
    assert ref.norm64([np.array([3.0, 4.0], np.float32)], 2.5, 0.5) == (2.5, 0.5, 0)
    assert ref.norm64([np.array([3.0, 4.0], np.float32)], 1.25, 0.5) == (2.5, 0.25, 0)
    assert ref.norm64([], 1.0, 0.5) == (0.0, 0.5, 0)


def test_random_bits_are_uniform_and_unrelated():
    """Over 2^20 elements: every bit is set half of the time, high bytes are uniform (chi-squared), and neighbours, tensors,
    steps, seeds and the three numbers of an element are uncorrelated, all within 5 standard deviations."""
    n = 1 << 20
    i = np.arange(n)
    streams = list(ref.random_bits(7, 3, 0, i))
    streams += [ref.random_bits(8, 3, 0, i)[1], ref.random_bits(7, 4, 0, i)[1], ref.random_bits(7, 3, 1, i)[1],
                ref.random_bits(7, 3, 0, i + (1 << 33))[1]]
    for s in streams:
        for b in range(16):
            assert abs(int(((s >> b) & 1).sum()) - n / 2) <= 5 * math.sqrt(n) / 2
        counts = np.bincount(s >> 8, minlength=256)
        chi2 = float(((counts - n / 256) ** 2 / (n / 256)).sum())
        assert abs(chi2 - 255) <= 5 * math.sqrt(2 * 255)
    unit = [(s - 32767.5) / math.sqrt((65536 ** 2 - 1) / 12) for s in streams]
    for a in range(len(unit)):
        for b in range(a):
            assert abs(float((unit[a] * unit[b]).mean())) <= 5 / math.sqrt(n), (a, b)
        for lag in (1, 2, 3, 8, 16, 32, 256):
            assert abs(float((unit[a][lag:] * unit[a][:-lag]).mean())) <= 5 / math.sqrt(n - lag), (a, lag)
