"""What random rounding of 8-bit moments keeps and what it does not, over all 65,536 random numbers of an element (no GPU; that the
library's codes are this reference's is tested on the GPU)."""
import numpy as np
import pytest

import optim_reference as ref


def _mean(x, kind, top):
    """Mean value that x (fp32, positive) is coded to in a block whose largest element is `top`."""
    rnd = np.arange(1 << 16)
    total = 0.0
    for part in rnd.reshape(-1, 128):  # 128 of them in a block's first elements, its largest behind
        block = np.full(129, x, np.float32)
        block[128] = top
        codes, exps = ref.encode(block, kind, np.append(part, 0))
        total += ref.decode(codes, exps, kind)[:128].sum()
    return total / rnd.size


@pytest.mark.parametrize("kind", ["m", "v"])
def test_the_mean_is_exact_from_code_1_on(kind):
    """The cut takes 16 of the 20 bits below it into account: the mean is off by 2^-16 of a code's step at most."""
    low = 1.125 * 2.0 ** -ref.SPAN[kind]  # code 1 in a block whose largest element is 1: base pattern 2^-span, a step of an eighth
    for x in (low, 1.06 * low, 1.111 * low, 1.2 * low, 2.7 * low, 1e-3, 0.3337, 0.99, 1.0):
        x = float(np.float32(x))
        step = 2.0 ** np.floor(np.log2(x)) / 8
        assert abs(_mean(x, kind, 1.0) - x) <= step * 2.0 ** -16 + 2.0 ** -40 * x, x


def test_first_moments_below_code_1_lose():
    """Between the base's value and code 1: code 1 with the probability that lies between them, else zero.  Below the base: zero.
    (Of the part's 20 bits the random number sees 16: so many of the 65,536 numbers carry.)"""
    base, code = 2.0 ** -15, 1.125 * 2.0 ** -15
    for part in (0.0, 0.25, 0.48, 0.5, 0.96875):
        x = base + part * (code - base)
        carries = (int(np.float32(x).view(np.uint32)) & 0xFFFFF) >> 4
        assert abs(carries / 65536 - part) <= 2.0 ** -16
        assert _mean(x, "m", 1.0) == carries / 65536 * code
    for x in (0.999 * base, 0.5 * base, 2.0 ** -40):
        assert _mean(x, "m", 1.0) == 0.0


def test_second_moments_below_code_1_are_raised_to_it():
    code = 1.125 * 2.0 ** -31
    for x in (0.99 * code, 0.9 * code, 2.0 ** -31, 2.0 ** -40, 2.0 ** -100):
        assert _mean(x, "v", 1.0) == code
    assert _mean(0.0, "v", 1.0) == 0.0
