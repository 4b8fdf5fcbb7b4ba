"""An eps below 2^-39 v_fix: the square root and the quotient are the correctly rounded ones, in every class of the step."""
import numpy as np
import pytest

import optim_reference as ref
from test_gpu_optim import SIZES, Buffers, _plan, _record, _state, _wide
from test_gpu_optim_lists import _check_step

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

# elements past a 512-byte boundary: none; the same one in every buffer; gradients alone (launches of their own), and in
# each buffer another
PLACES = [{}, dict.fromkeys(("weight", "grad", "masters", "m", "v"), 1), {"grad": 1},
          {"weight": 1, "grad": 2, "masters": 5, "m": 1, "v": 3}]


def _placed(host, place):
    b = {k: Buffers(v, place.get(k, 0)) for k, v in host.items()}
    names = {"weight": "weights", "grad": "grads"}
    return b, fr.OptPlan(**{names.get(k, k): x.tensors for k, x in b.items()})


@pytest.mark.parametrize("place", PLACES, ids=["aligned", "one offset", "gradients off", "all off"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("master", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("master", "f32")])
@pytest.mark.parametrize("eps", [1e-15, 1e-30])
def test_ordinary_gradients(eps, param, grad, bits, place):
    """Gradients whose squares are normal numbers: the bounds of optim_reference.step64, with both roundings' codes."""
    host = _state(41, SIZES + [70001], param, grad, bits)
    for rounding in {0, 1 if bits == 8 else 0}:
        b, plan = _placed(host, place)
        h, scale = ref.Numbers(eps=eps), 0.5
        assert eps < 2.0 ** -39 / np.sqrt(1 - h.beta2 ** h.step)
        plan.step(fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.step, h.seed, rounding), _record(scale))
        got = {k: x.get() for k, x in b.items()}
        _check_step(host, got, h, scale, rounding)
        if param == "master":
            for w, x in zip(got["weight"], got["masters"]):
                assert np.array_equal(w, ref.f32_to_bf16(x))


@pytest.mark.parametrize("place", PLACES, ids=["aligned", "one offset", "gradients off", "all off"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("master", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_subnormal_second_moments(param, grad, bits, place):
    """Gradients of 2^-66 to 2^-70, which bf16 holds, with eps = 1e-30: squares from 2^-132 to 2^-140, exact in fp32's
    subnormal numbers, as is the product with 1 - beta2 = 1/2; m and v of a first step are exact, and so are 8-bit codes'
    inputs.  The parameter moves by lr against the gradient's sign; what is left is the square root, v_fix = sqrt(2), its
    product, eps, the quotient, m_fix = 2 and lr: 8 u, and eps itself: 1.2e-9 of a denominator of 2^-70 and more."""
    n = 1000
    r = np.random.default_rng(8)
    g = (2.0 ** r.integers(-70, -65, n) * r.choice([-1, 1], n)).astype(np.float32)
    w = ref.f32_to_bf16(r.normal(size=n).astype(np.float32))
    host = {"weight": [w if param != "f32" else _wide(w)], "grad": [g if grad == "f32" else ref.f32_to_bf16(g)]}
    assert np.array_equal(_wide(host["grad"][0]), g)
    if param == "master":
        host["masters"] = [_wide(w) + np.float32(1e-5)]
    if bits == 8:
        host.update(m=[np.zeros(n, np.uint8)], v=[np.zeros(n, np.uint8)], m_exp=[np.zeros(4, np.uint8)], v_exp=[np.zeros(4, np.uint8)])
    else:
        host.update(m=[np.zeros(n, np.float32)], v=[np.zeros(n, np.float32)])
    b, plan = _placed(host, place)
    h = ref.Numbers(lr=0.25, beta1=0.5, beta2=0.5, eps=1e-30, weight_decay=0.0, step=1)
    plan.step(fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.step, h.seed, 0))
    got = {k: x.get()[0] for k, x in b.items()}
    p = _wide(host.get("masters", host["weight"])[0]).astype(np.float64)
    want = p - h.lr * np.sign(g)
    err = ref.U * np.abs(want) + h.lr * 8 * ref.U + 1e-8
    new = _wide(got["masters" if param == "master" else "weight"])
    if param == "bf16":  # between the roundings of both ends of what p may be
        assert (_wide(ref.f32_to_bf16((want - err).astype(np.float32))) <= new).all()
        assert (new <= _wide(ref.f32_to_bf16((want + err).astype(np.float32)))).all()
    else:
        assert (np.abs(new - want) <= err).all()
    if param == "master":
        assert np.array_equal(got["weight"], ref.f32_to_bf16(new))
    m2, v2 = ref.moments(h, np.zeros(n), np.zeros(n), g)
    for k, x in (("m", m2), ("v", v2)):
        if bits == 8:
            codes, exps = ref.encode(x, k)
            assert np.array_equal(got[k + "_exp"], exps) and np.array_equal(got[k], codes), k
        else:
            assert np.array_equal(got[k].view(np.uint32), x.view(np.uint32)), k


def test_the_two_arithmetics_agree_where_the_limit_lies():
    """Of one list stepped with an eps on either side of the limit, moments are the same bits and parameters differ by their
    bounds' sum at most (which moves by less than u with eps)."""
    host = _state(43, SIZES, "f32", "f32", 8)
    h, scale = ref.Numbers(beta2=0.999, step=1), 0.5
    limit = np.float32(2.0 ** -39) * np.float32(1 / np.sqrt(1 - h.beta2))
    sides = []
    for eps in (float(limit), float(np.nextafter(limit, np.float32(0)))):
        b, plan = _plan(host, 0)
        plan.step(fr.fr_adamw(h.lr, h.beta1, h.beta2, eps, h.weight_decay, h.step, h.seed, 1), _record(scale))
        sides.append({k: x.get() for k, x in b.items()})
        h.eps = eps
        _check_step(host, sides[-1], h, scale, 1)
    for k in ("m", "v", "m_exp", "v_exp"):
        assert all(np.array_equal(x, y) for x, y in zip(sides[0][k], sides[1][k])), k
