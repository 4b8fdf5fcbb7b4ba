"""The optimizer step over lists that its planning and its slower paths take apart: very many small tensors, runs of several
blocks per warp, buffers that start at different places, tiny second moments, long training against 64 bits."""
import math

import numpy as np
import pytest
import torch

import optim_reference as ref
from test_gpu_optim import Buffers, _plan, _record, _state, _wide

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _check_step(host, got, h, scale, rounding, factors=None):
    """Moments and codes of every tensor bit for bit, parameters within the bounds of optim_reference.step64."""
    n_tensors = len(host["weight"])
    for i in range(n_tensors):
        n = host["weight"][i].size
        if n == 0:
            continue
        rm, rv, _ = ref.random_bits(h.seed, h.step, i, np.arange(n)) if rounding else (None, None, None)
        eight = "m_exp" in host
        old = {k: host[k][i] for k in "mv"}
        if eight:
            old = {k: ref.decode(host[k][i], host[k + "_exp"][i], k).astype(np.float32) for k in "mv"}
        p, g = _wide(host.get("masters", host["weight"])[i]), _wide(host["grad"][i])
        m2, v2 = ref.moments(h, old["m"], old["v"], g, scale)
        p64, _, _, p_err, _, _ = ref.step64(h, p, old["m"], old["v"], g, scale)
        if eight:
            for k, x, r in (("m", m2, rm), ("v", v2, rv)):
                codes, exps = ref.encode(x, k, r)
                assert np.array_equal(got[k + "_exp"][i], exps) and np.array_equal(got[k][i], codes), (k, i)
        else:
            assert np.array_equal(got["m"][i].view(np.uint32), m2.view(np.uint32)), i
            assert np.array_equal(got["v"][i].view(np.uint32), v2.view(np.uint32)), i
        new = got["masters"][i] if "masters" in host else got["weight"][i]
        if new.dtype == np.float32:
            assert (np.abs(new - p64) <= p_err).all(), i
        else:  # one step of bf16 at most
            assert (np.abs(_wide(new) - p64) <= 2.0 ** -7 * np.abs(p64) + p_err).all(), i


def _hyper(h, rounding):
    return fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.step, h.seed, rounding)


@pytest.mark.parametrize("bits", [32, 8])
def test_very_many_small_tensors(bits):
    """Thousands of tensors of 0 to 9 elements, a large one among them: a warp's blocks lie in as many tensors."""
    r = np.random.default_rng(2)
    sizes = r.integers(0, 10, 3000).tolist()
    sizes[1500] = 40000
    sizes[2999] = 300
    host = _state(3, sizes, "f32", "f32", bits)
    b, plan = _plan(host, 0)
    h, scale = ref.Numbers(), 0.5
    plan.step(_hyper(h, 1), _record(scale))
    _check_step(host, {k: x.get() for k, x in b.items()}, h, scale, 1)
    norm, factor, bad = ref.norm64([_wide(x) for x in host["grad"]], 0.01, 0.25)
    rec = plan.clip(0.01, 0.25)
    got = [x.item() for x in fr.clip_view(rec)]
    assert abs(got[0] - norm) <= 33 * ref.U * norm and abs(got[1] - factor) <= 33 * ref.U * factor and got[2] == bad == 0


@pytest.mark.parametrize("param,grad", [("master", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
def test_runs_of_blocks(param, grad):
    """Enough blocks that a warp takes several of them in a row (7,296 times two and more), tensors ending inside the runs."""
    sizes = [2_000_003, 255, 256, 1_500_001, 77, 300_000, 512 * 256]
    host = _state(9, sizes, param, grad, 8)
    b, plan = _plan(host, 0)
    assert plan.n_blocks > 2 * 7296
    h, scale = ref.Numbers(seed=3), 0.37109375
    plan.step(_hyper(h, 1), _record(scale))
    _check_step(host, {k: x.get() for k, x in b.items()}, h, scale, 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["master", "bf16", "f32"])
def test_buffers_that_start_at_different_places(param, bits):
    """No common element at which all are on a vector's boundary, in a different way in each tensor."""
    sizes = [5000, 257, 70001, 1023]
    host = _state(13, sizes, param, "bf16", bits)
    shifts = {"weight": 1, "grad": 2, "masters": 5, "m": 0, "v": 3}
    b = {k: Buffers(v, shifts.get(k, 0)) for k, v in host.items()}
    names = {"weight": "weights", "grad": "grads"}
    plan = fr.OptPlan(**{names.get(k, k): x.tensors for k, x in b.items()})
    h, scale = ref.Numbers(), 0.5
    plan.step(_hyper(h, 1 if bits == 8 else 0), _record(scale))
    _check_step(host, {k: x.get() for k, x in b.items()}, h, scale, bits == 8)


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("param,grad", [("master", "f32"), ("master", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
def test_runs_of_blocks_have_the_same_bits_at_every_place(param, grad, bits, rounding):
    """As test_runs_of_blocks, three steps, every buffer or only some of them off the vectors' boundaries, by all numbers of
    bytes that a word has: each byte is the one that aligned buffers get, and none outside the tensors changes."""
    sizes = [2_000_003, 255, 256, 1_500_001, 77, 300_000, 512 * 256]
    host = _state(10, sizes, param, grad, bits)
    results = []
    for shifts in ({}, {"grad": 1}, {"m": 2, "v": 5, "weight": 3}, {"weight": 1, "grad": 3, "masters": 2, "m": 1, "v": 3}):
        b = {k: Buffers(v, shifts.get(k, 0)) for k, v in host.items()}
        names = {"weight": "weights", "grad": "grads"}
        plan = fr.OptPlan(**{names.get(k, k): x.tensors for k, x in b.items()})
        assert plan.n_blocks > 2 * 7296
        for t in range(1, 4):
            plan.step(_hyper(ref.Numbers(seed=3, step=t), rounding), _record(0.375))
        results.append({k: x.get() for k, x in b.items()})
    for other in results[1:]:
        for k, arrays in results[0].items():
            for x, y in zip(arrays, other[k]):
                assert x.tobytes() == y.tobytes(), k


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tiny_eps_keeps_the_formula_where_second_moments_are_subnormal(bits):
    """Gradients of 2^-66 to 2^-70 with eps = 1e-30: squares from 2^-132 to 2^-140, exact in fp32's subnormal numbers, as is the
    product with 1 - beta2 = 1/2; m and v of a first step are exact.  What is left is the square root (half a unit of v, none
    here), v_fix = sqrt(2), its product, eps, the quotient, m_fix = 2 and lr: 8 u."""
    n = 1000
    r = np.random.default_rng(8)
    g = (2.0 ** r.integers(-70, -65, n) * r.choice([-1, 1], n)).astype(np.float32)
    host = {"weight": [r.normal(size=n).astype(np.float32)], "grad": [g]}
    if bits == 8:
        host.update(m=[np.zeros(n, np.uint8)], v=[np.zeros(n, np.uint8)], m_exp=[np.zeros(4, np.uint8)], v_exp=[np.zeros(4, np.uint8)])
    else:
        host.update(m=[np.zeros(n, np.float32)], v=[np.zeros(n, np.float32)])
    b, plan = _plan(host, 0)
    h = ref.Numbers(lr=0.25, beta1=0.5, beta2=0.5, eps=1e-30, weight_decay=0.0, step=1)
    plan.step(_hyper(h, 0))
    want = host["weight"][0] - h.lr * np.sign(g)
    got = b["weight"].get()[0]
    assert (np.abs(got - want) <= ref.U * np.abs(want) + h.lr * 8 * ref.U + 1e-8).all()  # (eps under 2^-70: 1.2e-9)


def test_zero_gradients_and_states_stay_zero():
    n = 3000
    z = lambda t: [torch.zeros(n, dtype=t, device="cuda")]  # noqa: E731
    w = [torch.randn(n, device="cuda").bfloat16()]
    old = w[0].clone()
    m, v, me, ve = z(torch.uint8), z(torch.uint8), [torch.zeros(12, dtype=torch.uint8, device="cuda")], [torch.zeros(12, dtype=torch.uint8, device="cuda")]
    plan = fr.OptPlan(w, z(torch.bfloat16), m, v, m_exp=me, v_exp=ve)
    for t in range(1, 4):
        plan.step(fr.fr_adamw(0.1, 0.9, 0.999, 1e-8, 0.0, t, 5, fr.FR_ROUND_RANDOM), plan.clip())
    assert torch.equal(w[0], old) and not m[0].any() and not v[0].any()


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
def test_training_follows_64_bits(bits, rounding):
    """300 steps on a quadratic bowl with noisy gradients, beta2 = 0.999, against AdamW in 64 bits on the same noise.  32-bit
    moments follow it to 1e-4 of the distance travelled; 8-bit ones end as near the minimum (a factor of 1.5 on the final
    loss)."""
    n, steps = 4096, 300
    gen = torch.Generator(device="cuda").manual_seed(4)
    target = torch.randn(n, generator=gen, device="cuda", dtype=torch.float64)
    curve = torch.logspace(-2, 0, n, device="cuda", dtype=torch.float64)
    w = [torch.zeros(n, device="cuda")]
    g = [torch.zeros(n, device="cuda")]
    if bits == 8:
        st = dict(m=[torch.zeros(n, dtype=torch.uint8, device="cuda")], v=[torch.zeros(n, dtype=torch.uint8, device="cuda")],
                  m_exp=[torch.zeros(16, dtype=torch.uint8, device="cuda")], v_exp=[torch.zeros(16, dtype=torch.uint8, device="cuda")])
    else:
        st = dict(m=[torch.zeros(n, device="cuda")], v=[torch.zeros(n, device="cuda")])
    plan = fr.OptPlan(w, g, **st)
    p, m, v = (torch.zeros(n, device="cuda", dtype=torch.float64) for _ in range(3))
    for t in range(1, steps + 1):
        lr = 0.03 * (1 - (t - 1) / steps)
        noise = 0.05 * curve * torch.randn(n, generator=gen, device="cuda", dtype=torch.float64)
        g[0].copy_(curve * (w[0].double() - target) + noise)
        plan.step(fr.fr_adamw(lr, 0.9, 0.999, 1e-8, 0.01, t, 6, rounding))
        q = curve * (p - target) + noise
        m, v = 0.9 * m + 0.1 * q, 0.999 * v + 0.001 * q * q
        p = p - lr * ((m / (1 - 0.9 ** t)) / ((v / (1 - 0.999 ** t)).sqrt() + 1e-8) + 0.01 * p)
    loss = lambda x: float((curve * (x.double() - target).square()).mean())  # noqa: E731
    assert loss(p) < 0.2 * loss(torch.zeros_like(p))
    if bits == 32:
        assert float((w[0].double() - p).norm() / p.norm()) <= 1e-4
    assert loss(w[0]) <= 1.5 * loss(p)


def test_norm_that_fp32_cannot_hold():
    """Finite gradients whose norm is above fp32's range: the norm is infinite, the factor is not."""
    x = torch.full((100,), 3e38, device="cuda")
    rec = fr.OptPlan(grads=[x]).clip(max_norm=1e38)
    norm, scale, bad = (t.item() for t in fr.clip_view(rec))
    assert math.isinf(norm) and bad == 0 and abs(scale - 1e38 / 3e39) <= 2 * ref.U * (1e38 / 3e39)
    rec = fr.OptPlan(grads=[x]).clip()
    assert fr.clip_view(rec)[1].item() == 1.0
