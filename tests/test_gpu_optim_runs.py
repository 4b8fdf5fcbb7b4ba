"""Runs of 3 and of 8 blocks per warp, the most there are, in which each shared-memory slot of a warp is used again and again:
every block differs from every other, tensors end inside the runs, and every byte of the result is compared."""
import functools

import numpy as np
import pytest
import torch

import optim_reference as ref
import optim_reference_blocks as blocks
from test_gpu_optim import Buffers, _record, _state, _wide

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

ROUND = 7296  # blocks of a launch for each one that a warp takes: two waves of 3 CTAs of 8 warps on 152 SMs
MOST = 8
PLACES = {  # elements past a 512-byte boundary (and one to four more in later tensors)
    "aligned": {},
    "gradients off": {"grad": 1},
    "states off": {"m": 2, "v": 5, "weight": 3},
    "all off": {"weight": 1, "grad": 3, "masters": 2, "m": 1, "v": 3},
}


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _sizes(run):
    t = run * ROUND * 256 * 101 // 1000  # a tenth of the elements, and 1% more
    return [4 * t + 3, 255, 300, 3 * t + 1, 77, 256, 2 * t - 1, t + 7]


@functools.lru_cache(maxsize=1)
def _host(run, param, grad):
    host = _state(run, _sizes(run), param, grad, 32)
    for k in "mv":
        pairs = [blocks.encode(x, k) for x in host[k]]
        host[k], host[k + "_exp"] = [c for c, _ in pairs], [e for _, e in pairs]
    return host


def _train(host, place, rounding, steps):
    """The buffers' contents after each of the steps."""
    b = {k: Buffers(v, 0 if k.endswith("_exp") else PLACES[place].get(k, 0)) for k, v in host.items()}
    names = {"weight": "weights", "grad": "grads"}
    plan = fr.OptPlan(**{names.get(k, k): x.tensors for k, x in b.items()})
    out = []
    for t in range(3, 3 + steps):
        h = ref.Numbers(step=t)
        plan.step(fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, t, h.seed, rounding), _record(0.37109375))
        out.append({k: x.get() for k, x in b.items()})
    return out


def _launched_run(sizes, odd):
    """Blocks per warp in the launch that has the long tensors (off the vectors' boundaries: those of a whole block and more)."""
    n = sum(-(-s // 256) for s in sizes if s >= 256 or not odd)
    return min(n // ROUND, MOST)


@pytest.mark.parametrize("run,rounding", [(3, 1), (8, 0), (8, 1)])
@pytest.mark.parametrize("param,grad", [("bf16", "bf16"), ("master", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_runs_are_the_definition_at_every_place(param, grad, run, rounding):
    """bf16 weights and gradients alone take three slots a warp, the others two."""
    sizes = _sizes(run)
    assert _launched_run(sizes, False) == _launched_run(sizes, True) == run
    host = _host(run, param, grad)
    first, second = _train(host, "aligned", rounding, 2)
    h, scale = ref.Numbers(step=3), 0.37109375
    for i, n in enumerate(sizes):
        old = {k: blocks.decode(host[k][i], host[k + "_exp"][i], k) for k in "mv"}
        p, g = _wide(host.get("masters", host["weight"])[i]), _wide(host["grad"][i])
        m2, v2 = ref.moments(h, old["m"], old["v"], g, scale)
        rnd = ref.random_bits(h.seed, h.step, i, np.arange(n)) if rounding else (None, None, None)
        for k, x, r in (("m", m2, rnd[0]), ("v", v2, rnd[1])):
            codes, exps = blocks.encode(x, k, r)
            assert np.array_equal(first[k + "_exp"][i], exps) and np.array_equal(first[k][i], codes), (k, i)
        p64, _, _, p_err, _, _ = ref.step64(h, p, old["m"], old["v"], g, scale)
        if param == "bf16":  # one step of bf16 at most
            assert (np.abs(_wide(first["weight"][i]) - p64) <= 2.0 ** -7 * np.abs(p64) + p_err).all(), i
            continue
        new = first["masters" if param == "master" else "weight"][i]
        assert (np.abs(new - p64) <= p_err).all(), i
        if param == "master":
            assert np.array_equal(first["weight"][i], ref.f32_to_bf16(new)), i
    for place in list(PLACES)[1:]:
        other = _train(host, place, rounding, 2)[1]
        for k, arrays in second.items():
            for x, y in zip(arrays, other[k]):
                assert x.tobytes() == y.tobytes(), (place, k)
