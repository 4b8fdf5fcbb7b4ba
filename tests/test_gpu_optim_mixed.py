"""One list of every kind of tensor at once: weights, gradients and moments of all types, at all places, in random order."""
import numpy as np
import pytest
import torch

import optim_reference as ref
from test_gpu_optim import Buffers, _record, _state, _wide
from test_gpu_optim_lists import _check_step

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

KINDS = [(p, g, b) for p in ("master", "bf16", "f32") for g in ("bf16", "f32") for b in (32, 8)]


@pytest.mark.parametrize("eps", [1e-8, 1e-30])
@pytest.mark.parametrize("seed", range(4))
def test_a_list_of_all_kinds(seed, eps):
    """Twelve kinds, seven sizes of each, offsets of 0 to 8 elements in every buffer; lists of None where a tensor has no master
    or exponents.  Each tensor's result is that of its definition, by its own index in the list; the norm is the whole list's."""
    r = np.random.default_rng(seed)
    made = []  # (host arrays, buffers) of one tensor
    for param, grad, bits in KINDS:
        common = int(r.integers(0, 9))
        for n in (0, 1, 255, 256, 300, int(r.integers(257, 3000)), int(r.integers(3000, 40000))):
            host = _state(int(r.integers(1 << 30)), [n], param, grad, bits)
            place = [common if r.random() < 0.6 else int(r.integers(0, 9)) for _ in host]
            made.append((host, {k: Buffers(v, 0 if k.endswith("_exp") else s) for (k, v), s in zip(host.items(), place)}))
    made = [made[i] for i in r.permutation(len(made))]
    names = {"weights": "weight", "grads": "grad", "masters": "masters", "m": "m", "v": "v", "m_exp": "m_exp", "v_exp": "v_exp"}
    lists = {k: [b[x].tensors[0] if x in b else None for _, b in made] for k, x in names.items()}
    plan = fr.OptPlan(**lists)
    norm, scale, bad = ref.norm64([_wide(h["grad"][0]) for h, _ in made], 0.125, 0.5)
    rec = plan.clip(0.125, 0.5)
    got = [x.item() for x in fr.clip_view(rec)]
    assert abs(got[0] - norm) <= 33 * ref.U * norm and abs(got[1] - scale) <= 33 * ref.U * scale and got[2] == bad == 0
    h, scale = ref.Numbers(eps=eps, seed=seed), 0.37109375
    hyper = fr.fr_adamw(h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.step, h.seed, fr.FR_ROUND_RANDOM)
    plan.step(hyper, _record(scale))
    torch.cuda.synchronize()
    for i, (host, b) in enumerate(made):  # alone, but with the index that random bits go by
        n = host["weight"][0].size
        pad = {k: [np.empty(0, v[0].dtype)] * i + v for k, v in host.items()}
        out = {k: [np.empty(0, x.dtype)] * i + x.get() for k, x in b.items()}
        _check_step(pad, out, h, scale, 1 if "m_exp" in host else 0)
        if "masters" in host and n:
            assert np.array_equal(out["weight"][i], ref.f32_to_bf16(out["masters"][i])), i
