"""The record of the norm where fp32 is at its ends: norms and quotients that are subnormal there, factors that are not."""
import math

import numpy as np
import pytest
import torch

import optim_reference as ref

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")


@pytest.mark.parametrize("value,n,grad_scale,max_norm", [
    (1e8, 10000, 2.0 ** 20, 1e-26),      # a quotient of 1e-42, a factor of 1e-36
    (1e5, 300, 2.0 ** 40, 3e-38),        # a quotient that is zero in fp32
    (1e-5, 100, 1e-36, 1e-41),           # a norm of 1e-40
    (1e-5, 77, 3e-38, 1e-42),
    (3.0, 1000, 1e-42, 2e-41),           # everything subnormal
    (1.0, 3, 1e-44, 1e-45),
    (0.7, 3, 2.0 ** -149, 2.0 ** -149),
    (1.0, 4, 2.0 ** -149, 1.0),          # not clipped
    (1e-5, 100, 1e-36, math.inf),
    (1e18, 1000, 1e18, 1e-3),            # a norm above 1e37
])
def test_the_factor_keeps_its_precision_at_the_ends_of_fp32(value, n, grad_scale, max_norm):
    """Bounds as for ordinary norms: 33 u of the norm (64 squares in fp32, the rounding), one more rounding for the factor's
    own; what is below 2^-126 is rounded to a multiple of 2^-149 (by half of one at most)."""
    g = (np.random.default_rng(5).normal(size=n) * value).astype(np.float32)
    grad_scale, max_norm = float(np.float32(grad_scale)), float(np.float32(max_norm))
    record = fr.OptPlan(grads=[torch.from_numpy(g).cuda()]).clip(max_norm, grad_scale)
    norm, scale, bad = ref.norm64([g], max_norm, grad_scale)
    got_norm, got_scale, got_bad = (x.item() for x in fr.clip_view(record))
    assert got_bad == bad == 0
    assert abs(got_norm - norm) <= 33 * ref.U * norm + 2.0 ** -150
    assert abs(got_scale - scale) <= 34 * ref.U * scale + 2.0 ** -150


@pytest.mark.parametrize("size", [1e-30, 1.0, 1e25, 1e36])
def test_records_of_several_plans_joined_in_64_bits_are_the_whole_list_s(size):
    """Squares of norms, added in fp64 as the header says, against one plan over all tensors: 33 u for each."""
    r = np.random.default_rng(6)
    gs = [(r.normal(size=n) * size).astype(np.float32) for n in (5000, 70001, 3)]
    tensors = [torch.from_numpy(g).cuda() for g in gs]
    parts = [fr.clip_view(fr.OptPlan(grads=[t]).clip(grad_scale=0.5)) for t in tensors]
    norm = torch.cat([p[0] for p in parts]).double().square().sum().sqrt().item()
    whole, factor, bad = (x.item() for x in fr.clip_view(fr.OptPlan(grads=tensors).clip(size, 0.5)))
    want, want_factor, _ = ref.norm64(gs, float(np.float32(size)), 0.5)
    assert abs(norm - want) <= 34 * ref.U * want and abs(whole - want) <= 33 * ref.U * want
    assert abs(0.5 * np.float32(size) / norm - factor) <= 70 * ref.U * factor and bad == sum(p[2].item() for p in parts) == 0
