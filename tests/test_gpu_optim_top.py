"""8-bit moments at the top of fp32's range: which finite values a block holds, and what a gradient does whose square they
do not."""
import numpy as np
import pytest
import torch

import optim_reference as ref

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

LAST = 0x7F700000  # 1.875 * 2^127


@pytest.mark.parametrize("rounding", [fr.FR_ROUND_NEAREST, fr.FR_ROUND_RANDOM])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("pattern,lost", [(LAST - 1, False), (LAST, False), (LAST + 1, True), (0x7F7FFFFF, True), (0x7F800000, True)])
def test_a_block_holds_values_up_to_the_largest_codes(pattern, lost, aligned, rounding):
    x = np.full(700, 2.0 ** 120, np.float32)
    x[300] = np.uint32(pattern).view(np.float32)
    off = 0 if aligned else 1
    m, v, back_m, back_v = (torch.zeros(701, device="cuda")[off:off + 700] for _ in range(4))
    codes = [torch.zeros(701, dtype=torch.uint8, device="cuda")[off:off + 700] for _ in range(2)]
    exps = [torch.zeros(3, dtype=torch.uint8, device="cuda") for _ in range(2)]
    m.copy_(torch.from_numpy(x)), v.copy_(torch.from_numpy(x))
    src, dst = fr.OptPlan(m=[m], v=[v]), fr.OptPlan(m=codes[:1], v=codes[1:], m_exp=exps[:1], v_exp=exps[1:])
    src.convert_to(dst, rounding, 3)
    dst.convert_to(fr.OptPlan(m=[back_m], v=[back_v]))
    for e, back in zip(exps, (back_m, back_v)):
        got = back.cpu().numpy()
        assert e.tolist() == [247, 255 if lost else 254, 247]
        assert np.isnan(got[256:512]).all() == lost and np.isnan(got).sum() == (256 if lost else 0)
        if not lost:
            assert abs(float(got[300]) - float(x[300])) <= float(x[300]) / 8
            assert (got[np.arange(700) != 300] == 2.0 ** 120).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_finite_gradient_whose_square_overflows(bits):
    """Its element alone stands still in fp32 moments; with 8-bit ones its block of moments reads as NaN, and so do the block's
    parameters after the next step.  A clipped step does not come there."""
    n = 700
    g = np.full(n, 1e-3, np.float32)
    g[300] = 3e19
    for clipped in (False, True):
        w = torch.ones(n, device="cuda")
        grad = torch.from_numpy(g).cuda()
        if bits == 8:
            st = {k: [torch.zeros(n, dtype=torch.uint8, device="cuda")] for k in "mv"}
            st.update({k: [torch.zeros(3, dtype=torch.uint8, device="cuda")] for k in ("m_exp", "v_exp")})
        else:
            st = {k: [torch.zeros(n, device="cuda")] for k in "mv"}
        plan = fr.OptPlan([w], [grad], **st)
        for t in (1, 2):
            record = plan.clip(max_norm=1.0) if clipped else None
            assert not clipped or fr.clip_view(record)[2].item() == 0
            plan.step(fr.fr_adamw(1e-2, 0.9, 0.95, 1e-8, 0.0, t, 0, 0), record)
            grad.fill_(1e-3)
            got = w.cpu().numpy()
            lost = np.isnan(got)
            if clipped or bits == 32 or t == 1:
                assert not lost.any()
            else:
                assert lost[256:512].all() and not lost[:256].any() and not lost[512:].any()
        if not clipped and bits == 32:
            assert got[300] == 1.0 and (np.delete(got, 300) < 1.0).all()
