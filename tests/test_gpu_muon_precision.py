"""What include/flashrec.h promises of O's precision, at sides from 256 to a million, against fp64 on the GPU: products of both
halves to 2^-12, at least four times nearer than one product; one product to 0.2%, to 0.5% where fewer than 16 singular
values are not zero.  (Norms over all elements.  One product: 15 roundings, each off by half of 2^-11 on average, are 3.7e-3 of a
singular value if all go the same way; over 16 singular values their errors are independent, 3.7e-3 / 4 and what they have in
common.  Both halves: a part of a contraction has at most 12 * 64 additions in tensor memory, each
cut off by half of 2^-23 on average, of sums that are half of the last one on average: 768 * 2^-25 = 2.3e-5 of each of three
products in five iterations, 3.4e-4 if all of it went the same way through all of them; their 22 bits 5 * 6 * 2^-22.  2^-12 is
2.4e-4.)  Where all singular values are equal, or one is a thousand times the others, roundings go the same way: the worst
case of one product, 15 * 2^-11, is 7.3e-3, and the promise 5e-3 and 2^-10."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _matrix(shape, kind):
    gen = torch.Generator(device="cuda").manual_seed(0)
    if kind == "low":
        r = max(1, min(shape) // 16)
        return torch.randn(shape[0], r, generator=gen, device="cuda") @ torch.randn(r, shape[1], generator=gen, device="cuda")
    if kind == "equal":
        return torch.eye(*shape, device="cuda") + 1e-4 * torch.randn(shape, generator=gen, device="cuda")
    if kind == "outweighed":
        one = torch.randn(shape[0], 1, generator=gen, device="cuda") @ torch.randn(1, shape[1], generator=gen, device="cuda")
        return one + 1e-3 * torch.randn(shape, generator=gen, device="cuda")
    return torch.randn(shape, generator=gen, device="cuda") + (10.0 if kind == "shifted" else 0.0)


def _exact(g):
    x = g.double()
    x = x / x.norm()
    x = x if g.shape[0] <= g.shape[1] else x.T
    for a, b, c in fr.MUON_COEFFICIENTS:
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x if g.shape[0] <= g.shape[1] else x.T


def _orthogonal(g, products):
    out = torch.zeros_like(g)
    plan = fr.MuonPlan(grads=[g], updates=[out])
    plan.orthogonalize(fr.muon(products=products))
    assert plan.sync_status() == fr.FR_OK
    plan.close()
    return out


@pytest.mark.parametrize("kind", ["plain", "low", "shifted"])
@pytest.mark.parametrize("shape", [(256, 256), (1000, 1000), (1500, 3000), (4096, 256), (2049, 1025), (4096, 4096), (4097, 129), (300, 4224), (4096, 14336),
                                   (256, 16384), (128, 65536), (65537, 200), (1, 65536), (1, 1 << 20), (1 << 20, 3), (16, 1 << 20), (1 << 20, 128)])
def test_precision_does_not_fall_with_the_sides(shape, kind):
    g = _matrix(shape, kind)
    want = _exact(g)
    off = lambda o: float((o.double() - want).norm() / want.norm())  # noqa: E731
    both, one = off(_orthogonal(g, fr.FR_MUON_BY_TYPE)), off(_orthogonal(g, fr.FR_MUON_ONE))
    rank = max(1, min(shape) // 16) if kind == "low" else min(shape)
    assert one <= (5e-3 if rank < 16 else 2e-3), one
    assert both <= 2.0 ** -12, both
    assert both <= one / 4, (both, one)


@pytest.mark.parametrize("kind", ["equal", "outweighed"])
@pytest.mark.parametrize("shape", [(17, 40), (300, 700), (4096, 4096), (4096, 14336), (256, 1 << 18)])
def test_precision_where_roundings_go_the_same_way(shape, kind):
    g = _matrix(shape, kind)
    want = _exact(g)
    off = lambda o: float((o.double() - want).norm() / want.norm())  # noqa: E731
    both, one = off(_orthogonal(g, fr.FR_MUON_BY_TYPE)), off(_orthogonal(g, fr.FR_MUON_ONE))
    assert one <= 5e-3 and both <= 2.0 ** -10 and both <= one / 4, (both, one)


def test_bf16_outputs_by_products_of_both_halves():
    """They are the fp32 ones, rounded once: updates, and the weights of a step."""
    gs = [_matrix(s, "plain") for s in [(200, 300), (700, 130), (64, 64), (90, 5000)]]
    wide = [_orthogonal(g, fr.FR_MUON_BY_TYPE) for g in gs]
    outs = [torch.zeros_like(g, dtype=torch.bfloat16) for g in gs]
    plan = fr.MuonPlan(grads=gs, updates=outs, both_halves=True)
    plan.orthogonalize()
    for o, w in zip(outs, wide):
        assert torch.equal(o, w.bfloat16())
    plan.orthogonalize(fr.muon(products=fr.FR_MUON_ONE))
    one = [torch.zeros_like(o) for o in outs]
    fr.MuonPlan(grads=gs, updates=one).orthogonalize()
    for o, w in zip(outs, one):
        assert torch.equal(o, w)
    weights = [(w * 0.1).bfloat16() for w in wide]
    masters = [w.float() for w in weights]
    for w, both in ((weights, True), (masters, False)):
        fr.MuonPlan(w, gs, [torch.zeros_like(g) for g in gs], both_halves=both).step(fr.muon(lr=0.02, weight_decay=0.1))
    for w, m in zip(weights, masters):
        assert torch.equal(w, m.bfloat16())


@pytest.mark.parametrize("products", [fr.FR_MUON_BY_TYPE, fr.FR_MUON_ONE])
def test_a_long_matrix_gives_the_same_bits_in_any_list(products):
    """Of many parts, the last one short; among others that have one; in a list that goes phase by phase."""
    gs = [_matrix(s, "plain") for s in [(130, 70000), (40100, 300), (600, 700)]]
    alone = [_orthogonal(g, products) for g in gs]
    for count in (1, 40):
        many = gs + gs[2:] * count
        outs = [torch.zeros_like(g) for g in many]
        plan = fr.MuonPlan(grads=many, updates=outs)
        for _ in range(2):
            plan.orthogonalize(fr.muon(products=products))
        assert plan.sync_status() == fr.FR_OK
        for o, w in zip(outs, alone + alone[2:] * count):
            assert torch.equal(o, w)
        plan.close()
