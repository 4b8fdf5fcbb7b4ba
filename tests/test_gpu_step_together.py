"""Lookup, embedding gradient, clip record, orthogonalised update and AdamW as one step: in examples/train_language_model.py,
against the formulas, and captured in a graph."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import muon_reference as mref

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_language_model", os.path.join(ROOT, "examples", "train_language_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs_and_its_replicas_agree(example):
    losses = example.train(steps=5, quiet=True)  # raises where the replicas differ
    assert len(losses) == 5 and np.isfinite(losses).all()


def test_the_example_s_gradients(example):
    """The embedding's gradient is autograd's of indexing, the others' inputs are the same rows."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    masters = [torch.randn(s, generator=gen, device="cuda") / s[0] ** 0.5 for s in example.SHAPES]
    rank = example.Replica(masters)
    tokens = torch.randint(0, example.VOCAB, (example.BATCH, example.CONTEXT), generator=gen, device="cuda")
    target = torch.randint(0, example.VOCAB, (example.BATCH,), generator=gen, device="cuda")
    loss, grads = rank.differentiate(tokens, target)
    w = [x.detach().clone().requires_grad_() for x in rank.weights]
    rows = w[0][tokens]
    h = torch.relu(torch.relu(rows.flatten(1) @ w[1]) @ w[2])
    want_loss = torch.nn.functional.cross_entropy((h @ w[3]).float(), target)
    rows.retain_grad()
    want_loss.backward()
    assert torch.equal(loss, want_loss.detach())
    for got, x in zip(grads[1:], w[1:]):
        assert torch.equal(got, x.grad)
    # some 21 rows' gradients, equal to what autograd hands on, added in fp32 and rounded once
    exact = torch.zeros(example.VOCAB, example.DIM, dtype=torch.float64, device="cuda")
    exact.index_add_(0, tokens.view(-1), rows.grad.double().view(-1, example.DIM))
    size = torch.zeros_like(exact).index_add_(0, tokens.view(-1), rows.grad.double().abs().view(-1, example.DIM))
    assert ((grads[0].double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 100 * 2.0 ** -24 * size).all()


class _Rank:
    """Embedding and matrices of a rank, fp32, everything by its own plan."""

    def __init__(self, seed=0):
        r = np.random.default_rng(seed)
        dev = lambda x: torch.from_numpy(x.astype(np.float32)).cuda()  # noqa: E731
        self.table, self.w = dev(r.normal(size=(300, 40))), [dev(r.normal(size=s) * 0.1) for s in [(150, 280), (280, 64)]]
        self.table_grad, self.table_m, self.table_v = (torch.zeros_like(self.table) for _ in range(3))
        self.g = [dev(mref.matrix(r, *x.shape)) for x in self.w]
        self.m = [torch.zeros_like(x) for x in self.w]
        self.tokens = torch.from_numpy(r.integers(-2, 303, size=5000)).cuda()
        self.rows_grad = dev(r.normal(size=(5000, 40)) * 1e-2)
        self.out = torch.zeros(5000, 40, device="cuda")
        self.embed = fr.EmbedPlan(300, 40, 5000)
        self.all = fr.OptPlan(grads=[self.table_grad] + self.g)
        self.adamw = fr.OptPlan([self.table], [self.table_grad], [self.table_m], [self.table_v])
        self.muon = fr.MuonPlan(self.w, self.g, self.m)
        self.record = self.all.new_clip()

    def state(self):
        return [self.out, self.table, self.table_grad, self.table_m, self.table_v, *self.w, *self.m]

    def step(self, adamw, muon):
        self.embed.lookup(self.table, self.tokens, scale=2.0, out=self.out)
        self.embed.grad(self.rows_grad, self.tokens, self.table_grad)
        self.all.clip(max_norm=0.5, out=self.record)
        self.muon.step(muon, self.record)
        self.adamw.step(adamw, self.record)


def _numbers():
    return fr.fr_adamw(1e-2, 0.9, 0.99, 1e-8, 0.0, 1), fr.muon(lr=1e-2, nesterov=False)


def test_a_step_of_all_parts_is_the_formulas():
    a = _Rank()
    before = {k: x.cpu().numpy().astype(np.float64) for k, x in (("table", a.table), ("w", a.w[0]), ("g", a.g[0]))}
    a.step(*_numbers())
    torch.cuda.synchronize()
    grad = np.zeros((300, 40))
    tokens = a.tokens.cpu().numpy()
    inside = (tokens >= 0) & (tokens < 300)
    np.add.at(grad, tokens[inside], a.rows_grad.cpu().numpy().astype(np.float64)[inside])
    assert np.abs(a.table_grad.cpu().numpy() - grad).max() <= 60 * 2.0 ** -24 * 60 * 0.05
    norm = np.sqrt((grad ** 2).sum() + sum((x.cpu().numpy().astype(np.float64) ** 2).sum() for x in a.g))
    found, scale, bad = fr.clip_view(a.record)
    assert abs(float(found) - norm) <= 1e-5 * norm and abs(float(scale) - min(1.0, 0.5 / norm)) <= 1e-5 and int(bad) == 0
    want = before["w"] - 1e-2 * mref.orthogonal(before["g"] * 0.05 * float(scale))
    o = mref.bound(split=True, shape=(150, 280))
    assert np.linalg.norm(a.w[0].cpu().numpy() - want) <= 1e-2 * o * np.sqrt(150) * 1.3 + 4 * 2.0 ** -24 * np.linalg.norm(before["w"])
    # a first step of AdamW: lr times the gradient's sign, where it is not tiny
    moved = (a.table.cpu().numpy() - before["table"])[np.abs(grad) > 1e-4]
    assert np.abs(moved + 1e-2 * np.sign(grad[np.abs(grad) > 1e-4])).max() <= 1e-2 * 0.01


def test_the_whole_step_in_a_graph():
    eager, graphed = _Rank(), _Rank()
    numbers = _numbers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(*numbers)
    for _ in range(3):
        eager.step(*numbers)
        graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(eager.state(), graphed.state()):
        assert torch.equal(x, y)


def test_a_nonfinite_embedding_gradient_leaves_every_part():
    a = _Rank()
    a.rows_grad[17, 3] = float("inf")
    a.tokens[17] = 5
    before = [x.clone() for x in (a.table, a.table_m, a.table_v, *a.w, *a.m)]
    a.step(*_numbers())
    torch.cuda.synchronize()
    assert int(fr.clip_view(a.record)[2]) == 1
    for x, y in zip(before, (a.table, a.table_m, a.table_v, *a.w, *a.m)):
        assert torch.equal(x, y)
