"""The embedding's lookup and gradient on the GPU against their definition: lookups bit for bit, gradients within a bound
that counts the fp32 additions of each row."""
import numpy as np
import pytest
import torch

import optim_reference as ref
from test_gpu_optim import Buffers, _wide

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _typed(x, kind):
    x = x.astype(np.float32).ravel()
    return ref.f32_to_bf16(x) if kind == "bf16" else x


def _tokens(rng, n, first, rows, index, how="mixed"):
    """In and around the slice; some negative, some at the type's ends."""
    if how == "mixed":
        t = first + rng.integers(-rows // 4 - 1, rows + rows // 4 + 1, size=n)
        ends = np.iinfo(index)
        odd = np.array([-1, -100, ends.min, ends.max, first - 1, first + rows, first, first + rows - 1], np.int64)
        where = rng.random(n) < 0.1
        t = np.where(where, odd[rng.integers(0, len(odd), size=n)], t)
    elif how == "zipf":
        t = first + np.minimum((rows + 1) ** rng.random(n) - 1, rows - 1).astype(np.int64)
    else:  # one row for `how` of them
        t = np.where(rng.random(n) < how, first + rows // 3, first + rng.integers(0, rows, size=n))
    return np.clip(t, np.iinfo(index).min, np.iinfo(index).max).astype(index)


def _rows_of(tokens, first, rows):
    t = tokens.astype(object) - first if first > 2 ** 40 else tokens.astype(np.int64) - first
    if tokens.dtype == np.int64:  # (a difference may wrap)
        ok = (tokens >= first) & (tokens < first + rows)
        return np.where(ok, t, -1).astype(np.int64)
    return np.where((t >= 0) & (t < rows), t, -1)


DIMS = [1, 2, 3, 8, 31, 100, 256, 264, 321, 776]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("table,out,index", [("bf16", "bf16", np.int64), ("f32", "bf16", np.int32), ("bf16", "f32", np.int32),
                                             ("f32", "f32", np.int64)])
def test_lookup_is_its_definition(table, out, index, dim, shift):
    rng = np.random.default_rng(dim)
    rows, first, n = 57, 1000, 333
    scale = np.float32(1.0 if dim % 2 else 0.3)
    host = _typed(rng.normal(size=(rows, dim)), table)
    tokens = _tokens(rng, n, first, rows, index)
    w = Buffers([host], shift)
    o = Buffers([np.full(n * dim, 7, np.uint16 if out == "bf16" else np.float32)], shift)
    t = torch.from_numpy(tokens).cuda()
    plan = fr.EmbedPlan(rows, dim, 1000, first=first)
    got = plan.lookup(w.tensors[0].view(rows, dim), t, scale=float(scale), out=o.tensors[0].view(n, dim))
    torch.cuda.synchronize()
    at = _rows_of(tokens, first, rows)
    wide = _wide(host).reshape(rows, dim)
    want = np.where((at >= 0)[:, None], (wide[np.maximum(at, 0)] * scale).astype(np.float32), np.float32(0))
    want = _typed(want, out).reshape(n, dim)
    assert o.get()[0].reshape(n, dim).tobytes() == want.tobytes()
    assert got.data_ptr() == o.tensors[0].data_ptr()
    w.check()


def _gradient(rng, rows, first, dim, tokens, out, grad, accumulate, scale, shift=0, max_tokens=None, plan=None, outs=None):
    n = tokens.size
    o = _typed(rng.normal(size=(n, dim)) * 1e-2, out) if outs is None else outs
    old = _typed(rng.normal(size=(rows, dim)) * 1e-2, grad)
    ob, gb = Buffers([o], shift), Buffers([old], shift)
    t = torch.from_numpy(tokens).cuda()
    plan = plan or fr.EmbedPlan(rows, dim, max_tokens or n, first=first)
    plan.grad(ob.tensors[0].view(n, dim), t, gb.tensors[0].view(rows, dim), scale=scale, accumulate=accumulate)
    torch.cuda.synchronize()
    ob.check()
    return _wide(o).reshape(n, dim), _wide(old).reshape(rows, dim), gb.get()[0].reshape(rows, dim)


def _check(rows, first, tokens, o, old, got, accumulate, scale):
    dim = o.shape[1]
    at = _rows_of(tokens, first, rows)
    inside = at >= 0
    total, size = np.zeros((rows, dim)), np.zeros((rows, dim))
    np.add.at(total, at[inside], o[inside].astype(np.float64))
    np.add.at(size, at[inside], np.abs(o[inside].astype(np.float64)))
    count = np.bincount(at[inside], minlength=rows)
    scale = float(np.float32(scale))
    want = scale * total + (old if accumulate else 0.0)
    bf16 = got.dtype == np.uint16
    new = _wide(got.ravel()).reshape(got.shape).astype(np.float64)
    # additions and the product in fp32, then the output's own rounding
    slack = (count[:, None] + 2) * 2.0 ** -24 * abs(scale) * size + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want)
    assert (np.abs(new - want) <= slack).all(), np.abs(new - want).max()
    empty = count == 0
    if accumulate:
        assert np.array_equal(new[empty], old[empty])
    else:
        assert not got[empty].view(np.uint16 if bf16 else np.uint32).any()  # +0


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("out,grad,index", [("bf16", "bf16", np.int64), ("f32", "bf16", np.int32), ("bf16", "f32", np.int32),
                                            ("f32", "f32", np.int64)])
def test_gradient_is_its_definition(out, grad, index, dim, shift, accumulate):
    rng = np.random.default_rng(dim + 1)
    rows, first = 57, 1000
    tokens = _tokens(rng, 700, first, rows, index)
    o, old, got = _gradient(rng, rows, first, dim, tokens, out, grad, accumulate, 0.7, shift)
    _check(rows, first, tokens, o, old, got, accumulate, 0.7)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,n,dim,how", [
    (1, 1, 5, "mixed"), (1, 5000, 40, "mixed"), (2, 4096, 8, "mixed"), (3, 4097, 8, 0.9), (2047, 4096, 16, "zipf"),
    (2048, 8192, 24, "zipf"), (2049, 8193, 16, "zipf"), (2050, 60000, 33, 0.3), (50257, 32768, 64, "zipf"), (50257, 3, 64, "zipf"),
    (130000, 300001, 8, "zipf"), (259, 500001, 21, 0.33), (5000000, 20000, 4, "zipf"), (400, 70000, 2048, 0.6),
    (9, 100000, 512, 1.0), (1 << 23, 9000, 1, "mixed"), (100, 12000, 4104, "zipf"), (100000, 70000, 3, "zipf"),
    (70001, 300, 1, "zipf"), (20000, 6000, 131, "mixed"), (300000, 70000, 4, "mixed")])
def test_batches_and_slices_of_many_sizes(rows, n, dim, how, accumulate):
    rng = np.random.default_rng(rows + n)
    tokens = _tokens(rng, n, 5, rows, np.int32, how)
    o, old, got = _gradient(rng, rows, 5, dim, tokens, "bf16", "f32", accumulate, -1.5)
    _check(rows, 5, tokens, o, old, got, accumulate, -1.5)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("grad", ["bf16", "f32"])
def test_gradient_of_fewer_tokens_than_rows(grad, dim, shift):
    rng = np.random.default_rng(dim + 2)
    tokens = _tokens(rng, 300, 1000, 1500, np.int64)
    o, old, got = _gradient(rng, 1500, 1000, dim, tokens, "bf16", grad, False, 0.7, shift)
    _check(1500, 1000, tokens, o, old, got, False, 0.7)


@pytest.mark.parametrize("accumulate", [False, True])
def test_batches_that_meet_nothing(accumulate):
    rng = np.random.default_rng(1)
    for tokens in (np.full(5000, -1, np.int64), np.full(100, 900, np.int64), np.zeros(0, np.int64)):
        o, old, got = _gradient(rng, 600, 10, 24, tokens, "f32", "bf16", accumulate, 1.0, max_tokens=6000)
        _check(600, 10, tokens, o, old, got, accumulate, 1.0)


def test_a_plan_s_next_calls_know_nothing_of_the_ones_before():
    """Batches of other sizes, other rows, and both modes in turn."""
    rng = np.random.default_rng(2)
    plan = fr.EmbedPlan(3000, 40, 30000, first=0)
    for n, how, accumulate in [(30000, "zipf", False), (5, "mixed", False), (9000, 0.5, True), (100, "zipf", False), (30000, 1.0, True),
                               (20000, "mixed", False), (4096, "zipf", True), (1, "zipf", False)]:
        tokens = _tokens(rng, n, 0, 3000, np.int64, how)
        o, old, got = _gradient(rng, 3000, 0, 40, tokens, "bf16", "f32", accumulate, 1.0, plan=plan)
        _check(3000, 0, tokens, o, old, got, accumulate, 1.0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dim", [72, 264, 1032, 321])
@pytest.mark.parametrize("how", ["zipf", 0.7])
def test_repeated_calls_and_other_addresses_give_the_same_bits(how, dim, accumulate):
    """On and off the vectors' boundaries."""
    tokens = _tokens(np.random.default_rng(3), 50000, 0, 700, np.int64, how)
    first = None
    for shift in (0, 0, 8, 1):
        _, _, got = _gradient(np.random.default_rng(4), 700, 0, dim, tokens, "bf16", "f32", accumulate, 1.0, shift)
        first = got if first is None else first
        assert got.tobytes() == first.tobytes()


def test_nonfinite_gradients_stay_in_their_rows():
    rng = np.random.default_rng(5)
    tokens = _tokens(rng, 3000, 0, 50, np.int32, "zipf")
    o = rng.normal(size=(3000, 24)).astype(np.float32)
    hit = np.flatnonzero(tokens == 7)[0]
    o[hit, 3] = np.inf
    _, _, got = _gradient(rng, 50, 0, 24, tokens, "f32", "f32", False, 1.0, outs=o.ravel())
    bad = ~np.isfinite(got)
    assert bad[7, 3] and bad.sum() == 1


def test_lookup_of_nonfinite_rows():
    table = torch.tensor([[float("inf"), -0.0], [float("nan"), 1.0]], device="cuda")
    plan = fr.EmbedPlan(2, 2, 10)
    got = plan.lookup(table, torch.tensor([[1, 0], [5, -3]], device="cuda"), scale=2.0).cpu().numpy()
    assert np.isnan(got[0, 0, 0]) and got[0, 0, 1] == 2.0 and np.isposinf(got[0, 1, 0])
    assert np.signbit(got[0, 1, 1]) and not np.signbit(got[1]).any() and not got[1].any()


def test_gradient_against_autograd_and_differences():
    """A loss through lookup: its gradient by grad() is autograd's of indexing, and that of differences of the loss."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    rows, dim, scale = 40, 24, 1.5
    table = torch.randn(rows, dim, generator=gen, device="cuda")
    tokens = torch.randint(-3, rows + 3, (4, 50), generator=gen, device="cuda")
    target = torch.randn(4, 50, dim, generator=gen, device="cuda")
    plan = fr.EmbedPlan(rows, dim, 200)
    y = plan.lookup(table, tokens, scale=scale)
    grad = plan.grad(y - target, tokens, scale=scale)

    def loss(w):
        inside = (tokens >= 0) & (tokens < rows)
        z = torch.where(inside[..., None], w[tokens.clamp(0, rows - 1)] * scale, 0.0)
        return 0.5 * (z - target.double()).square().sum()

    w = table.double().requires_grad_()
    want, = torch.autograd.grad(loss(w), w)
    # some 5 tokens a row: y, its difference, the sum, each rounded to 2^-24 of numbers up to 5
    assert (grad.double() - want).abs().max() <= 50 * 5 * 2.0 ** -24 * 5
    d = torch.randn(rows, dim, generator=gen, device="cuda").double()
    eps = 1e-4
    slope = (loss(table.double() + eps * d) - loss(table.double() - eps * d)) / (2 * eps)
    assert abs(slope - (grad.double() * d).sum()) <= 1e-5 * abs(slope) + 1e-3


def test_calls_on_a_stream_and_from_a_graph():
    rng = np.random.default_rng(7)
    rows, dim, n = 3000, 40, 20000
    tokens = torch.from_numpy(_tokens(rng, n, 0, rows, np.int64, "zipf")).cuda()
    other = torch.from_numpy(_tokens(rng, n, 0, rows, np.int64, 0.4)).cuda()
    o = torch.randn(n, dim, device="cuda")
    want = []
    plan = fr.EmbedPlan(rows, dim, n)
    for t in (tokens, other):
        want.append(plan.grad(o, t).clone())
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = plan.grad(o, tokens, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want[0])
    held, grad, table = tokens.clone(), torch.empty(rows, dim, device="cuda"), torch.randn(rows, dim, device="cuda")
    out = torch.empty(n, dim, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.lookup(table, held, out=out)
        plan.grad(o, held, grad)
    for t, w in ((tokens, want[0]), (other, want[1]), (tokens, want[0])):
        held.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, w)
        assert torch.equal(out, table[t])


def test_offsets_past_32_bits():
    """A table of more than 2^32 elements, an output of more than 2^31."""
    rows, dim = 1 << 21, 2056
    table = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([rows - 1, 0, rows - 2, rows - 1], device="cuda")
    table[tokens[:3]] = torch.randn(3, dim, device="cuda").bfloat16()
    plan = fr.EmbedPlan(rows, dim, 4)
    got = plan.lookup(table, tokens)
    assert torch.equal(got, table[tokens])
    plan.grad(got, tokens, table, scale=1.0)
    want = torch.zeros(4, dim, device="cuda")
    want[0] = 2 * got[0].float()
    want[1], want[2] = got[1].float(), got[2].float()
    assert torch.equal(table[tokens[0]].float(), want[0].bfloat16().float())
    assert torch.equal(table[tokens[1:3]].float(), want[1:3])
    assert int(torch.count_nonzero(table[1:rows - 2])) == 0


def test_an_empty_slice_and_empty_rows():
    plan = fr.EmbedPlan(0, 6, 100, first=50)
    tokens = torch.arange(40, 60, device="cuda")
    table = torch.empty(0, 6, device="cuda")
    out = plan.lookup(table, tokens, out=torch.full((20, 6), 7.0, device="cuda"))
    assert not out.any()
    assert plan.grad(out, tokens).shape == (0, 6)
    empty = fr.EmbedPlan(4, 0, 100)
    assert empty.lookup(torch.empty(4, 0, device="cuda"), tokens).shape == (20, 0)
    assert empty.grad(torch.empty(20, 0, device="cuda"), tokens).shape == (4, 0)
    torch.cuda.synchronize()


def test_calls_that_the_binding_refuses():
    plan = fr.EmbedPlan(10, 4, 8)
    table, tokens = torch.zeros(10, 4, device="cuda"), torch.zeros(5, dtype=torch.int64, device="cuda")
    out = torch.zeros(5, 4, device="cuda")
    for bad in (lambda: plan.lookup(table[:9], tokens), lambda: plan.lookup(table, tokens, out=out[:4]), lambda: plan.lookup(table.half(), tokens),
                lambda: plan.lookup(table, tokens.short()), lambda: plan.lookup(table, tokens.cpu()), lambda: plan.lookup(table.cpu(), tokens),
                lambda: plan.lookup(torch.zeros(4, 10, device="cuda").t(), tokens), lambda: plan.grad(out, tokens, table[:, :3]),
                lambda: plan.grad(out, tokens, accumulate=True), lambda: plan.grad(out[:4], tokens)):
        with pytest.raises(ValueError):
            bad()
    many = torch.zeros(9, dtype=torch.int32, device="cuda")
    with pytest.raises(fr.FlashrecError, match="more tokens"):
        plan.lookup(table, many)
    with pytest.raises(fr.FlashrecError, match="scale"):
        plan.lookup(table, tokens, scale=float("nan"))
    with pytest.raises(fr.FlashrecError, match="scale"):
        plan.grad(out, tokens, scale=1e39)
    torch.cuda.synchronize()


def test_a_batch_among_two_streams():
    """Lookups of one plan on two streams at once (they use no memory of it)."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    table = torch.randn(500, 64, generator=gen, device="cuda")
    plan, streams = fr.EmbedPlan(500, 64, 30000), [torch.cuda.Stream() for _ in range(2)]
    tokens = [torch.randint(0, 500, (30000,), generator=gen, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    got = [plan.lookup(table, t, stream=s) for t, s in zip(tokens, streams)]
    torch.cuda.synchronize()
    for t, o in zip(tokens, got):
        assert torch.equal(o, table[t])
