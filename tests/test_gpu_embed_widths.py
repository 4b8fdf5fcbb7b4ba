"""The embedding's kernels at the widths of a lane's part that other sizes do not bring up: rows of twice an odd number of elements and
buffers two elements off (vectors of two), and of 1,024 elements and more (two vectors per lane), in all types, with a row long
enough to be put together from several CTAs' parts."""
import numpy as np
import pytest
import torch

from test_gpu_embed import _check, _gradient, _rows_of, _tokens, _typed
from test_gpu_optim import Buffers, _wide

pytestmark = pytest.mark.gpu

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")

TYPES = [("bf16", "bf16", np.int64), ("f32", "bf16", np.int32), ("bf16", "f32", np.int32), ("f32", "f32", np.int64)]
# (dim, shift): rows of 6, 66, 130, 258 and 1,002 elements by vectors of two; of 264 two elements off; of 1,024 and 1,032 by two vectors per lane
WIDTHS = [(6, 0), (66, 2), (130, 0), (130, 2), (258, 0), (1002, 0), (1002, 2), (264, 2), (1024, 0), (1032, 0), (1032, 2), (2056, 4)]


@pytest.fixture(autouse=True)
def _free_memory():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dim,shift", WIDTHS)
@pytest.mark.parametrize("table,out,index", TYPES)
def test_lookup_at_every_width(table, out, index, dim, shift):
    rng = np.random.default_rng(dim)
    rows, first, n = 57, 1000, 333
    host = _typed(rng.normal(size=(rows, dim)), table)
    tokens = _tokens(rng, n, first, rows, index)
    w = Buffers([host], shift)
    o = Buffers([np.full(n * dim, 7, np.uint16 if out == "bf16" else np.float32)], shift)
    plan = fr.EmbedPlan(rows, dim, 1000, first=first)
    plan.lookup(w.tensors[0].view(rows, dim), torch.from_numpy(tokens).cuda(), scale=0.3, out=o.tensors[0].view(n, dim))
    torch.cuda.synchronize()
    at = _rows_of(tokens, first, rows)
    wide = _wide(host).reshape(rows, dim)
    want = np.where((at >= 0)[:, None], (wide[np.maximum(at, 0)] * np.float32(0.3)).astype(np.float32), np.float32(0))
    assert o.get()[0].tobytes() == _typed(want, out).tobytes()
    w.check()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dim,shift", WIDTHS)
@pytest.mark.parametrize("out,grad,index", TYPES)
def test_gradient_at_every_width(out, grad, index, dim, shift, accumulate):
    """One of 57 rows has 0.6 of 9,000 tokens: several CTAs' parts of it."""
    rng = np.random.default_rng(dim + 1)
    rows, first = 57, 1000
    tokens = _tokens(rng, 9000, first, rows, index, 0.6)
    o, old, got = _gradient(rng, rows, first, dim, tokens, out, grad, accumulate, 0.7, shift)
    _check(rows, first, tokens, o, old, got, accumulate, 0.7)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,rows", [(1, 1), (1, 3), (2, 2), (3, 1)])
@pytest.mark.parametrize("out,grad", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_first_and_last_rows_of_odd_length(out, grad, n, rows, accumulate):
    """Buffers of few rows off the granules' boundaries: every row is the first or the last one of `out` or the table."""
    rng = np.random.default_rng(n + 10 * rows)
    for dim, shift in ((129, 1), (385, 3), (1001, 5)):
        tokens = rng.integers(0, rows, size=n)
        o, old, got = _gradient(rng, rows, 0, dim, tokens, out, grad, accumulate, 1.5, shift)
        _check(rows, 0, tokens, o, old, got, accumulate, 1.5)
