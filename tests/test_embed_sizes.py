"""The binding's fr_embed_lookup and fr_embed_grad compare their tensors with the plan before the library gets addresses.  No GPU:
host tensors that claim to be on one, and a library that must not be called, or whose call is looked at."""
import pytest
import torch

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")


class _Claims:
    is_cuda = True

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index


class _Library:
    def __init__(self):
        self.calls = []

    def fr_embed_lookup(self, *args):
        self.calls.append(args)
        return fr.FR_OK

    fr_embed_grad = fr_embed_lookup


@pytest.fixture
def library(monkeypatch):
    """A plan of 10 rows of 4 elements, for 8 tokens."""
    lib = _Library()
    monkeypatch.setattr(fr, "lib", lib)
    monkeypatch.setattr(fr, "fr_embed_info", lambda plan: (10, 4, 8, 0))
    return lib


def _f(*shape, device=0):
    return _Claims(torch.zeros(*shape), device)


def _tokens(n):
    return _Claims(torch.zeros(n, dtype=torch.int64))


@pytest.mark.parametrize("table,n,out", [((9, 4), 5, (5, 4)), ((10, 5), 5, (5, 4)), ((10, 4), 5, (4, 4)), ((10, 4), 5, (5, 3)), ((10, 4), 6, (5, 4)),
                                         ((11, 4), 5, (5, 4)), ((0, 4), 5, (5, 4)), ((10, 4), 5, (0, 4)), ((10, 4), 0, (5, 4))])
def test_other_sizes_are_refused(library, table, n, out):
    with pytest.raises(ValueError, match="holds"):
        fr.fr_embed_lookup(1, _f(*table), _tokens(n), 1.0, _f(*out), stream=0)
    with pytest.raises(ValueError, match="holds"):
        fr.fr_embed_grad(1, _f(*out), _tokens(n), _f(*table), stream=0)
    assert not library.calls


def test_several_devices_are_refused(library):
    with pytest.raises(ValueError, match="several devices"):
        fr.fr_embed_lookup(1, _f(10, 4), _tokens(5), 1.0, _f(5, 4, device=1), stream=0)
    with pytest.raises(ValueError, match="several devices"):
        fr.fr_embed_grad(1, _f(5, 4), _tokens(5), _f(10, 4, device=1), stream=0)
    assert not library.calls


def test_the_plan_s_sizes_go_on(library):
    table, tokens, out = _f(10, 4), _tokens(5), _f(5, 4)
    fr.fr_embed_lookup(1, table, tokens, 2.0, out, stream=0)
    fr.fr_embed_grad(1, out, tokens, table, 2.0, True, stream=0)
    a, b = library.calls
    assert a[:7] == (1, table.data_ptr(), fr.FR_DT_F32, tokens.data_ptr(), 8, 5, 2.0) and a[7] == out.data_ptr()
    assert b[1] == out.data_ptr() and b[5:8] == (5, 2.0, table.data_ptr()) and b[9] == 1
