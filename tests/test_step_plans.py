"""Planners and refusals of the orthogonalised update and of the embedding on the host (csrc/muon_api.cu, csrc/embed_api.cu
over tests/c/fake_cuda.h), and what the binding refuses.  No GPU."""
import shutil
import subprocess

import pytest
import torch

from host_tests import build_host_test
from paper_2509_03047_gb300 import build

fr = pytest.importorskip("paper_2509_03047_gb300.flashrec")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
@pytest.mark.parametrize("name", ["muon_plan", "embed_plan"])
def test_planner(name, tmp_path):
    r = subprocess.run([build_host_test(name + "_test", tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert name + " ok" in r.stdout


class _Claims:
    """A host tensor that claims to be on the GPU."""

    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def test_lists_that_the_binding_refuses():
    f, e = torch.zeros(2, 3), torch.empty(0, 3)
    with pytest.raises(ValueError, match="needs weights"):
        fr.fr_muon_create()
    with pytest.raises(ValueError, match="not on a CUDA device"):
        fr.fr_muon_create(grads=[f])
    with pytest.raises(ValueError, match="dimensions"):
        fr.fr_muon_create(grads=[torch.empty(0)])
    with pytest.raises(ValueError, match="unsupported dtype"):
        fr.fr_muon_create(momenta=[e.bfloat16()])
    with pytest.raises(ValueError, match="holds 2 matrices, not 1"):
        fr.fr_muon_create(weights=[e], grads=[e, e])
    with pytest.raises(ValueError, match="not contiguous"):
        fr._muon_array(None, [_Claims(torch.zeros(3, 2).t())], None, None, None, None, None, None)
    with pytest.raises(ValueError, match="1 to 10 iterations"):
        fr.muon(coefficients=[])


def test_numbers_of_a_step():
    h = fr.muon(lr=0.5, coefficients=[(1, 2, 3), (4, 5, 6)], nesterov=False, step=7, seed=9, rounding=1, products=1)
    assert (h.lr, h.beta, h.iterations, h.nesterov, h.step, h.seed, h.rounding, h.products) == (0.5, 0.95, 2, 0, 7, 9, 1, 1)
    assert list(h.coef[1]) == [4.0, 5.0, 6.0] and list(h.coef[2]) == [0.0, 0.0, 0.0]


@pytest.mark.parametrize("files,digest", [(build.MUON_KERNEL_FILES, build.muon_digest), (build.EMBED_KERNEL_FILES, build.embed_digest)])
def test_a_digest_changes_with_its_own_sources(files, digest, monkeypatch, tmp_path):
    csrc = tmp_path / "csrc"
    shutil.copytree(build.CSRC, csrc)
    monkeypatch.setattr(build, "CSRC", str(csrc))
    before = digest()
    for name in build.SOURCES + build.HEADERS:
        path = csrc / name
        text = path.read_text()
        path.write_text(text + "\n// a comment\n")
        assert digest() == before
        path.write_text(text + "\nint more;\n")
        assert (digest() != before) == (name in files), name
        path.write_text(text)
    assert digest() == before
