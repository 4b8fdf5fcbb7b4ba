"""The digests by which a profile says what it measured: each changes with the kernels that it stands for, and only with them."""
import os
import shutil

import pytest

from paper_2509_03047_gb300 import build

OPTIM = ["optim.h", "optim_math.cuh", "optim_block.cuh", "optim_clip.cu", "optim_step.cu", "optim_convert.cu"]
SWEEPS = ["sweep_fp.cu", "sweep_pack.cu", "sweep_unpack.cu", "sweep_unpack_fp.cu", "finalize.cu", "gf2.cuh", "layout.h", "sweep_impl.cuh"]


@pytest.fixture
def edited(monkeypatch, tmp_path):
    """The three digests (whole library, sweeps, optimizer step) with `text` after a source's end."""
    csrc = str(tmp_path / "csrc")
    shutil.copytree(build.CSRC, csrc)
    monkeypatch.setattr(build, "CSRC", csrc)

    def digests(name=None, text=""):
        if name is None:
            return build.source_digest(), build.source_digest(kernels_only=True), build.optim_digest()
        path = os.path.join(csrc, name)
        with open(path, "a+") as f:
            end = f.tell()
            f.write(text)
            f.flush()
            found = digests()
            f.truncate(end)
        return found

    return digests


@pytest.mark.parametrize("name", OPTIM + SWEEPS + ["kernels.h", "api.cu", "optim_api.cu"])
def test_a_digest_changes_with_its_own_sources(edited, name):
    whole, sweeps, optim = edited()
    assert edited(name, "\n// a comment\n") == (whole, sweeps, optim)
    new = edited(name, "\nint more;\n")
    both = name == "kernels.h"  # how kernels are launched and wait for one another
    assert new[0] != whole
    assert (new[1] != sweeps) == (both or name in SWEEPS)
    assert (new[2] != optim) == (both or name in OPTIM)
    assert edited() == (whole, sweeps, optim)
