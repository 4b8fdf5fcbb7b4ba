"""A wait that a product gives up, by tests/c/muon_wait_test.cu: a count that nothing reaches, a limit of milliseconds."""
import os
import subprocess

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_wait_that_is_given_up(tmp_path):
    from paper_2509_03047_gb300 import build

    build.build()
    exe = str(tmp_path / "muon_wait_test")
    objects = [os.path.join(build.OUT_DIR, s.replace(".cu", ".o")) for s in build.SOURCES if s != "muon_api.cu"]
    cmd = [build.nvcc()] + build.ARCH + ["-O1", "-std=c++17", "-I", build.CSRC, os.path.join(ROOT, "tests", "c", "muon_wait_test.cu")]
    r = subprocess.run(cmd + objects + ["-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "muon_wait ok" in r.stdout
