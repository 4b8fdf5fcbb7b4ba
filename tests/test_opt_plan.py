"""The optimizer step's planner and refusals on the host (csrc/optim_api.cu over tests/c/fake_cuda.h).  No GPU."""
import shutil
import subprocess

import pytest

from host_tests import build_host_test


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_every_element_of_a_launch_comes_up_once(tmp_path):
    r = subprocess.run([build_host_test("opt_plan_test", tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "opt_plan ok" in r.stdout
