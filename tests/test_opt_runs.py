"""Blocks per warp of the 8-bit step (csrc/optim_api.cu over tests/c/fake_cuda.h).  No GPU."""
import shutil
import subprocess

import pytest

from host_tests import build_host_test


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_long_lists_take_runs_of_up_to_eight_blocks(tmp_path):
    r = subprocess.run([build_host_test("opt_runs_test", tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "opt_runs ok" in r.stdout
