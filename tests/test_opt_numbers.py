"""Numbers of an optimizer step that the library refuses (csrc/optim_api.cu over tests/c/fake_cuda.h).  No GPU."""
import shutil
import subprocess

import pytest

from host_tests import build_host_test


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_products_that_fp32_does_not_hold_are_refused(tmp_path):
    r = subprocess.run([build_host_test("opt_numbers_test", tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "opt_numbers ok" in r.stdout
