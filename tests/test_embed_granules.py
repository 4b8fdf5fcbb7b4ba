"""Copies of rows of odd length stay in their buffers, by tests/c/embed_granules_test.cc.  No GPU."""
import shutil
import subprocess

import pytest

from host_tests import build_host_test


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_granules_lie_in_their_buffer(tmp_path):
    r = subprocess.run([build_host_test("embed_granules_test", tmp_path)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "embed_granules ok" in r.stdout
