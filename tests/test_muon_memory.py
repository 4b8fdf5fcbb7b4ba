"""The device memory of a plan of the orthogonalised update, by tests/c/muon_memory_test.cc.  No GPU."""
import shutil
import subprocess

import pytest

from host_tests import build_host_test


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_places_of_a_plan(tmp_path):
    r = subprocess.run([build_host_test("muon_memory_test", tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "muon_memory ok" in r.stdout
