"""examples/train_and_recover.py: clipped AdamW steps on two replicas that stay bit-identical, through a failure and a restore."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("paper_2509_03047_gb300.flashrec")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("bits", [8, 32])
def test_replicas_train_through_a_failure(bits):
    spec = importlib.util.spec_from_file_location("train_and_recover", os.path.join(ROOT, "examples", "train_and_recover.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.train(bits=bits, steps=60, fail_at=25, quiet=True)  # raises where the replicas differ
    assert len(losses) == 60
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5])
