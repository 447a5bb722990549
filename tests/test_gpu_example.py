"""The example trains with Muon, AdamW and the head losses together: the losses fall."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_train_and_distill_example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_distill.py")
    spec = importlib.util.spec_from_file_location("train_and_distill", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(["--steps", "80", "--dim", "128", "--vocab", "1000", "--rows", "32"])
    # a chain that repeats seven times in eight: far below log 1000 = 6.9 once it is learnt
    assert r["first"] > 6.5 and r["taught"] < r["first"] - 1.5 and r["teacher"][-1] < r["teacher"][0] - 1.5
    assert r["student"][-1] < r["student"][0] - 0.5 and r["final"] < r["first"] - 0.5
