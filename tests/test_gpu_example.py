"""The example that runs the row operators together with a verification step."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_raises_acceptance(gpu_lib):
    spec = importlib.util.spec_from_file_location("distill_draft", os.path.join(ROOT, "examples", "distill_draft.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    h = example.run(steps=60, report=None)
    first, last = h[:5], h[-5:]
    assert sum(b for _, b in last) < 0.7 * sum(b for _, b in first)
    assert sum(a for a, _ in last) > sum(a for a, _ in first)
