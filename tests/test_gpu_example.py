"""The example that runs the operators and the memory together: the draft gets better at what its target answers."""
import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_draft_learns_from_the_memory():
    spec = importlib.util.spec_from_file_location("draft_distillation", os.path.join(ROOT, "examples", "draft_distillation.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.main(rounds=60, say=lambda *a: None)
    stood, loss = [h[0] for h in history], [h[1] for h in history]
    # (seen: 1.01 -> 0.26 and 0.38 -> 1.74)
    assert sum(loss[-5:]) < 0.5 * sum(loss[:5]), loss
    assert sum(stood[-5:]) > 2 * sum(stood[:5]), stood
