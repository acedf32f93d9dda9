"""The example with a draft whose memory is a matrix per head: it runs, and its gradients are those of the recurrence."""
import importlib.util
import math
import os

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("draft_distillation", os.path.join(ROOT, "examples", "draft_distillation.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_runs(example):
    history = example.main(rounds=3, memory_of="matrix", say=lambda *a: None)
    assert len(history) == 3 and all(math.isfinite(x) for h in history for x in h)


def test_gradients_of_its_model(example):
    """Against differences of a loss along random directions, in 32 bits: the loss is a sum of some thousand products of size 1, each
    off by some 2^-20, so that differences over a step of 2e-3 are off by up to 0.05; the slopes are of size 10 to 100."""
    torch.manual_seed(0)
    model = example.MatrixModel(40, 32, 2, seed=1)
    token = torch.randint(-1, 41, (3, 70), device="cuda:0", dtype=torch.int32)
    state = torch.randn(3, model.state, device="cuda:0")
    length = torch.tensor([70, 0, 33], device="cuda:0", dtype=torch.int32)
    inside = (torch.arange(70, device="cuda:0") < length[:, None])[:, :, None]
    up, up_state = torch.randn(3, 70, 40, device="cuda:0") * inside, torch.randn(3, model.state, device="cuda:0")

    def loss():
        logits, last = model(token, state, length)
        return (logits.double() * up).sum() + (last.double() * up_state).sum()
    for p in model.parameters():
        p.requires_grad_(True)
    grads = torch.autograd.grad(loss(), model.parameters())
    with torch.no_grad():
        for p, g in zip(model.parameters(), grads):
            d = g / g.norm()                                     # along the gradient: the slope is its length
            step = 1e-3
            p += step * d
            above = float(loss())
            p -= 2 * step * d
            slope = (above - float(loss())) / (2 * step)
            p += step * d
            assert abs(slope - float(g.norm())) < 0.05 + 0.02 * float(g.norm()), (slope, float(g.norm()))
