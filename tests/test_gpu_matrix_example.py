"""The example that trains with the matrix operators, where a step goes wrong."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("orthogonalised_training", os.path.join(ROOT, "examples", "orthogonalised_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_a_skipped_update_leaves_biases_alone(example):
    import torch
    net = example.FeedForward(40, 24, 48, 1, 10)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(32, 40, generator=gen, device="cuda").bfloat16()
    y = torch.randint(0, 10, (32,), generator=gen, device="cuda")
    net.step(x, y, 0.02)
    w, b = net.w.clone(), net.b.clone()
    bad = x.clone()
    bad[3, 5] = float("inf")
    net.step(bad, y, 0.02)
    assert int(net.skipped) == 1
    assert torch.equal(net.w, w) and torch.equal(net.b, b)
    net.step(x, y, 0.02)
    assert int(net.skipped) == 0 and bool(torch.isfinite(net.w).all()) and not torch.equal(net.b, b)


def test_a_skipped_step_of_a_cnn_changes_no_weight(example, monkeypatch):
    """A step whose gradients are not finite says so and leaves none; training goes on as if it had not been."""
    step, calls = example.B.SeqTrainer.step, []

    def sometimes(self, x, y, lr, grads=None, **kw):
        r = step(self, x, y, lr, grads, **kw)
        calls.append(1)
        if len(calls) in (2, 5):
            grads.fill_(float("inf"))
            r["skipped"] = True
        return r

    monkeypatch.setattr(example.B.SeqTrainer, "step", sometimes)
    losses = example.train_cnn(steps=30, batch=32)
    assert all(v == v and v < 100 for v in losses) and losses[2] == losses[1]
    assert losses[-1] < 0.5 * losses[0]
