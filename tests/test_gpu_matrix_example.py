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


@pytest.mark.parametrize("precision", ["BF16", "FP16", "FP32"])
def test_updated_weights_leave_the_training_state_alone(example, precision):
    """Weights put back as they were between the steps change nothing: neither momentum, nor running statistics, nor loss scale."""
    import numpy as np
    import torch
    W, B = example.W, example.B
    units = W.resnet_basic([1, 1], 10, base=16)
    x, y = torch.from_numpy(W.make_images(8, 16, 16, 3)).cuda(), torch.from_numpy(W.make_labels(8, 10)).cuda()
    seen = []
    for again in (False, True):
        t = B.SeqTrainer(units, k_segments=2, precision=getattr(W, precision), batch=8, height=16, width=16, channels=3, num_classes=10, momentum=0.9)
        t.set_params(W.make_params(units, 16, 16))
        out = []
        for i in range(4):
            out.append(t.step(x, y, lr=0.05))
            if again and i < 3:
                p = t.get_params()
                t.update_params(p if i % 2 else torch.from_numpy(p).cuda())
        seen.append((out, t.get_params(), t.running_stats(), t.predict(x).cpu()))
    (a, pa, ra, qa), (b, pb, rb, qb) = seen
    assert a == b and np.array_equal(pa, pb) and np.array_equal(np.asarray(ra), np.asarray(rb)) and torch.equal(qa, qb)


def test_the_cnn_keeps_its_statistics_from_step_to_step(example, monkeypatch):
    """Inference with the running statistics of the whole training knows the batch that it has learnt."""
    import torch
    trainers = []
    make = example.B.SeqTrainer.__init__
    monkeypatch.setattr(example.B.SeqTrainer, "__init__", lambda self, *a, **kw: (trainers.append(self), make(self, *a, **kw))[1])
    example.train_cnn(steps=40, batch=32)
    t = trainers[0]
    x, y = torch.from_numpy(example.W.make_images(32, 16, 16, 3)).cuda(), torch.from_numpy(example.W.make_labels(32, 10)).cuda().long()
    assert float(torch.nn.functional.cross_entropy(t.predict(x), y)) < 1.0  # (guessing: 2.3)
