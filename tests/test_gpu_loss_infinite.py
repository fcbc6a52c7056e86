"""Losses that the formula makes infinite: a term whose factor is zero is no term, whatever it would be multiplied by."""
import pytest

from tests.test_gpu_loss import DTYPES, _dt, _randn, _t, _teacher_entries

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin", [(3, 2048), (40, 71), (300, 72)])
def test_a_class_of_infinite_logit(rows, cin, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x, w = _randn(rows, cin, seed=1).to(dt), _randn(200, cin, seed=2, scale=cin ** -0.5).to(dt)
    bias = _randn(200, seed=3).float()
    bias[190] = INF
    labels = (torch.arange(rows, device="cuda") % 180).int()
    labels[1] = -1
    used = labels >= 0
    for z in (0.0, 1e-3):
        loss, lse = B.cross_entropy_forward(x, w, labels, bias, z_loss=z)
        assert bool((lse == INF).all()) and bool((loss[used] == INF).all()) and not bool(loss[~used].any())
    idx, t = _teacher_entries(rows, 180, 5, 7, torch.float32)
    idx[0] = torch.arange(5, device="cuda")
    t[0] = 0.0
    loss, lse = B.distillation_forward(x, w, idx, t, bias)
    assert bool((lse == INF).all()) and bool(((loss == INF) | (loss == 0)).all()) and float(loss[0]) == INF


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin", [(3, 2048), (40, 71), (300, 72)])
def test_a_label_that_smoothing_leaves_nothing_of(rows, cin, name):
    """label_smoothing = 1: the target is the same for all classes, the one that is left out among them: infinite, whatever the label."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x, w = _randn(rows, cin, seed=1).to(dt), _randn(200, cin, seed=2, scale=cin ** -0.5).to(dt)
    bias = _randn(200, seed=3).float()
    bias[30] = -INF
    labels = torch.full((rows,), 30, dtype=torch.int32, device="cuda")
    labels[1] = 31
    loss, lse = B.cross_entropy_forward(x, w, labels, bias, label_smoothing=1.0)
    assert bool(torch.isfinite(lse).all()) and bool((loss == INF).all())
