"""A teacher's logits of any finite value, a type's lowest and largest among them, at temperatures below and above one.

Tolerances: a probability is off by its exponent's rounding, u = 2^-24 of it and of its product each, and by four more; entries far below a row's
largest one are zero in fp32 as in the formula to 2^-126, and so are a student's probabilities below that."""
import pytest

from tests.test_gpu_loss import DTYPES, Reference, U, _dt, _randn, _t, _teacher_target, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tau", [0.01, 0.5, 1.0, 3.0])
@pytest.mark.parametrize("name", DTYPES)
def test_lowest_and_largest_logits(name, tau):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    low, high = torch.finfo(dt).min, torch.finfo(dt).max
    t = torch.tensor([[low, low, low], [0.5, low, 0.25], [high, high, 0.0], [low, high, low], [low, low, -float("inf")], [1.0, 2.0, 0.5]]).to(dt).cuda()
    rows = t.shape[0]
    idx = torch.tensor([[3, 70, 5]] * rows, dtype=torch.int32, device="cuda")
    x, w = _randn(rows, 72, seed=1).to(dt), _randn(90, 72, seed=2, scale=72 ** -0.5).to(dt)
    target, used, entropy = _teacher_target(idx, t, 90, tau)
    assert bool(used.all())
    ref = Reference(name, x, w, None, target, used, tau=tau, entropy=entropy)
    loss, lse = B.distillation_forward(x, w, idx, t, temperature=tau)
    _within(lse, ref.lse, ref.lse_tol, "lse")
    # (logits that matter are within 1 / tau of each other)
    more = (8 + 8 / tau) * U
    _within(loss, ref.loss, ref.loss_tol + more * (1 + target * (ref.s - ref.lse[:, None]).abs()).sum(1), "loss")
    # ds through dbias, which sums it unrounded: one row at a time
    for r in range(rows):
        d = torch.zeros(rows, device="cuda")
        d[r] = 1.0
        db = B.distillation_backward(d, x, w, idx, t, lse, temperature=tau, need=("dbias",))[2]
        p = torch.exp(ref.s[r] - lse[r].double())
        want = (p - target[r]) / tau
        tol = (p * (ref.ds_logit[r] + U * (16 + 5 * ((ref.s[r] - lse[r].double()).abs() + ref.s[r].abs()))) + (more + 8 * U) * target[r]) / tau + 8 * U * want.abs() + 2.0 ** -126 / tau
        _within(db, want, tol, "dbias of row %d" % r)


def test_an_entry_of_no_weight_has_to_be_of_a_class():
    """Its logit is the lowest one: that it weighs nothing does not make its index right."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x, w = _randn(3, 72, seed=1).float(), _randn(90, 72, seed=2).float()
    idx = torch.tensor([[1, 2], [1, 90], [1, -1]], dtype=torch.int32, device="cuda")
    t = torch.tensor([[0.0, torch.finfo(torch.float32).min]] * 3, device="cuda")
    loss = B.distillation_forward(x, w, idx, t, temperature=0.5)[0]
    assert torch.isnan(loss).tolist() == [False, True, False]
