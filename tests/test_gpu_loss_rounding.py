"""The gradients of the losses over many classes in 16 bits: each value is rounded once, whatever the number of rows.

Tolerances are those of the other tests of these gradients (test_gpu_loss.py) with ds known to twice the storage type's bits: e = eps / 2,
off by e^2 of itself instead of e.  Besides that a value of dx or dw is off by its own rounding, e, and by what fp32 makes of its sum: one
addition for each four products of ds and w (or x), 40 more for the parts and the joins, 2^-23 of the sum of the absolute products each; the
second plane's additions are of terms e times as large."""
import math

import pytest

from tests.test_gpu_loss import U, U23, Reference, _adds, _dt, _entropy_target, _mm, _rand, _randn, _t, _teacher_entries, _teacher_target, _within

pytestmark = pytest.mark.gpu

TYPES = ("bf16", "fp16")


def _gradients(ref, lse, dloss, x_floor=0.0):
    """((dx, tolerance), (dw, tolerance)); x_floor [rows, 1]: what x may be off by in dw."""
    torch = _t()
    dt = _dt(ref.name)
    e = torch.finfo(dt).eps / 2
    k = lse.double()[:, None]
    a = 1 + 2 * ref.z_loss * k
    p = torch.exp(ref.s - k)
    g = torch.where(ref.used, dloss.double() / ref.tau, torch.zeros_like(dloss.double()))[:, None]
    near = U * (3 * (ref.s - k).abs() + 2 * (ref.s.abs() + k.abs()))
    ds = g * (a * p - ref.target)
    exact = g.abs() * (a.abs() * p * (ref.ds_logit + near + 8 * U) + 4 * U * (ref.target + a.abs() * p))
    held = exact + e ** 2 * ds.abs() + (g.abs() * a.abs().clamp_min(1) * 2.0 ** -38 if ref.name == "fp16" else 0)
    floor = 2.0 ** -25 if ref.name == "fp16" else 2.0 ** -134
    out = []
    for left, d, right, off, n in ((ds, held, ref.w, 0.0, ref.w.shape[0]), (ds.T, held.T, ref.x, x_floor, ref.x.shape[0])):
        xe = off + torch.zeros_like(right)
        sums = _mm(d, right.abs() + xe) + _mm(left.abs(), xe) + (_adds(n, ref.name) + 40) * U23 * _mm(left.abs(), right.abs())
        exactly = _mm(left, right)
        out.append((exactly, sums + e * (exactly.abs() + sums) + floor))
    return out


# (rows, in, classes): one row more than are held otherwise, logits in tiles of 64, 128 and 256 (small weights for the last: a logit's own error is its
# products'), the gradients in one launch and apart, parts of a reduction, several pieces of the classes
SIZES = [(65, 64, 129), (130, 40, 300), (300, 64, 1031), (700, 72, 3000), (2300, 712, 7001), (30011, 24, 9601)]


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,cin,classes", SIZES)
def test_gradients_are_rounded_once(rows, cin, classes, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x = _randn(rows, cin, seed=rows).to(dt)
    w = _randn(classes, cin, seed=rows + 1, scale=(0.2 if cin > 512 else 1.0) * cin ** -0.5).to(dt)
    dloss = (_rand(rows, seed=rows + 2) + 0.5).float()  # (rows that weigh differently: no target is a power of two)
    labels = torch.randint(-1, classes, (rows,), generator=torch.Generator().manual_seed(rows), dtype=torch.int32).cuda()
    target, used = _entropy_target(labels, classes, 0.0)
    ref = Reference(name, x, w, None, target, used, z_loss=1e-3)
    lse = B.cross_entropy_forward(x, w, labels, z_loss=1e-3)[1]
    got = B.cross_entropy_backward(dloss, x, w, labels, lse, z_loss=1e-3)
    for what, g, (r, tol) in zip(("dx", "dw"), got, _gradients(ref, lse, dloss)):
        _within(g, r, tol, what)
    del ref, target
    idx, t = _teacher_entries(rows, classes, 7, rows + 3, torch.float32)
    target, used, _ = _teacher_target(idx, t, classes, 2.0)
    ref = Reference(name, x, w, None, target, used, tau=2.0)
    # (a teacher's probabilities are off by their exponent's rounding, 2 u of logits of up to 20)
    ref.ds_logit += 20 * U
    lse = B.distillation_forward(x, w, idx, t, temperature=2.0)[1]
    got = B.distillation_backward(dloss, x, w, idx, t, lse, temperature=2.0)
    for what, g, (r, tol) in zip(("dx", "dw"), got, _gradients(ref, lse, dloss)):
        _within(g, r, tol, what)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows", [40, 300])
def test_classes_that_only_rows_of_small_factors_reach(rows, name):
    """One row weighs 256, the others 1e-4 to 1e-5 of that, and its softmax is nothing but its own two classes: what the others' classes
    get is as exact as if that row were not there.  fp16: the first 2^11 of a row's distance from the largest are ds', which has the bits to spare; beyond
    that x is held smaller, whose smallest step is 2^-24."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x, w = _randn(rows, 72, seed=rows, scale=0.1), _randn(64, 72, seed=rows + 1, scale=0.3)
    x[:, 71], x[0] = 0.0, 0.0
    x[0, 71], w[:, 71], w[0, 71] = 1.0, 0.0, 60.0
    x, w = x.to(dt), w.to(dt)
    labels = (2 + torch.arange(rows, device="cuda") % 62).int()
    labels[0] = 1
    dloss = (256 * 10 ** (-4 - _rand(rows, seed=rows + 2))).float()
    dloss[0] = 256.0
    target, used = _entropy_target(labels, 64, 0.0)
    ref = Reference(name, x, w, None, target, used)
    lse = B.cross_entropy_forward(x, w, labels)[1]
    got = B.cross_entropy_backward(dloss, x, w, labels, lse)
    x_floor = 2.0 ** -25 * (256 / dloss.double() * 2.0 ** -11).clamp_min(1)[:, None] if name == "fp16" else 0.0
    for what, g, (r, tol) in zip(("dx", "dw"), got, _gradients(ref, lse, dloss, 0.0 if name != "fp16" else x_floor)):
        _within(g, r, tol, what)
    # the norms too: of a correct rounding of the classes beyond the first two
    dw = _mm((dloss.double()[:, None] * (torch.exp(ref.s - lse.double()[:, None]) - target)).T, ref.x)[2:]
    assert float((got[1][2:].double() - dw).norm()) <= torch.finfo(dt).eps / 2 * float(dw.norm())
