"""The gradients of layer norm and of the losses against differences of their forward calls, along the gradient itself.

Of L = sum(c f): D(t) = (L(+t v) - L(-t v)) / 2t is off by a t^2 + ..., so D(t / 2) by about a third of |D(t) - D(t / 2)|, and by the rounding of the
values and of the steps over t.  v = grad / |grad|, so that what D has to be is |grad|, and the steps are as long as the bound needs to be less than
5 % of that (which is asserted, so that no test passes for want of a bound)."""
import pytest

from tests import test_gpu_loss as loss_tests
from tests import test_gpu_norm as norm_tests

pytestmark = pytest.mark.gpu

U, U23 = 2.0 ** -24, 2.0 ** -23


def _check(value, operands, which, grad, noise, t, what):
    """value(operands): L in float64; noise: what rounding may make of it."""
    v = grad / grad.norm()

    def slope(t):
        p, q = list(operands), list(operands)
        p[which], q[which] = p[which] + t * v, q[which] - t * v
        step = ((p[which].double() - q[which].double()) * v.double()).sum() / v.double().square().sum()
        return float((value(p) - value(q)) / step)
    wide, near = slope(t), slope(t / 2)
    want = float((grad.double() * v.double()).sum())
    # (the steps are rounded to fp32 as well: u of every value, times its gradient)
    bound = abs(wide - near) + 2 * noise / t + 2 * U / t * float((grad.abs().double() * operands[which].abs().double()).sum())
    assert bound <= 0.05 * want, "%s: the bound says nothing: %.3g of %.3g" % (what, bound, want)
    assert abs(near - want) <= bound, "%s: %.6g, and the gradient's length is %.6g (bound %.3g)" % (what, near, want, bound)


@pytest.mark.parametrize("rows,cols,t", [(3, 5, 2.0 ** -4), (4, 130, 0.25), (2, 5000, 0.5), (40, 700, 0.5), (3, 9000, 1.0), (2, 20000, 2.0)])
def test_layer_norm(rows, cols, t):
    from paper_2105_00619_amd import binding as B
    randn = norm_tests._randn
    operands = [randn(*s, seed=cols + k).float().cuda() for k, s in enumerate(((rows, cols), (cols,), (cols,)))]
    c = randn(rows, cols, seed=9).float().cuda()
    y, mean, rstd = B.layer_norm_forward(*operands, save_stats=True)
    grads = B.layer_norm_backward(c, operands[0], mean, rstd, operands[1])
    noise = float((c.abs().double() * (y.abs() + 1)).sum()) * (norm_tests._row_adds(cols) + 12) * U
    for which, name in enumerate(("x", "weight", "bias")):
        _check(lambda p: (c.double() * B.layer_norm_forward(*p).double()).sum(), operands, which, grads[which], noise, t, name)


@pytest.mark.parametrize("rows,cin,classes,t", [(4, 6, 9, 0.25), (33, 70, 150, 0.5), (70, 130, 1031, 1.0)])
@pytest.mark.parametrize("kind", ["entropy", "distillation"])
def test_losses(kind, rows, cin, classes, t):
    from paper_2105_00619_amd import binding as B
    torch = loss_tests._t()
    randn = loss_tests._randn
    operands = [randn(rows, cin, seed=1).float(), randn(classes, cin, seed=2, scale=cin ** -0.5).float(), randn(classes, seed=3).float()]
    c = randn(rows, seed=4).float()
    if kind == "entropy":
        labels = torch.randint(-1, classes, (rows,), generator=torch.Generator().manual_seed(5), dtype=torch.int32).cuda()
        fwd, bwd, args, kw = B.cross_entropy_forward, B.cross_entropy_backward, (labels,), {"label_smoothing": 0.2, "z_loss": 0.05}
    else:
        fwd, bwd, args, kw = B.distillation_forward, B.distillation_backward, loss_tests._teacher_entries(rows, classes, 5, 60, torch.float32), {"temperature": 1.5}
    loss, lse = fwd(operands[0], operands[1], *args, operands[2], **kw)
    grads = bwd(c, operands[0], operands[1], *args, lse, operands[2], **kw)
    noise = float((c.abs() * (loss.abs() + lse.abs() + 4)).double().sum()) * (loss_tests._adds(cin, "fp32") + 120) * U23
    for which, name in enumerate(("x", "w", "bias")):
        _check(lambda p: (c.double() * fwd(p[0], p[1], *args, p[2], **kw)[0].double()).sum(), operands, which, grads[which], noise, t, name)
