"""Classes that a finite bias masks, as one of a type's lowest value does: nothing of them is left in a loss or a gradient, also where
all classes of a tile, or of a run whose sums are kept together, are masked."""
import pytest

from tests.test_gpu_loss import DTYPES, U, _dt, _randn, _t

pytestmark = pytest.mark.gpu

LOWEST = {"fp32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38, "fp16": -65504.0}
MASKS = (LOWEST["fp32"], LOWEST["bf16"], -1e30, -1e12, -1.2345e10, -2.5e9, -1e9, LOWEST["fp16"])
INF = float("inf")


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin", [(1, 2048), (16, 2048), (40, 72), (40, 71), (300, 72), (2100, 712)])
def test_masked_classes_are_as_if_left_out(rows, cin, name):
    """exp of a masked logit is zero in fp32, so the bits are those with a bias of -infinity."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    classes, kept = 1700, 150
    x, w = _randn(rows, cin, seed=1).to(dt), _randn(classes, cin, seed=2, scale=2 * cin ** -0.5).to(dt)
    labels = torch.randint(0, kept, (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    idx = labels[:, None].repeat(1, 3)
    idx[:, 1] = (idx[:, 0] + 7) % kept
    idx[:, 2] = (idx[:, 0] + 60) % kept
    t = _randn(rows, 3, seed=4).float()
    d = torch.rand(rows, generator=torch.Generator().manual_seed(5)).cuda() + 0.5

    def everything(bias):
        loss, lse = B.cross_entropy_forward(x, w, labels, bias, z_loss=1e-3)
        out = [loss, lse, *B.cross_entropy_backward(d, x, w, labels, lse, bias, z_loss=1e-3)]
        loss, lse = B.distillation_forward(x, w, idx, t, bias, temperature=2.0)
        return out + [loss, lse, *B.distillation_backward(d, x, w, idx, t, lse, bias, temperature=2.0)]
    bias = _randn(classes, seed=6).float()
    # whole tiles, single runs of 16, and some between those that are kept
    masked = torch.arange(classes, device="cuda") >= kept
    masked[1500:1600] = False
    masked[20:36] = True
    masked[labels.long()] = masked[idx.long().flatten()] = False
    bias[masked] = -INF
    want = everything(bias)
    assert all(bool(torch.isfinite(v).all()) for v in want)
    for v in MASKS:
        bias[masked] = v
        for k, (got, ref) in enumerate(zip(everything(bias), want)):
            assert torch.equal(got, ref), (v, k)


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin", [(16, 2048), (40, 71), (300, 72)])
def test_rows_of_masked_classes_alone(rows, cin, name):
    """Every logit is near the mask's value: lse is that value but for fp32's rounding of it, and so is a loss."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x, w = _randn(rows, cin, seed=1).to(dt), _randn(700, cin, seed=2, scale=cin ** -0.5).to(dt)
    labels = torch.arange(rows, dtype=torch.int32, device="cuda")
    for v in MASKS[:-1]:
        loss, lse = B.cross_entropy_forward(x, w, labels, torch.full((700,), v, device="cuda"))
        # (the logits' own size, a few units, is below half a step of such a value but for the smallest)
        assert bool(((lse.double() - v).abs() <= 4 * U * abs(v) + 64).all()), v
        assert bool((loss.abs().double() <= 8 * U * abs(v) + 64).all()), v


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows", [40, 300])
def test_large_logits(rows, name):
    """Logits of 1e3 to 1e12: lse is off by its own rounding and its parts', and what is sure has no gradient."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x = torch.zeros(rows, 72, device="cuda", dtype=dt)
    x[:, :64] = torch.eye(64, device="cuda", dtype=dt).repeat((rows + 63) // 64, 1)[:rows]
    labels = (torch.arange(rows, device="cuda") % 64).int()
    w = torch.zeros(300, 72, device="cuda", dtype=dt)
    w[:64, :64] = torch.eye(64, device="cuda", dtype=dt)
    for size in (1e3, 3e4) if name == "fp16" else (1e3, 1e5, 1e7, 1e9, 3e10, 1e12):
        s = float(torch.tensor(size).to(dt))
        loss, lse = B.cross_entropy_forward(x, w * s, labels)
        assert bool(((lse.double() - s).abs() <= 4 * U * s).all()), size
        assert bool((loss.abs().double() <= 8 * U * s).all()), size
        dx, dw, _ = B.cross_entropy_backward(torch.ones(rows, device="cuda"), x, w * s, labels, torch.full_like(lse, s))
        assert not bool(dx.any()) and not bool(dw.any()), size
