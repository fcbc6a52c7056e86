"""Infinities, NaNs and the ends of the range in the matrix operators: what they make of results, and what they cost."""
import pytest

pytestmark = pytest.mark.gpu


def _us(f):
    """The best of five runs of a call, after one that is not counted."""
    import torch
    times = []
    for _ in range(6):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return min(times[1:])


@pytest.mark.parametrize("rows,cin,cout", [(700, 520, 900), (48, 2048, 700), (2000, 1500, 40)])
@pytest.mark.parametrize("bad", ["nan row of x", "all infinite", "nan in w"])
def test_values_that_are_not_finite_cost_a_few_times_as_much(rows, cin, cout, bad):
    """fp32 values are planes, whose products an infinity makes NaN; such a tile is made three times.  A training step that has
    diverged must not look like one that hangs: at most six times as long, with 100 us beside it for what launches cost."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(s, generator=gen, device="cuda") for s in ((rows, cin), (cout, cin), (rows, cout)))
    fine = [_us(lambda: B.linear_forward(x, w)), _us(lambda: B.linear_backward(dy, x, w))]
    if bad == "nan row of x":
        x[rows // 2] = float("nan")
        dy[rows // 3] = float("nan")
    elif bad == "all infinite":
        x.fill_(float("inf"))
        dy.fill_(float("-inf"))
    else:
        w[3, 5] = float("nan")
    took = [_us(lambda: B.linear_forward(x, w)), _us(lambda: B.linear_backward(dy, x, w))]
    for t, f in zip(took, fine):
        assert t <= 6 * f + 100, (took, fine)
    want = torch.mm(x.double(), w.double().T.contiguous())
    y = B.linear_forward(x, w)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.isinf(y), torch.isinf(want))


@pytest.mark.parametrize("rows,cin,cout", [(20, 264, 33), (600, 264, 33), (300, 264, 200), (1500, 72, 1500)])
def test_fp32_infinities_beside_ordinary_values(rows, cin, cout):
    """An infinity times a value of one bf16 plane is that infinity, not NaN; the neighbours of such a sum are as they would be without it; a
    sum that leaves the range of fp32 by itself is infinite too; the largest floats, which bf16 rounds to infinity, are values like others."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, w = torch.randint(-3, 4, (rows, cin), generator=gen, device="cuda").float(), torch.randn(cout, cin, generator=gen, device="cuda")
    bias, res = torch.randn(cout, generator=gen, device="cuda"), torch.randn(rows, cout, generator=gen, device="cuda")
    clean = B.linear_forward(x, w, bias, residual=res, activation="gelu")
    big = torch.finfo(torch.float32).max
    x[1, 7], x[rows - 1, cin - 1], x[5, 0], x[9, 3], x[9, 11] = float("inf"), float("-inf"), float("nan"), big, 1.0
    w[cout - 1, 2], w[4, 3], w[4, 11] = float("inf"), 0.5, 0.0
    w[6, 3], w[6, 11] = 4.0, 0.0
    want = torch.mm(x.double(), w.double().T.contiguous()) + bias.double()
    most = big * (1 + 2.0 ** -25)  # (what rounds to infinity)
    infinite = want.abs() >= most
    want[infinite] = torch.sign(want[infinite]) * float("inf")
    y, z = B.linear_forward(x, w, bias, residual=res, activation="gelu", save_pre=True)
    assert torch.equal(torch.isnan(z), torch.isnan(want))
    assert torch.equal(torch.isposinf(z), torch.isposinf(want)) and torch.equal(torch.isneginf(z), torch.isneginf(want))
    fine = torch.isfinite(want)
    assert bool(torch.isinf(z[9, 6])) and abs(float(z[9, 4]) / (big * 0.5) - 1) < 1e-5
    same = torch.ones_like(fine)
    same[[1, 5, 9, rows - 1]] = False
    same[:, [cout - 1, 4, 6]] = False
    assert bool(fine[same].all()) and torch.equal(y[same], clean[same])
    # in place on the skip connection: groups that wait for the second pass find it as it was
    y2 = res.clone()
    B.linear_forward(x, w, bias, residual=y2, activation="gelu", out=y2)
    assert torch.equal(torch.nan_to_num(y2, nan=7.0), torch.nan_to_num(y, nan=7.0))
    dy = torch.randint(-2, 3, (rows, cout), generator=gen, device="cuda").float()
    dy[3, 1] = float("inf")
    dx, dw, _ = B.linear_backward(dy, x, w)
    # (products that leave the range of fp32 by themselves are infinities in the sum, so the reference multiplies in fp32)
    for got, ref in ((dx, (dy[:, :, None] * w[None]).double().sum(1)), (dw, (dy[:, :, None] * x[:, None]).double().sum(0))):
        ref[ref.abs() >= most] = torch.sign(ref[ref.abs() >= most]) * float("inf")
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(torch.isposinf(got), torch.isposinf(ref)) and torch.equal(torch.isneginf(got), torch.isneginf(ref))


@pytest.mark.parametrize("name,rows,cin", [("fp32", 2 ** 28 + 40, 2), ("bf16", 2 ** 30 + 72, 1)])
def test_batches_of_more_blocks_than_one_row_of_a_grid(name, rows, cin):
    """2^28 samples of few outputs straight from memory and 2^30 as tiles of 64 are 2^32 threads, more than a launch has along x."""
    import torch
    from paper_2105_00619_amd import binding as B
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[name]
    x = torch.empty(rows, cin, dtype=dt, device="cuda")
    x.copy_((torch.arange(rows, device="cuda") % 251 - 125)[:, None])  # (whole numbers that bf16 holds)
    w = torch.tensor([[0.5, -0.25][:cin]], dtype=dt, device="cuda")
    y = B.linear_forward(x, w)
    want = x[:, 0] * (0.25 if cin == 2 else 0.5)
    assert torch.equal(y[:, 0], want)


@pytest.mark.parametrize("name", ["fp32", "bf16", "fp16"])
def test_what_relu_masks_is_zero(name):
    """An infinite or NaN gradient of an output that ReLU has cut off reaches nothing."""
    import torch
    from paper_2105_00619_amd import binding as B
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]
    gen = torch.Generator(device="cuda").manual_seed(4)
    dy, x, w, z = (torch.randn(s, generator=gen, device="cuda").to(dt) for s in ((70, 33), (70, 20), (33, 20), (70, 33)))
    z[3], z[5, 7] = 0.0, -1.0
    masked = z <= 0
    clean = B.linear_backward(dy, x, w, z, activation="relu")
    dy[masked] = float("inf")
    dy[5, 7], dy[3, 1] = float("nan"), float("-inf")
    assert all(torch.equal(a, b) for a, b in zip(B.linear_backward(dy, x, w, z, activation="relu"), clean))


def test_buffers_side_by_side_are_apart():
    """Operands and results whose rows lie between each other's share no element; those that do are refused."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(6)
    buf = torch.randn(90, 200, generator=gen, device="cuda")
    x, y, dy = buf[:, :60], buf[:, 60:100], buf[:, 100:140]
    w = torch.randn(40, 60, generator=gen, device="cuda")
    want = B.linear_forward(x, w)
    assert torch.equal(B.linear_forward(x, w, out=y), want) and torch.equal(y, want)
    dx = B.linear_backward(dy, x, w, need=("dx",))[0]
    assert torch.equal(B.linear_backward(dy, x, w, need=("dx",), dx=buf[:, 140:])[0], dx)
    square = torch.randn(60, 60, generator=gen, device="cuda")
    with pytest.raises(B.OptorchError, match="x and y overlap"):
        B.linear_forward(x, square, out=x)
    with pytest.raises(B.OptorchError, match="dy and dx overlap"):
        B.linear_backward(x, x, square, need=("dx",), dx=buf[:, 1:61])
    p = B.Orthogonalizer([(8, 9)])
    v = torch.randn(300, generator=gen, device="cuda")
    with pytest.raises(B.OptorchError, match="g and o overlap"):
        p.orthogonalize(v[:72], v[71:143])
    with pytest.raises(B.OptorchError, match="w and v overlap"):
        p.muon_update(v[:72], v[:72], v[100:172], lr=0.1)
