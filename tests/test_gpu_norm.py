"""Layer norm and its gradient against plain float64 computations, through the Python binding.

Tolerances, with u = 2^-24.  A result is rounded once to its type: at most eps / 2 of its value.  A sum of fp32 values with n additions one after
the other is off by at most n u times the sum of their absolute values.  A row's sums: 16 values a thread at most up to 16384 columns, eight more for every 8192
beyond, six additions across a wavefront and 16 across the wavefronts.  The mean is corrected by the mean of the deviations from it, which are off by u of themselves, so what counts is their size and not the mean's.  The
deviations are summed with their squares: the variance is off by as many u, and rstd by half of that and four more."""
import math

import pytest

pytestmark = pytest.mark.gpu

DTYPES = ("fp32", "bf16", "fp16")
U = 2.0 ** -24


def _t():
    import torch
    return torch


def _dt(name):
    torch = _t()
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _randn(*shape, seed, scale=1.0, shift=0.0):
    torch = _t()
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale + shift


def _strided(v, dt, pad, shift):
    """v in the type dt on the GPU, its rows `pad` elements further apart and `shift` elements off an aligned address; and the whole buffer."""
    torch = _t()
    r, c = v.shape
    buf = torch.full((shift + r * (c + pad) + 8,), 7.5, dtype=dt, device="cuda")
    m = buf[shift:shift + r * (c + pad)].view(r, c + pad)[:, :c]
    m.copy_(v.to("cuda"))
    return m, buf


def _row_adds(cols):
    return 16 * math.ceil(cols / 16384) + 22


def _column_adds(rows, cols):
    # a thread's rows, its block's, the blocks': up to 256 blocks and more; rows longer than 8192: 32 rows or more for a block's eight threads
    return rows / 256 + 32 + 32 + 40


def _within(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bool(bad.any()), "%s: %d of %d outside, worst %.3g times the tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - ref).abs() / tol.clamp_min(1e-300)).max()))


def _untouched(buf, before, rows, cols, pad, shift):
    torch = _t()
    a, b = buf.clone(), before.clone()
    for t in (a, b):
        t[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols].zero_()
    assert torch.equal(a, b), "values outside the result were written"


# (rows, cols): single values, one row, one column, odd sizes, the ends of each kind of block and their neighbours, rows longer than a block keeps
SIZES = [(1, 1), (5, 1), (1, 8), (3, 5), (2, 17), (33, 128), (70, 129), (257, 256), (64, 264), (31, 512), (5, 1000), (9, 1024), (9, 1031), (5, 2048),
         (1030, 2049), (1, 4096), (7, 4097), (3, 8192), (5, 8200), (2, 16384), (3, 16385), (37, 20000), (2, 40001), (20011, 24), (2100, 640), (300, 2348), (4, 600)]


def _case(rows, cols, name):
    i = SIZES.index((rows, cols))
    dt, pad, shift = _dt(name), (0, 8, 3)[i % 3], (0, 8, 1)[i % 3]
    x, _ = _strided(_randn(rows, cols, seed=i, scale=1.5) + _randn(rows, 1, seed=i + 50, scale=4.0), dt, pad, shift)
    w, b = _randn(cols, seed=i + 100, shift=1.0).float().cuda(), _randn(cols, seed=i + 200).float().cuda()
    return dt, pad, shift, x, w, b


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt, pad, shift, x, w, b = _case(rows, cols, name)
    out, buf = _strided(torch.zeros(rows, cols), dt, pad, shift)
    before = buf.clone()
    y, mean, rstd = B.layer_norm_forward(x, w, b, eps=1e-5, save_stats=True, out=out)
    assert y is out
    v = x.double()
    m = v.mean(1, keepdim=True)
    d = v - m
    var = d.square().mean(1, keepdim=True)
    r = (var + 1e-5) ** -0.5
    n = _row_adds(cols)
    size = d.abs().mean(1, keepdim=True)
    _within(mean, m[:, 0], U * m[:, 0].abs() + (n + 4) * U * size[:, 0], "mean")
    _within(rstd, r[:, 0], (n / 2 + 5) * U * r[:, 0], "rstd")
    h = d * r
    ref = h * w.double() + b.double()
    fp32 = U * (w.double().abs() * ((n / 2 + 10) * h.abs() + (n + 4) * size * r) + 2 * (ref.abs() + b.double().abs()))
    _within(y, ref, torch.finfo(dt).eps / 2 * (ref.abs() + fp32) + fp32, "y")
    _untouched(buf, before, rows, cols, pad, shift)
    # without weight, bias and statistics
    plain = B.layer_norm_forward(x, eps=1e-5)
    fp32 = U * ((n / 2 + 10) * h.abs() + (n + 4) * size * r + 2 * h.abs())
    _within(plain, h, torch.finfo(dt).eps / 2 * (h.abs() + fp32) + fp32, "y without weight and bias")


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(rows, cols, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt, pad, shift, x, w, _ = _case(rows, cols, name)
    i = SIZES.index((rows, cols))
    dy, _ = _strided(_randn(rows, cols, seed=i + 300, scale=0.1), dt, pad, shift)
    res, _ = _strided(_randn(rows, cols, seed=i + 400, scale=0.1), dt, pad, shift)
    v = x.double()
    mean = v.mean(1).float()
    rstd = ((v - mean.double()[:, None]).square().mean(1) + 1e-5).rsqrt().float()
    out, buf = _strided(torch.zeros(rows, cols), dt, pad, shift)
    before = buf.clone()
    dx, dw, db = B.layer_norm_backward(dy, x, mean, rstd, w, residual=res, dx=out)
    assert dx is out
    r = rstd.double()[:, None]
    h = (v - mean.double()[:, None]) * r
    g = dy.double()
    u = g * w.double()
    mu, muh = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    ref = r * (u - mu - h * muh)
    n = _row_adds(cols)
    fp32 = U * r * (4 * u.abs() + (n + 6) * u.abs().mean(1, keepdim=True) + h.abs() * ((n + 10) * (u * h).abs().mean(1, keepdim=True)))
    full = ref + res.double()
    fp32_full = fp32 + U * (ref.abs() + full.abs())
    e = torch.finfo(dt).eps / 2
    _within(dx, full, e * (full.abs() + fp32_full) + fp32_full, "dx")
    _untouched(buf, before, rows, cols, pad, shift)
    nr = _column_adds(rows, cols)
    _within(dw, (g * h).sum(0), (nr + 4) * U * (g * h).abs().sum(0), "dweight")
    _within(db, g.sum(0), nr * U * g.abs().sum(0), "dbias")
    # each gradient alone is what it was beside the others; dx may be the residual; ones for the weight
    assert torch.equal(B.layer_norm_backward(dy, x, mean, rstd, w, need=("dweight",))[1], dw)
    assert torch.equal(B.layer_norm_backward(dy, x, mean, rstd, w, need=("dbias",))[2], db)
    B.layer_norm_backward(dy, x, mean, rstd, w, residual=res, dx=res, need=("dx",))
    assert torch.equal(res, dx)
    plain = B.layer_norm_backward(dy, x, mean, rstd, need=("dx",))[0]
    ref = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    fp32 = U * (r * (4 * g.abs() + (n + 6) * g.abs().mean(1, keepdim=True) + h.abs() * ((n + 10) * (g * h).abs().mean(1, keepdim=True))) + 2 * ref.abs())
    _within(plain, ref, e * (ref.abs() + fp32) + fp32, "dx without weight")


def test_gradients_are_the_forward_calls_differences():
    """Along a direction, of L = sum(c y): D(t) = (L(+t) - L(-t)) / 2t is off by a t^2 + ..., so D(t / 2) by about a third of
    |D(t) - D(t / 2)|, and by the rounding of L, 2 u |y| and a row's sums in each value, over t."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    for rows, cols in ((3, 5), (4, 130), (2, 5000)):
        x, w, b = (_randn(*s, seed=cols + k).float().cuda() for k, s in enumerate(((rows, cols), (cols,), (cols,))))
        c = _randn(rows, cols, seed=9).float().cuda()
        y, mean, rstd = B.layer_norm_forward(x, w, b, save_stats=True)
        dx, dw, db = B.layer_norm_backward(c, x, mean, rstd, w)
        noise = float((c.abs().double() * (y.abs() + 1)).sum()) * (_row_adds(cols) + 12) * U
        for which, grad in ((0, dx), (1, dw), (2, db)):
            v = _randn(*grad.shape, seed=77).float().cuda()
            v /= v.norm()

            def slope(t):
                p, q = [x, w, b], [x, w, b]
                p[which], q[which] = p[which] + t * v, q[which] - t * v
                step = ((p[which].double() - q[which].double()) * v.double()).sum() / v.double().square().sum()
                f = [(c.double() * B.layer_norm_forward(*a).double()).sum() for a in (p, q)]
                return float((f[0] - f[1]) / step)
            t = 2.0 ** -4
            wide, near = slope(t), slope(t / 2)
            want = float((grad.double() * v.double()).sum())
            # (the steps are rounded to fp32 as well: u of every value of x, w or b, times its gradient)
            rounding = 2 * noise / t + 2 * U / t * float((grad.abs().double() * [x, w, b][which].abs().double()).sum())
            assert abs(near - want) <= abs(wide - near) + rounding, (rows, cols, which, near, want, wide)


def test_a_large_mean_does_not_cost_the_deviations():
    """fp32 rows around 10000: the deviations keep the bits that the inputs have of them."""
    from paper_2105_00619_amd import binding as B
    x = (_randn(5, 3000, seed=1) + 1e4).float().cuda()
    y = B.layer_norm_forward(x, eps=0.0)
    v = x.double()
    d = v - v.mean(1, keepdim=True)
    h = d / d.square().mean(1, keepdim=True).sqrt()
    n = _row_adds(3000)
    _within(y, h, U * ((n / 2 + 12) * h.abs() + (n + 4)), "y")


@pytest.mark.parametrize("name", DTYPES)
def test_equal_values_and_values_that_are_not_finite(name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x = _randn(6, 300, seed=3).to(dt).cuda()
    x[1] = 2.5
    x[2, 7], x[3, 299], x[4, 0] = float("inf"), float("nan"), -float("inf")
    b = _randn(300, seed=4).float().cuda()
    y, mean, rstd = B.layer_norm_forward(x, None, b, save_stats=True)
    assert torch.equal(y[1], b.to(dt)), "equal values: nothing but the bias"
    assert bool(torch.isnan(y[2:5]).all())
    assert torch.equal(y[[0, 5]], B.layer_norm_forward(x[[0, 5]], None, b)), "other rows know nothing of it"
    dy = _randn(6, 300, seed=5).to(dt).cuda()
    dx, dw, db = B.layer_norm_backward(dy, x, mean, rstd)
    assert bool(torch.isfinite(dx[[0, 1, 5]]).all()) and bool(torch.isnan(dx[2:5]).all())
    assert bool(torch.isnan(dw).all()) and bool(torch.isfinite(db).all())


@pytest.mark.parametrize("name", DTYPES)
def test_empty_batches(name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x = torch.empty(0, 70, dtype=_dt(name), device="cuda")
    y, mean, rstd = B.layer_norm_forward(x, save_stats=True)
    assert y.shape == x.shape and mean.numel() == 0
    junk = torch.full((70,), 3.0, device="cuda")
    dx, dw, db = B.layer_norm_backward(x, x, mean, rstd, dweight=junk)
    assert dx.shape == x.shape and not bool(dw.any()) and not bool(db.any()) and dw is junk


def test_replayed_in_a_graph_and_on_another_stream():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x, dy = _randn(700, 520, seed=1).bfloat16().cuda(), _randn(700, 520, seed=2).bfloat16().cuda()
    w, b = _randn(520, seed=3).float().cuda(), _randn(520, seed=4).float().cuda()

    def both():
        y, mean, rstd = B.layer_norm_forward(x, w, b, save_stats=True)
        return (y, mean, rstd) + B.layer_norm_backward(dy, x, mean, rstd, w, residual=dy)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    for k in range(3):
        x.copy_(_randn(700, 520, seed=10 + k))
        dy.copy_(_randn(700, 520, seed=20 + k))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(kept, both()):
            assert torch.equal(got, want)
        with torch.cuda.stream(side):
            other = both()
        torch.cuda.synchronize()
        for got, want in zip(kept, other):
            assert torch.equal(got, want)
