"""The matrix operators against plain float64 computations, through the Python binding.

Tolerances.  A result is rounded once to its type: at most eps/2 of its value.  The sums before that are fp32 with products that
are exact (16 bits) or off by 2^-24 (fp32 as planes): with n additions one after the other an element is off by at most n * 2^-23
times the sum of the absolute products (2^-23, not 2^-24: the matrix cores cut off instead of rounding).  n is at most one
addition for each four products and plane pair, and a few for joining parts and the epilogue."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

DTYPES = ("fp32", "bf16", "fp16")
ACTS = ("none", "relu", "gelu", "silu")
U23 = 2.0 ** -23


def _t():
    import torch
    return torch


def _dt(name):
    torch = _t()
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _adds(k, name):
    return k / 4 * (6 if name == "fp32" else 1) + 48


def _randn(*shape, seed, scale=1.0):
    torch = _t()
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale)


def _strided(v, dt, pad, shift):
    """v in the type dt on the GPU, its rows `pad` elements further apart and `shift` elements off an aligned address; and the whole buffer."""
    torch = _t()
    r, c = v.shape
    buf = torch.full((shift + r * (c + pad) + 8,), 7.5, dtype=dt, device="cuda")
    m = buf[shift:shift + r * (c + pad)].view(r, c + pad)[:, :c]
    m.copy_(v.to("cuda"))
    return m, buf


def _act64(name, z):
    torch = _t()
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope64(name, z):
    torch = _t()
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _within(got, ref, tol, what):
    bad = (got.double() - ref).abs() > tol
    assert not bool(bad.any()), "%s: %d of %d outside, worst %.3g times the tolerance" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - ref).abs() / tol.clamp_min(1e-300)).max()))


# (rows, in, out): single values, one row, one column, odd sizes, tile edges and their neighbours, long sums with few tiles
SIZES = [(1, 1, 1), (1, 8, 8), (2, 3, 1), (3, 5, 7), (1, 264, 100), (17, 64, 33), (16, 512, 10), (63, 65, 127), (64, 64, 64), (65, 8, 129),
         (128, 128, 128), (130, 200, 136), (257, 513, 300), (40, 4096, 24), (31, 1000, 1001), (300, 72, 1030), (2050, 40, 2049)]


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_forward(rows, cin, cout, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    i = SIZES.index((rows, cin, cout))
    act, pad, shift = ACTS[i % 4], (0, 8, 3)[i % 3], (0, 8, 1)[i % 3]
    x, _ = _strided(_randn(rows, cin, seed=i), dt, pad, shift)
    w, _ = _strided(_randn(cout, cin, seed=i + 100, scale=cin ** -0.5), dt, pad, shift)
    r, _ = _strided(_randn(rows, cout, seed=i + 200), dt, pad, shift)
    bias = _randn(cout, seed=i + 300).float().cuda()
    y, ybuf = _strided(torch.zeros(rows, cout), dt, pad, shift)
    before = ybuf.clone()
    out, z = B.linear_forward(x, w, bias, residual=r, activation=act, save_pre=True, out=y)
    assert out is y
    zr = x.double() @ w.double().T + bias.double()
    yr = _act64(act, zr) + r.double()
    sums = x.double().abs() @ w.double().abs().T + bias.double().abs()
    e, n = torch.finfo(dt).eps / 2, _adds(cin, name) * U23
    _within(z, zr, e * 1.01 * zr.abs() + n * sums, "z")
    _within(y, yr, e * 1.01 * yr.abs() + 1.13 * n * sums + 8 * U23 * (zr.abs() + yr.abs()), "y")
    y.zero_()
    before_m = before[shift:shift + rows * (cout + pad)].view(rows, cout + pad)[:, :cout]
    before_m.zero_()
    assert torch.equal(ybuf, before), "values outside y were written"
    # without bias, skip connection and z; y may be the skip connection
    plain = B.linear_forward(x, w)
    pr = x.double() @ w.double().T
    _within(plain, pr, e * 1.01 * pr.abs() + n * sums, "plain")
    y.copy_(r)
    B.linear_forward(x, w, bias, residual=y, activation=act, out=y)
    assert torch.equal(y, B.linear_forward(x, w, bias, residual=r, activation=act))


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin,cout", SIZES)
def test_backward(rows, cin, cout, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    i = SIZES.index((rows, cin, cout))
    act, pad, shift = ACTS[(i + 1) % 4], (8, 3, 0)[i % 3], (8, 1, 0)[i % 3]
    x, _ = _strided(_randn(rows, cin, seed=i + 1), dt, pad, shift)
    w, _ = _strided(_randn(cout, cin, seed=i + 101, scale=cin ** -0.5), dt, pad, shift)
    z, _ = _strided(_randn(rows, cout, seed=i + 201, scale=2.0), dt, pad, shift)
    dy, _ = _strided(_randn(rows, cout, seed=i + 301), dt, pad, shift)
    dx, dw, db = B.linear_backward(dy, x, w, z if act != "none" else None, activation=act)
    dz = dy.double() * _slope64(act, z.double())
    e = torch.finfo(dt).eps / 2
    once = (e if name != "fp32" else 0.0) + 16 * U23  # dz itself: rounded to 16 bits, made from fp32 functions
    # a slope near its zero is off by a few fp32 roundings of the terms that cancel there, not of itself
    off = once * dz.abs() + 16 * U23 * dy.double().abs()
    dxr, dwr, dbr = dz @ w.double(), dz.T @ x.double(), dz.sum(0)
    _within(dx, dxr, 1.01 * (e * dxr.abs() + off @ w.double().abs() + _adds(cout, name) * U23 * (dz.abs() @ w.double().abs())), "dx")
    _within(dw, dwr, 1.01 * (e * dwr.abs() + off.T @ x.double().abs() + _adds(rows, name) * U23 * (dz.abs().T @ x.double().abs())), "dw")
    _within(db, dbr, 1.01 * (16 * U23 * (dz.abs() + dy.double().abs()).sum(0) + (rows / 8 + 64) * U23 * dz.abs().sum(0)), "dbias")
    # one gradient at a time: the same bits, the others not made
    for k, full in (("dx", dx), ("dw", dw), ("dbias", db)):
        got = B.linear_backward(dy, x, w, z if act != "none" else None, activation=act, need=(k,))
        assert [g is not None for g in got] == [n == k for n in ("dx", "dw", "dbias")]
        assert torch.equal(got[("dx", "dw", "dbias").index(k)], full)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_are_differences(act):
    """fp32: the gradients against central differences of the layer itself, summed in float64.  A step h changes the loss by
    h times the gradient, up to h^2 times the third derivative, and the outputs carry fp32 errors: 1e-2 at h = 2^-7."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    rows, cin, cout, h = 9, 12, 7, 2.0 ** -7
    x, w = _randn(rows, cin, seed=1).float().cuda(), _randn(cout, cin, seed=2, scale=0.5).float().cuda()
    b, c = _randn(cout, seed=3).float().cuda(), _randn(rows, cout, seed=4).float().cuda()
    if act == "relu":  # keep every pre-activation away from the kink by more than a step can move it
        z = x.double() @ w.double().T + b.double()
        assert float(z.abs().min()) > 0
        c = torch.where(z.abs() > 0.1, c, torch.zeros_like(c))
    loss = lambda x, w, b: float((B.linear_forward(x, w, b, activation=act).double() * c.double()).sum())  # noqa: E731
    y, z = B.linear_forward(x, w, b, activation=act, save_pre=True)
    grads = B.linear_backward(c, x, w, z, activation=act)
    for arg, g in zip((0, 1, 2), grads):
        for k in (0, 5, -1):
            d = []
            for s in (h, -h):
                a = [x.clone(), w.clone(), b.clone()]
                a[arg].view(-1)[k] += s
                d.append(loss(*a))
            assert abs((d[0] - d[1]) / (2 * h) - float(g.view(-1)[k])) <= 1e-2 * max(1.0, float(g.abs().max()))


@pytest.mark.parametrize("name", DTYPES)
def test_infinities_and_nans_stay_where_arithmetic_puts_them(name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    rows, cin, cout = 70, 96, 140
    x, w = _randn(rows, cin, seed=5).to(dt).cuda(), _randn(cout, cin, seed=6).to(dt).cuda()
    ref = x.double() @ w.double().T
    x[3, 7] = float("inf")
    x[66, 95] = float("nan")
    w[130, 2] = float("-inf")
    want = x.double() @ w.double().T
    y = B.linear_forward(x, w)
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(torch.isposinf(y), torch.isposinf(want)) and torch.equal(torch.isneginf(y), torch.isneginf(want))
    fine = torch.isfinite(want)
    assert bool(fine.any()) and bool((~fine).any())
    tol = torch.finfo(dt).eps / 2 * 1.01 * ref.abs() + _adds(cin, name) * U23 * (torch.nan_to_num(x.double().abs(), posinf=0) @ torch.nan_to_num(w.double().abs(), posinf=0).T)
    _within(y[fine], want[fine], tol[fine], "y")
    if name == "fp32":  # the largest float is not the largest bf16
        big = torch.full((1, 8), torch.finfo(torch.float32).max, device="cuda")
        one = torch.zeros(1, 8, device="cuda")
        one[0, 3] = 0.5
        assert float(B.linear_forward(big, one)) == pytest.approx(3.4028235e38 / 2, rel=1e-6)
    # the same in the gradients: an infinity in one sample reaches that sample's dx and everything of dw's column
    dy = _randn(rows, cout, seed=7).to(dt).cuda()
    dy[11, 13] = float("inf")
    x, w = _randn(rows, cin, seed=5).to(dt).cuda(), _randn(cout, cin, seed=6).to(dt).cuda()
    dx, dw, db = B.linear_backward(dy, x, w)
    dxr, dwr = dy.double() @ w.double(), dy.double().T @ x.double()
    for got, want in ((dx, dxr), (dw, dwr)):
        assert torch.equal(torch.isposinf(got), torch.isposinf(want)) and torch.equal(torch.isneginf(got), torch.isneginf(want))
        assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert math.isinf(float(db[13])) and bool(torch.isfinite(db[:13]).all())


def test_empty_batch():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x, w = torch.zeros(0, 24, device="cuda", dtype=torch.bfloat16), torch.ones(10, 24, device="cuda", dtype=torch.bfloat16)
    assert B.linear_forward(x, w).shape == (0, 10)
    dx, dw, db = B.linear_backward(torch.zeros(0, 10, device="cuda", dtype=torch.bfloat16), x, w)
    assert dx.shape == (0, 24) and int(dw.abs().sum()) == 0 and int(db.abs().sum()) == 0 and dw.shape == (10, 24)


def test_rows_further_apart_than_32_bits():
    """Rows whose offsets pass 2^31 elements: the last rows of a long matrix with a large leading dimension."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    ld, rows, cin, cout = 1 << 21, 1100, 64, 40
    buf = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")  # 4.6 GB
    x = buf.view(rows, ld)[:, 8:8 + cin]
    x.copy_(_randn(rows, cin, seed=1))
    w = _randn(cout, cin, seed=2).to(torch.bfloat16).cuda()
    assert torch.equal(B.linear_forward(x, w), B.linear_forward(x.contiguous(), w))
    dy = _randn(rows, cout, seed=3).to(torch.bfloat16).cuda()
    a, b = B.linear_backward(dy, x, w), B.linear_backward(dy, x.contiguous(), w)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_linear_on_another_stream_and_in_a_graph():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x, w = _randn(300, 200, seed=1).to(torch.float16).cuda(), _randn(100, 200, seed=2).to(torch.float16).cuda()
    b = _randn(100, seed=3).float().cuda()
    dy = _randn(300, 100, seed=4).to(torch.float16).cuda()

    def layer():
        y, z = B.linear_forward(x, w, b, activation="gelu", save_pre=True)
        return (y, z) + B.linear_backward(dy, x, w, z, activation="gelu")

    ref = [t.clone() for t in layer()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = layer()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer()
    for k in range(3):
        x.copy_(_randn(300, 200, seed=10 + k))
        g.replay()
        torch.cuda.synchronize()
        want = layer()
        assert all(torch.equal(p, q) for p, q in zip(want, out))


# ---- orthogonalised updates ------------------------------------------------------------------------------------------------

CO = (3.4445, -4.7750, 2.0315)
# A relative error of the first iterate grows by at most a at each step.  Its planes and those of the products are off by 2^-24
# of a value each, the sums by 2^-23: with all of them as large as the first one, at five steps,
ORTHO_TOL = CO[0] ** 5 * 2.0 ** -22


def _newton_schulz(g, steps=5, co=None, eps=1e-7):
    torch = _t()
    x = g.double()
    x = x / max(float(x.norm()), eps)
    co = co or [CO] * steps
    tall = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if tall else x
    for a, b, c in co:
        s = torch.mm(x, x.T.contiguous())
        x = a * x + torch.mm(b * s + c * torch.mm(s, s), x)
    return x.T if tall else x


def _flat(mats, name, seed, scale=1.0):
    torch = _t()
    return torch.cat([_randn(r * c, seed=seed + i, scale=scale) for i, (r, c) in enumerate(mats)]).to(_dt(name)).cuda()


LISTS = [[(1, 1)], [(1, 9)], [(9, 1)], [(7, 5)], [(8, 27), (8, 72), (10, 8)], [(64, 64)], [(65, 63), (63, 65), (64, 200), (200, 64)],
         [(100, 512), (512, 100), (3, 1000), (1000, 3)], [(129, 1153), (300, 257), (17, 17), (256, 64), (64, 27), (1, 3), (130, 520)],
         [(512, 1024), (1024, 512), (512, 512)], [(48, 9000)]]


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("i", range(len(LISTS)))
def test_orthogonalize(i, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = LISTS[i]
    g = _flat(mats, name, 50 + i, scale=(1.0, 1e-3)[i % 2])
    p = B.Orthogonalizer(mats)
    o = p.orthogonalize(g)
    at = 0
    for r, c in mats:
        ref = _newton_schulz(g[at:at + r * c].view(r, c))
        err = float((o[at:at + r * c].view(r, c).double() - ref).norm() / ref.norm())
        assert err <= ORTHO_TOL + torch.finfo(_dt(name)).eps / 2, "%d x %d: %.3g" % (r, c, err)
        at += r * c
    assert torch.equal(o, p.orthogonalize(g))  # nothing is kept from call to call
    h = g.clone()
    assert p.orthogonalize(h, h) is h and torch.equal(h, o)  # in place
    p.close()


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
def test_orthogonalize_steps_and_coefficients(steps):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = [(40, 90), (90, 40), (33, 33)]
    g = _flat(mats, "fp32", 7)
    co = [(2.0 + 0.05 * k, -1.5, 0.5) for k in range(steps)]
    o = B.Orthogonalizer(mats, steps=steps, coefficients=co).orthogonalize(g)
    at = 0
    for r, c in mats:
        ref = _newton_schulz(g[at:at + r * c].view(r, c), steps, co)
        grown = float(np.prod([a for a, _, _ in co]))
        assert float((o[at:at + r * c].view(r, c).double() - ref).norm() / ref.norm()) <= grown * 2.0 ** -21
        at += r * c


def test_orthogonalize_spectra():
    """Matrices of one large and many small singular values: what is lost in the small ones is multiplied by a at each step."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    m, n = 96, 200
    u, v = torch.linalg.qr(_randn(m, m, seed=1))[0], torch.linalg.qr(_randn(n, m, seed=2))[0]
    for lo in (1e-1, 1e-2, 1e-4):
        g = ((u * torch.logspace(0, math.log10(lo), m, dtype=torch.float64)) @ v.T).float().cuda()
        ref = _newton_schulz(g)
        o = B.Orthogonalizer([(m, n)]).orthogonalize(g.view(-1)).view(m, n)
        assert float((o.double() - ref).norm() / ref.norm()) <= ORTHO_TOL


def test_orthogonalize_extremes():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = [(24, 40)] * 6
    n = 24 * 40
    g = _flat(mats, "fp32", 3)
    ref = _newton_schulz(g[:n].view(24, 40))
    g[n:2 * n] = 0                              # zeros
    g[2 * n:3 * n] = g[:n] * 2.0 ** 100         # squares beyond fp32
    g[3 * n:4 * n] = g[:n] * 2.0 ** -100        # smaller than eps: divided by it
    g[4 * n + 5] = float("inf")
    g[5 * n + 7] = float("nan")
    o = B.Orthogonalizer(mats).orthogonalize(g)
    assert float((o[:n].view(24, 40).double() - ref).norm() / ref.norm()) <= ORTHO_TOL
    assert int(torch.count_nonzero(o[n:2 * n])) == 0
    assert float((o[2 * n:3 * n].view(24, 40).double() - ref).norm() / ref.norm()) <= ORTHO_TOL
    assert float(o[3 * n:4 * n].abs().max()) < 1e-15
    assert bool(torch.isnan(o[4 * n:]).all())
    o = B.Orthogonalizer(mats[:4], eps=1e-38).orthogonalize(g[:4 * n].clone())
    assert float((o[3 * n:].view(24, 40).double() - ref).norm() / ref.norm()) <= ORTHO_TOL


def test_orthogonalize_places_and_types():
    """Matrices side by side, rows apart, odd offsets; elements between them are left alone; output of another type."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = [(3, 10, 20, 50), (3 + 23, 10, 27, 50), (777, 33, 65, 71)]
    g = _randn(777 + 33 * 71, seed=9).to(torch.bfloat16).cuda()
    p = B.Orthogonalizer(mats)
    for name in DTYPES:
        out = torch.full_like(g, 5.0, dtype=_dt(name))
        p.orthogonalize(g, out)
        inside = torch.zeros_like(g, dtype=torch.bool)
        for off, r, c, ld in mats:
            view = lambda t: torch.as_strided(t, (r, c), (ld, 1), off)  # noqa: E731
            ref = _newton_schulz(view(g))
            assert float((view(out).double() - ref).norm() / ref.norm()) <= ORTHO_TOL + torch.finfo(_dt(name)).eps / 2
            view(inside).fill_(True)
        assert bool((out[~inside] == 5.0).all())


def _muon64(w, v, g, mats, lr, mu, nesterov, decay, scale, gs):
    torch = _t()
    w, v, g = w.double(), v.double(), g.double() * gs
    v = mu * v + g
    u = g + mu * v if nesterov else v
    out, at = [], 0
    for r, c in mats:
        s = {"none": 1.0, "aspect": math.sqrt(max(1.0, r / c)), "rms": 0.2 * math.sqrt(max(r, c))}[scale]
        out.append(-lr * s * _newton_schulz(u[at:at + r * c].view(r, c)).reshape(-1))
        at += r * c
    d = torch.cat(out)
    return (1 - lr * decay) * w + d, v, d


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("i", [4, 6, 8, 9])
def test_muon_update(i, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = LISTS[i]
    scale, nesterov, gs = ("none", "aspect", "rms")[i % 3], i % 2 == 0, (1.0, 1 / 1024)[name == "fp16"]
    g = _flat(mats, name, 20 + i, scale=1e-2 / gs * 0.1)
    w, v = _flat(mats, "fp32", 300 + i), _flat(mats, "fp32", 400 + i, scale=1e-3)
    w16 = torch.zeros_like(w, dtype=torch.bfloat16 if i % 2 else torch.float16)
    flag = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    p = B.Orthogonalizer(mats)
    for step in range(2):
        wr, vr, d = _muon64(w, v, g, mats, 0.02, 0.95, nesterov, 0.1, scale, gs)
        p.muon_update(w, v, g, lr=0.02, momentum=0.95, nesterov=nesterov, weight_decay=0.1, scale=scale, grad_scale=gs, weights16=w16, skipped=flag)
        assert int(flag) == 0
        _within(v, vr, 2 * U23 * (vr.abs() + g.double().abs() * gs), "v")
        # three roundings of the weight, one of the step; the direction is off by its tolerance in norm
        off = w.double() - wr
        assert float(off.norm()) <= 2 * U23 * float(wr.norm()) + ORTHO_TOL * float(d.norm())
        assert torch.equal(w16, w.to(w16.dtype))
    p.close()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_muon_skips_an_update_that_is_not_finite(bad):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = LISTS[8]
    g, w, v = _flat(mats, "bf16", 1), _flat(mats, "fp32", 2), _flat(mats, "fp32", 3)
    w16 = w.to(torch.bfloat16)
    p = B.Orthogonalizer(mats)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = g.clone()
    g[-3] = bad
    w0, v0, h0 = w.clone(), v.clone(), w16.clone()
    p.muon_update(w, v, g, lr=0.1, weights16=w16, skipped=flag)
    assert int(flag) == 1
    assert torch.equal(w, w0) and torch.equal(v, v0) and torch.equal(w16, h0)
    p.muon_update(w, v, good, lr=0.1, weights16=w16, skipped=flag)  # and the next one is made
    assert int(flag) == 0 and not torch.equal(w, w0)
    w1, v1 = w0.clone(), v0.clone()
    B.Orthogonalizer(mats).muon_update(w1, v1, good, lr=0.1)
    assert torch.equal(w, w1) and torch.equal(v, v1)


def test_muon_leaves_the_rest_of_a_flat_vector_alone():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = [(5, 16, 27, 27), (5 + 16 * 27 + 32, 8, 16, 16)]  # a convolution, its 16 scales and shifts, another layer
    n = 5 + 16 * 27 + 32 + 8 * 16 + 11
    g, w, v = _randn(n, seed=1).float().cuda(), _randn(n, seed=2).float().cuda(), _randn(n, seed=3).float().cuda()
    w0, v0 = w.clone(), v.clone()
    B.Orthogonalizer(mats).muon_update(w, v, g, lr=0.1)
    changed = torch.zeros(n, dtype=torch.bool, device="cuda")
    for off, r, c, ld in mats:
        changed[off:off + r * c] = True
    assert torch.equal(w[~changed], w0[~changed]) and torch.equal(v[~changed], v0[~changed])
    assert bool((w[changed] != w0[changed]).all())


def test_muon_on_another_stream_and_in_a_graph():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    mats = LISTS[6]
    g, w, v = _flat(mats, "bf16", 1), _flat(mats, "fp32", 2), _flat(mats, "fp32", 3)
    p = B.Orthogonalizer(mats)
    q = B.Orthogonalizer(mats)
    w0, v0 = w.clone(), v.clone()
    for k in range(4):
        q.muon_update(w0, v0, g, lr=0.1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.muon_update(w, v, g, lr=0.1)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.muon_update(w, v, g, lr=0.1)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
    assert torch.equal(w, w0) and torch.equal(v, v0)


def test_refusals_of_device_arguments():
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    with pytest.raises(ValueError, match="w: expected"):
        B.linear_forward(x, torch.zeros(6, 9, device="cuda"))
    with pytest.raises(TypeError, match="w: expected"):
        B.linear_forward(x, w.half())
    with pytest.raises(TypeError, match="float32"):
        B.linear_forward(x, w, torch.zeros(6, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError, match="bias"):
        B.linear_forward(x, w, torch.zeros(7, device="cuda"))
    with pytest.raises(ValueError, match="next to each other"):
        B.linear_forward(torch.zeros(8, 4, device="cuda").T, w)
    with pytest.raises(TypeError, match="float64"):
        B.linear_forward(x.double(), w.double())
    with pytest.raises(ValueError, match="z "):
        B.linear_backward(torch.zeros(4, 6, device="cuda"), x, w, activation="relu")
    p = B.Orthogonalizer([(4, 8)])
    with pytest.raises(ValueError, match="at least 32"):
        p.orthogonalize(torch.zeros(31, device="cuda"))
    with pytest.raises(TypeError, match="unexpected type"):
        p.muon_update(torch.zeros(32, device="cuda").half(), torch.zeros(32, device="cuda"), torch.zeros(32, device="cuda"), lr=0.1)
    with pytest.raises(ValueError, match="scale"):
        p.muon_update(torch.zeros(32, device="cuda"), torch.zeros(32, device="cuda"), torch.zeros(32, device="cuda"), lr=0.1, scale="max")
