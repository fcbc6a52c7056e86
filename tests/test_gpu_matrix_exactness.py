"""How exact the matrix operators are in the 2-norm, where the limits of single elements (test_gpu_matrix.py) see little."""
import math

import pytest

pytestmark = pytest.mark.gpu

CO = (3.4445, -4.7750, 2.0315)


def _steps(g, dtype, steps=5):
    """Newton-Schulz steps in elementary operations of one type, on the CPU."""
    import torch
    a, b, c = CO
    x = (g.double() / g.double().norm()).to(dtype)
    for _ in range(steps):
        s = torch.mm(x, x.T.contiguous())
        x = a * x + torch.mm(b * s + c * torch.mm(s, s), x)
    return x


def _spectrum(m, n, small, large, seed):
    """An m x n matrix of `large` singular values of 1, the others `small`."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    u = torch.linalg.qr(torch.randn(m, m, generator=gen, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(n, m, generator=gen, dtype=torch.float64))[0]
    s = torch.full((m,), small, dtype=torch.float64)
    s[:large] = 1.0
    return torch.mm(u * s, v.T.contiguous()).float()


def _far(x, ref):
    return float((x.double().cpu() - ref).norm() / ref.norm())


@pytest.mark.parametrize("steps", [2, 3, 4, 5])
@pytest.mark.parametrize("m,n", [(2, 5), (8, 72), (10, 64), (32, 64), (64, 300), (100, 512), (192, 700)])
def test_orthogonalize_where_few_directions_outweigh_the_others(m, n, steps):
    """An error d of A grows by at most a^2 = 11.9 until the next step on A, whose P is then off by 4.775 / 3.4445 of that, relative to what it
    does to small directions.  With three roundings of 2^-23 a product: two steps on A between iterates, 11.9 * 1.39 * 3 * 2^-23 = 6e-6 < 2^-17 beside the
    error of the same steps in fp32 (its roundings and these are not the same ones: twice); three steps, 11.9 times as much, < 2^-13."""
    import torch
    from paper_2105_00619_amd import binding as B
    for small in (0.5, 0.2, 0.1, 0.05, 0.02, 0.01, 3e-3, 1e-3):
        for large in {1, max(1, m // 16)}:
            g = _spectrum(m, n, small, large, seed=m + n)
            ref = _steps(g, torch.float64, steps)
            plain = _far(_steps(g, torch.float32, steps), ref)
            plan = B.Orthogonalizer([(m, n)], steps=steps)
            for dt, more in ((torch.float32, 2.0 ** -17), (torch.float16, 2.0 ** -17), (torch.bfloat16, 2.0 ** -13)):
                out = torch.empty(m * n, dtype=dt, device="cuda")
                plan.orthogonalize(g.reshape(-1).cuda(), out)
                rounding = _far(ref.to(dt), ref) if dt != torch.float32 else 0.0
                assert _far(out.view(m, n), ref) <= 2 * plain + more + 1.05 * rounding, (small, large, dt, plain)
            # an update of nothing but this step
            w, v = torch.zeros(m * n, device="cuda"), torch.zeros(m * n, device="cuda")
            plan.muon_update(w, v, g.reshape(-1).cuda(), lr=1.0, momentum=0.0, scale="none")
            assert _far(-w.view(m, n), ref) <= 2 * plain + 2.0 ** -17 + 2.0 ** -23, (small, large, "update", plain)
            plan.close()


def test_an_iterate_made_in_place_is_the_one_made_apart():
    """Three steps take one iterate on the way, which low matrices make where the first one lies; beside a taller matrix they do not."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator().manual_seed(3)
    low, tall = [(40, 3000), (3000, 40)], [(600, 640)]
    n = sum(r * c for r, c in low)
    g = torch.randn(n + 600 * 640, generator=gen).cuda()
    one, two = B.Orthogonalizer(low, steps=3), B.Orthogonalizer(low + tall, steps=3)
    assert one.workspace_bytes < 2 * 4 * 2 * 64 * 3008
    a, b = one.orthogonalize(g[:n].clone()), two.orthogonalize(g)
    for at in (0, 40 * 3000):
        ref = _steps(g[at:at + 120000].cpu().view((40, 3000) if at == 0 else (3000, 40)), torch.float64, 3) if at == 0 else \
            _steps(g[at:at + 120000].cpu().view(3000, 40).T.contiguous(), torch.float64, 3).T
        for o in (a, b):
            assert _far(o[at:at + 120000].view(ref.shape), ref) <= 1e-5


def _slope64(act, z):
    import torch
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return (z > 0).double() if act == "relu" else torch.ones_like(z)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["gelu", "silu", "relu", "none"])
@pytest.mark.parametrize("rows,cin,cout", [(3, 40, 24), (257, 333, 514), (1000, 64, 8), (2100, 520, 2056), (24, 1000, 4100)])
def test_gradients_in_16_bits_are_rounded_once(rows, cin, cout, act, name):
    """What the rounding of the result makes, and nothing of its size beside it: dz is held to twice the bits of the type (2^-16 and
    less), its products are exact and added in fp32 (2^-20 and less of a result whose terms have either sign)."""
    import torch
    from paper_2105_00619_amd import binding as B
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[name]
    gen = torch.Generator(device="cuda").manual_seed(rows)
    make = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(dt)  # noqa: E731
    dy, x, w, z = make(rows, cout), make(rows, cin), make(cout, cin, cin ** -0.5), make(rows, cout, 1.5)
    dx, dw, _ = B.linear_backward(dy, x, w, z, activation=act)
    dz = dy.double() * _slope64(act, z.double())
    for got, ref in ((dx, torch.mm(dz, w.double())), (dw, torch.mm(dz.T.contiguous(), x.double()))):
        once = float((ref.to(dt).double() - ref).norm() / ref.norm())
        assert float((got.double() - ref).norm() / ref.norm()) <= once * (1 + 2.0 ** -6) + 2.0 ** -16


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("rows,cin,cout", [(5, 24, 16), (300, 264, 520), (1100, 72, 40)])
def test_gradients_in_fp16_have_the_range_of_their_results(rows, cin, cout, act):
    """dy near the largest fp16 times a slope above 1 is no infinity where dx and dw are none; an infinite weight or sample makes the
    infinities and NaNs that one product of fp32 values makes, whatever the planes of dz."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(rows)
    dy = torch.randint(-3, 4, (rows, cout), generator=gen, device="cuda").half()
    z = torch.randn(rows, cout, generator=gen, device="cuda").half()
    x, w = (torch.randn(rows, cin, generator=gen, device="cuda") * 1e-3).half(), (torch.randn(cout, cin, generator=gen, device="cuda") * 1e-2).half()
    dy[2, 3], dy[4, 7], z[2, 3], z[4, 7] = 65000.0, -65000.0, 1.5, 2.25
    slope = _slope64(act, z.double())
    assert float((dy.double() * slope).abs().max()) > 65504 * 1.05
    dx, dw, db = B.linear_backward(dy, x, w, z, activation=act)
    dz = dy.double() * slope
    for got, ref in ((dx, torch.mm(dz, w.double())), (dw, torch.mm(dz.T.contiguous(), x.double()))):
        once = float((ref.half().double() - ref).norm() / ref.norm())
        assert float((got.double() - ref).norm() / ref.norm()) <= once * (1 + 2.0 ** -6) + 2.0 ** -16
    w[5, 2], x[3, 1], x[1, 0] = float("inf"), float("-inf"), float("nan")
    dx, dw, db = B.linear_backward(dy, x, w, z, activation=act)
    for got, ref in ((dx, torch.mm(dz, w.double())), (dw, torch.mm(dz.T.contiguous(), x.double()))):
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(torch.isposinf(got), torch.isposinf(ref)) and torch.equal(torch.isneginf(got), torch.isneginf(ref))


@pytest.mark.parametrize("name", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,width", [(40, 40), (1000, 40), (2000, 200)])
def test_gelu_and_its_slope_have_their_bits_in_the_tail(rows, width, name):
    """x = z, w = 1: every output is GELU of one value, relative to which (not to 1) it is off by the polynomial (fp32 2e-8, 16 bits 4e-6) and
    a handful of roundings: 2^-20 and 2^-16, beside the rounding to 16 bits (of values below the smallest normal one: of that)."""
    import torch
    from paper_2105_00619_amd import binding as B
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]
    far = -12.5 if name != "fp16" else -5.0
    z = torch.linspace(far, 9.0, rows * width, device="cuda", dtype=torch.float64)[torch.randperm(rows * width, device="cuda")].view(rows, width).to(dt)
    one = torch.eye(width, device="cuda", dtype=dt)
    y = B.linear_forward(z, one, activation="gelu")
    phi = 0.5 * torch.special.erfc(-z.double() / math.sqrt(2))
    density = torch.exp(-z.double() ** 2 / 2) / math.sqrt(2 * math.pi)
    info = torch.finfo(dt)
    more, half = (2.0 ** -20, 0.0) if name == "fp32" else (2.0 ** -16, info.eps / 2)
    least = info.smallest_normal * half
    want = z.double() * phi
    assert bool(((y.double() - want).abs() <= (more + half) * want.abs() + least).all())
    dx, _, _ = B.linear_backward(torch.ones_like(z), z, one, z, activation="gelu")
    want = phi + z.double() * density
    assert bool(((dx.double() - want).abs() <= more * (phi + z.double().abs() * density) + half * want.abs() + least).all())


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("size", [1e-1, 1e-3, 1e-4, 2e-5])
@pytest.mark.parametrize("rows,cin,cout", [(130, 264, 96), (520, 1032, 2056), (3085, 4104, 72), (72, 3080, 4104)])
def test_small_gradients_in_fp16_keep_their_bits(rows, cin, cout, size, act):
    """dy near fp16's smallest values, weights and samples of order one: dz = dy act'(z) has more bits than fp16 has there, and so have the
    results, which are rounded once."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(rows)
    make = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).half()  # noqa: E731
    dy, x, w, z = make(rows, cout, size), make(rows, cin), make(cout, cin), make(rows, cout, 1.5)
    dx, dw, _ = B.linear_backward(dy, x, w, z, activation=act)
    dz = dy.double() * _slope64(act, z.double())
    for got, ref in ((dx, torch.mm(dz, w.double())), (dw, torch.mm(dz.T.contiguous(), x.double()))):
        once = float((ref.half().double() - ref).norm() / ref.norm())
        assert float((got.double() - ref).norm() / ref.norm()) <= once * (1 + 2.0 ** -6) + 2.0 ** -16
