"""Every tile that the matrix operators choose, at sizes for which the library says that it chooses them: 64, 128 and 256 values square, sums whole
and cut, in each direction and type."""
import ctypes as C
import math

import pytest

pytestmark = pytest.mark.gpu

DT = {"fp32": 0, "bf16": 1, "fp16": 2}
ACT = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


def _torch_type(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _layer(rows, cin, cout, name, act):
    """(edge, cut?) of y, dx and dw, asked from the library's own host function; aligned operands, as torch gives them."""
    from paper_2105_00619_amd import binding as B
    f = getattr(B.load_library(), "_ZN4oseq12linear_shapeEPK16optorch_linear_tbi")
    f.argtypes, f.restype = [C.POINTER(B.optorch_linear_t), C.c_bool, C.c_int], C.c_int
    a = B.optorch_linear_t()
    a.precision, a.activation, a.rows, a.in_features, a.out_features = DT[name], ACT[act], rows, cin, cout
    for n, cols in (("x", cin), ("w", cin), ("y", cout), ("z", cout), ("dy", cout), ("dx", cin), ("dw", cin)):
        setattr(a, n, 1 << 20)
        setattr(a, "ld" + n, cols)
    s = [f(C.byref(a), k > 0, k) for k in range(3)]
    return {n: (v // 1000, v % 1000 > 1) for n, v in zip(("y", "dx", "dw"), s)}


def _far(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


def _sums(k, name):
    """Relative error of sums of k products in the 2-norm: fp32 additions, for fp32 operands six for each sixteen values of k, each off by 2^-25
    of the sum in the mean, in either direction; half as much again, and the rounding of an fp32 result.  (Two planes of three: 2.2e-6.)"""
    return 1.5 * math.sqrt(k / 16 * (6 if name == "fp32" else 1)) * 2.0 ** -25 + 2.0 ** -23


# product, tile and cut; a layer that has it for each type
LAYERS = [
    ("y", 64, False, dict(fp32=(267, 65, 70), bf16=(267, 65, 70), fp16=(270, 64, 72))),
    ("y", 64, True, dict(fp32=(267, 523, 66), bf16=(270, 2061, 66), fp16=(264, 2056, 72))),
    ("y", 128, False, dict(fp32=(1029, 67, 3085), bf16=(1033, 64, 3080), fp16=(1027, 69, 3083))),
    ("y", 128, True, dict(fp32=(267, 1035, 2059), bf16=(521, 3080, 1032), fp16=(515, 3085, 1031))),
    ("y", 256, False, dict(fp32=(4091, 257, 4091), bf16=(3085, 72, 4104), fp16=(3083, 65, 4101))),
    ("y", 256, True, dict(fp32=(2051, 6151, 4099), bf16=(1035, 6152, 4104), fp16=(1031, 6157, 4099))),
    ("dx", 64, False, dict(fp32=(65, 66, 67), bf16=(65, 72, 64), fp16=(65, 66, 67))),
    ("dx", 64, True, dict(fp32=(65, 66, 523), bf16=(70, 72, 2064), fp16=(65, 67, 2059))),
    ("dx", 128, False, dict(fp32=(1029, 3085, 66), bf16=(1029, 3080, 64), fp16=(1027, 3083, 69))),
    ("dx", 128, True, dict(fp32=(267, 2059, 1035), bf16=(521, 1032, 3080), fp16=(515, 1031, 3085))),
    ("dx", 256, False, dict(fp32=(4091, 4091, 257), bf16=(3085, 4104, 72), fp16=(3083, 4101, 65))),
    ("dx", 256, True, dict(fp32=(2051, 4099, 6151), bf16=(1035, 4104, 6152), fp16=(1031, 4099, 6157))),
    ("dw", 64, False, dict(fp32=(65, 66, 67), bf16=(65, 72, 64), fp16=(65, 66, 67))),
    ("dw", 64, True, dict(fp32=(523, 66, 65), bf16=(2059, 72, 64), fp16=(2061, 65, 67))),
    ("dw", 128, False, dict(fp32=(66, 1029, 3085), bf16=(66, 1032, 3080), fp16=(69, 1027, 3083))),
    ("dw", 128, True, dict(fp32=(1035, 267, 2059), bf16=(3083, 520, 1032), fp16=(3085, 515, 1031))),
    ("dw", 256, False, dict(fp32=(257, 4091, 4091), bf16=(72, 3080, 4104), fp16=(65, 3083, 4101))),
    ("dw", 256, True, dict(fp32=(6151, 2051, 4099), bf16=(6152, 1032, 4104), fp16=(6157, 1031, 4099))),
]


@pytest.mark.parametrize("name", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("i", range(len(LAYERS)))
def test_layers(i, name):
    """Once without an activation and once with GELU, whose dz has two planes in 16 bits: results as exact as their sums and one rounding, the
    sums of every part and edge among them (the worst element is within what test_gpu_matrix.py allows); an infinity and a NaN where
    arithmetic puts them."""
    import torch
    from paper_2105_00619_amd import binding as B
    product, edge, cut, sizes = LAYERS[i]
    rows, cin, cout = sizes[name]
    dt = _torch_type(name)
    gen = torch.Generator(device="cuda").manual_seed(i)
    make = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(dt)  # noqa: E731
    x, w, dy, z = make(rows, cin), make(cout, cin, cin ** -0.5), make(rows, cout), make(rows, cout)
    k = {"y": cin, "dx": cout, "dw": rows}[product]
    half = torch.finfo(dt).eps / 2
    for act in ("none", "gelu"):
        if not (act == "gelu" and product != "y" and name != "fp32"):  # (twice as long a reduction: its own sizes below)
            assert _layer(rows, cin, cout, name, act)[product] == (edge, cut), (act, _layer(rows, cin, cout, name, act))

        def run(x, w, dy):
            if product == "y":
                return B.linear_forward(x, w, activation=act)
            return B.linear_backward(dy, x, w, z if act != "none" else None, activation=act, need=(product,))[product == "dw"]

        def exact(x, w, dy):
            x, w, dy = x.double(), w.double(), dy.double()
            if act == "gelu":
                phi = lambda t: 0.5 * torch.special.erfc(-t / math.sqrt(2))  # noqa: E731
                t = z.double()
                dy = dy * (phi(t) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi))
            if product == "y":
                t = torch.mm(x, w.T.contiguous())
                return t * phi(t) if act == "gelu" else t
            return torch.mm(dy, w) if product == "dx" else torch.mm(dy.T.contiguous(), x)

        got, ref = run(x, w, dy), exact(x, w, dy)
        once = _far(ref.to(dt), ref)
        assert _far(got, ref) <= once * (1 + 2.0 ** -6) + _sums(k, name) + 2.0 ** -20 * (act == "gelu") + 2.0 ** -16 * (name != "fp32")
        size = {"y": (x, w), "dx": (dy, w), "dw": (dy, x)}[product]
        worst = float(size[0].double().norm(dim=1).max() if product != "dw" else size[0].double().norm(dim=0).max()) * float(
            size[1].double().norm(dim=1 if product == "y" else 0).max())
        assert float((got.double() - ref).abs().max()) <= half * 1.01 * float(ref.abs().max()) + (k / 4 * (6 if name == "fp32" else 1) + 48) * 2.0 ** -23 * 1.2 * worst
        # the last sample, output and feature, where a tile or a part ends
        a, b, c = x.clone(), w.clone(), dy.clone()
        if product == "y":
            a[rows - 1, cin - 1], b[cout - 1, 0] = float("inf"), float("nan")
        elif product == "dx":
            c[rows - 1, cout - 1], b[0, cin - 1] = float("inf"), float("nan")
        else:
            c[rows - 1, cout - 1], a[0, cin - 1] = float("inf"), float("nan")
        bad, fine = run(a, b, c), torch.ones_like(got, dtype=torch.bool)
        fine[-1], fine[:, -1] = False, False
        assert torch.equal(bad[fine], got[fine])
        assert not bool(torch.isfinite(bad[-1]).any()) and bool(torch.isnan(bad[:, -1]).all())


TWICE = [("dx", 64, False, (65, 72, 64)), ("dx", 64, True, (70, 72, 1040)), ("dx", 128, False, (1029, 3080, 64)), ("dx", 128, True, (521, 1032, 2056)),
         ("dx", 256, False, (3085, 4104, 72)), ("dx", 256, True, (1035, 4104, 3496)),
         ("dw", 64, False, (65, 72, 64)), ("dw", 64, True, (1031, 72, 64)), ("dw", 128, False, (66, 1032, 3080)), ("dw", 128, True, (2059, 520, 1032)),
         ("dw", 256, False, (72, 3080, 4104)), ("dw", 256, True, (3501, 1032, 4104))]


@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("product,edge,cut,size", TWICE)
def test_gradients_with_two_planes(product, edge, cut, size, act, name):
    import torch
    from paper_2105_00619_amd import binding as B
    rows, cin, cout = size
    assert _layer(rows, cin, cout, name, act)[product] == (edge, cut), _layer(rows, cin, cout, name, act)
    dt = _torch_type(name)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    make = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(dt)  # noqa: E731
    x, w, dy, z = make(rows, cin), make(cout, cin, cin ** -0.5), make(rows, cout), make(rows, cout)
    t = z.double()
    s = torch.sigmoid(t)
    slope = 0.5 * torch.special.erfc(-t / math.sqrt(2)) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi) if act == "gelu" else s * (1 + t * (1 - s))
    dz = dy.double() * slope
    got = B.linear_backward(dy, x, w, z, activation=act, need=(product,))[product == "dw"]
    ref = torch.mm(dz, w.double()) if product == "dx" else torch.mm(dz.T.contiguous(), x.double())
    assert _far(got, ref) <= _far(ref.to(dt), ref) * (1 + 2.0 ** -6) + 2.0 ** -16


# ---- orthogonalised updates ------------------------------------------------------------------------------------------------

CO = (3.4445, -4.7750, 2.0315)
GRAM, CHAIN, APPLY, LAST, WEIGHTS = range(5)


def _plan_shape(plan, which):
    from paper_2105_00619_amd import binding as B
    f = getattr(B.load_library(), "_ZN4oseq11ortho_shapeEPK13optorch_orthoi")
    f.argtypes, f.restype = [C.c_void_p, C.c_int], C.c_int
    v = f(plan.handle, which)
    return v // 1000, bool(v % 1000)


def _steps(g, dtype, steps):
    import torch
    a, b, c = CO
    x = (g.double() / g.double().norm()).to(dtype)
    tall = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if tall else x
    for _ in range(steps):
        s = torch.mm(x, x.T.contiguous())
        x = a * x + torch.mm(b * s + c * torch.mm(s, s), x)
    return x.T if tall else x


LISTS = [
    ([(299, 1205)], 3, {GRAM: (64, True), CHAIN: (64, False), LAST: (64, False)}),
    ([(1299, 1307)] * 4, 3, {CHAIN: (64, True)}),
    ([(699, 2805), (2805, 699)] * 2, 3, {GRAM: (128, True)}),
    ([(1999, 2007), (2007, 1999)] * 2, 3, {CHAIN: (128, True)}),
    ([(299, 4805), (4805, 299)] * 2, 3, {APPLY: (128, False), LAST: (128, False)}),
    ([(519, 8327), (8327, 519)], 2, {WEIGHTS: (128, False)}),
    ([(2499, 2507)], 2, {GRAM: (128, False), CHAIN: (128, False)}),
    ([(2499, 2507), (2507, 2499)] * 2, 3, {GRAM: (256, False), CHAIN: (256, False)}),
    ([(2999, 4507)], 2, {GRAM: (256, True), WEIGHTS: (256, False)}),
    ([(4505, 4499), (4499, 4505)], 3, {CHAIN: (256, True)}),
    ([(1299, 10405), (10405, 1299)], 3, {APPLY: (256, False)}),
    ([(999, 16005), (16005, 999)], 2, {LAST: (256, False)}),
    ([(2999, 4507), (4507, 2999), (17, 40)], 2, {WEIGHTS: (256, False)}),
]


@pytest.mark.parametrize("i", range(len(LISTS)))
def test_orthogonalised_updates(i):
    """Against the same steps in 64 bits, by the limits of test_gpu_matrix_exactness.py."""
    import torch
    from paper_2105_00619_amd import binding as B
    mats, steps, want = LISTS[i]
    plan = B.Orthogonalizer(mats, steps=steps)
    assert {k: _plan_shape(plan, k) for k in want} == want, [_plan_shape(plan, k) for k in range(5)]
    gen = torch.Generator(device="cuda").manual_seed(i)
    g = torch.randn(plan.span, generator=gen, device="cuda")
    o32, o16 = plan.orthogonalize(g), torch.empty(plan.span, dtype=torch.bfloat16, device="cuda")
    plan.orthogonalize(g, o16)
    w, v, w16 = torch.zeros_like(g), torch.zeros_like(g), torch.empty_like(o16)
    plan.muon_update(w, v, g, lr=1.0, momentum=0.0, scale="none", weights16=w16)
    assert torch.equal(w16, w.bfloat16())
    at = 0
    for r, c in mats:
        of = lambda t: t[at:at + r * c].view(r, c)  # noqa: E731
        ref = _steps(of(g), torch.float64, steps)
        plain = _far(_steps(of(g), torch.float32, steps), ref)
        assert _far(of(o32), ref) <= 2 * plain + 2.0 ** -17, (r, c, plain)
        assert _far(-of(w), ref) <= 2 * plain + 2.0 ** -17 + 2.0 ** -23, (r, c, plain)
        assert _far(of(o16), ref) <= 2 * plain + 2.0 ** -13 + 1.05 * _far(ref.bfloat16(), ref), (r, c, plain)
        at += r * c
