"""The matrix operators together, as examples/orthogonalised_training.py uses them, and gradients into a caller's tensors."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("orthogonalised_training", os.path.join(ROOT, "examples", "orthogonalised_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_feed_forward_learns_its_batch(example):
    """A network of more weights than samples fits one batch of random labels: well below the log(10) of guessing."""
    losses = example.train_feed_forward(steps=60, batch=64, width=96, hidden=200, blocks=2)
    assert losses[-1] < 0.5 * losses[0]
    assert losses == example.train_feed_forward(steps=60, batch=64, width=96, hidden=200, blocks=2)  # bit for bit


def test_cnn_learns_its_batch(example):
    losses = example.train_cnn(steps=30, batch=32)
    assert losses[-1] < 0.5 * losses[0]


def test_feed_forward_gradients_are_the_plain_networks(example):
    """In fp32 against autograd in float64.  Every product is off by at most K 2^-23 of its absolute sum, K <= 200, over six layers with
    gains of order one: 1e-4 of the largest gradient of a matrix."""
    import torch
    net = example.FeedForward(75, 33, 50, 2, 10, dtype=torch.float32, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(70, 75, generator=gen, device="cuda")
    d = torch.randn(70, 10, generator=gen, device="cuda")
    logits, kept = net.forward(x)
    net.backward(d, kept)
    ws = [w.double().cpu().requires_grad_() for w in net.weights]
    bs = [b.double().cpu().requires_grad_() for b in net.biases]
    act = lambda t: 0.5 * t * torch.special.erfc(-t / 2 ** 0.5)  # noqa: E731
    h = act(x.double().cpu() @ ws[0].T + bs[0])
    for i in (1, 3):
        h = h + (act(h @ ws[i].T + bs[i]) @ ws[i + 1].T + bs[i + 1])
    y = h @ ws[5].T + bs[5]
    assert float((logits.double().cpu() - y).abs().max()) < 1e-4 * float(y.abs().max())
    (y * d.double().cpu()).sum().backward()
    for got, ref in list(zip(net.dweights, ws)) + list(zip(net.dbiases, bs)):
        assert float((got.double().cpu() - ref.grad).abs().max()) < 1e-4 * float(ref.grad.abs().max())


def test_gradients_into_given_tensors():
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(1)
    dy, x, w = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((70, 33), (70, 20), (33, 20)))
    ref = B.linear_backward(dy, x, w)
    dx, db = torch.empty(70, 24, dtype=torch.bfloat16, device="cuda")[:, :20], torch.empty(33, device="cuda")
    flat = torch.full((33 * 20 + 7,), 5.0, dtype=torch.bfloat16, device="cuda")
    got = B.linear_backward(dy, x, w, dx=dx, dw=flat[3:3 + 33 * 20].view(33, 20), dbias=db)
    assert all(torch.equal(a, b) for a, b in zip(got, ref)) and got[0] is dx and got[2] is db
    assert bool((flat[:3] == 5).all()) and bool((flat[-4:] == 5).all())
    with pytest.raises(ValueError, match="not in need"):
        B.linear_backward(dy, x, w, need=("dx",), dw=ref[1])
    with pytest.raises(ValueError, match="dw"):
        B.linear_backward(dy, x, w, dw=ref[0])
    with pytest.raises(TypeError, match="dbias"):
        B.linear_backward(dy, x, w, dbias=db.bfloat16())


def test_small_matrices_in_one_launch_are_those_in_many():
    """A list of small matrices takes its m x m products in one launch, the same matrices beside a larger one in many: both are within
    a^steps 2^-22 of the exact result (an error of the first iterate grows by at most a = 3.4445 a step), so within twice that of each other."""
    import torch
    from paper_2105_00619_amd import binding as B
    shapes = [(8, 27), (33, 40), (64, 64), (65, 300), (128, 129), (300, 97), (1, 5)]
    gen = torch.Generator(device="cuda").manual_seed(2)
    n = sum(r * c for r, c in shapes)
    g = torch.randn(n + 130 * 140, generator=gen, device="cuda")
    for steps in (1, 2, 3, 5, 7):
        small = B.Orthogonalizer(shapes, steps=steps).orthogonalize(g[:n].clone())
        large = B.Orthogonalizer(shapes + [(130, 140)], steps=steps).orthogonalize(g)
        at = 0
        for r, c in shapes:
            a, b = small[at:at + r * c], large[at:at + r * c]
            assert float((a - b).norm()) <= 2 * 3.4445 ** steps * 2.0 ** -22 * float(b.norm()), (steps, r, c)
            at += r * c


@pytest.mark.parametrize("small", [1.0, 1e-1, 1e-2, 3e-3, 1e-3])
def test_bf16_results_where_one_direction_outweighs_the_others(small):
    """All steps of a bf16 result are made on X X^T: a rounding there (2^-24) reaches a direction of relative size s times 1 / s^2, grows with
    it until its size is of order one, and shows by the slope of the polynomial: up to about 2^-10, beside the rounding to bf16, at most
    2^-8 of a value."""
    import torch
    from paper_2105_00619_amd import binding as B
    gen = torch.Generator().manual_seed(4)
    u = torch.linalg.qr(torch.randn(192, 192, generator=gen, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(700, 192, generator=gen, dtype=torch.float64))[0]
    s = torch.full((192,), small, dtype=torch.float64)
    s[0] = 1.0
    g = torch.mm(u * s, v.T.contiguous()).float()
    x = g.double() / g.double().norm()
    for _ in range(5):
        a = torch.mm(x, x.T.contiguous())
        x = 3.4445 * x + torch.mm(-4.7750 * a + 2.0315 * torch.mm(a, a), x)
    out = torch.empty(192 * 700, dtype=torch.bfloat16, device="cuda")
    B.Orthogonalizer([(192, 700)]).orthogonalize(g.reshape(-1).cuda(), out)
    assert float((out.double().cpu().view(192, 700) - x).norm()) <= (2.0 ** -8 + 2.0 ** -10) * float(x.norm())


@pytest.mark.parametrize("name", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cin,cout", [(512, 8, 1), (513, 9, 3), (700, 263, 16), (1111, 517, 17), (530, 4099, 33), (600, 7, 64), (520, 1031, 64),
                                           (3, 8, 5), (5, 11, 7), (40, 4505, 70), (17, 519, 33), (64, 1001, 15)])
def test_forward_straight_from_memory(rows, cin, cout, name):
    """Few samples or few outputs, rows at any address.  Products are exact (16 bits) or off by 2^-24 (fp32 as planes); at most a fourth
    of them (six plane pairs in fp32) is added one after the other, cut off at 2^-23 of the absolute sum; one rounding at the end."""
    import torch
    from paper_2105_00619_amd import binding as B
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]
    gen = torch.Generator(device="cuda").manual_seed(rows + cin)
    make = lambda r, c: torch.randn(r, c + 3, generator=gen, device="cuda").to(dt)[:, 1:1 + c]  # noqa: E731
    x, w, res = make(rows, cin), make(cout, cin), make(rows, cout)
    bias = torch.randn(cout, generator=gen, device="cuda")
    y, z = B.linear_forward(x, w, bias, residual=res, activation="relu", save_pre=True)
    zr = torch.mm(x.double(), w.double().T.contiguous()) + bias.double()
    sums = torch.mm(x.double().abs(), w.double().abs().T.contiguous()) + bias.double().abs()
    off = (cin / 4 * (6 if name == "fp32" else 1) + 48) * 2.0 ** -23 * sums
    e = 1.01 * torch.finfo(dt).eps / 2
    assert bool(((z.double() - zr).abs() <= e * zr.abs() + off).all())
    yr = zr.clamp_min(0) + res.double()
    assert bool(((y.double() - yr).abs() <= e * yr.abs() + off + 2.0 ** -23 * (zr.abs() + yr.abs())).all())
    # an infinity and a NaN reach their sample or output only, at the row's end too
    for at in (0, cin - 1):
        x2, w2 = x.clone(), w.clone()
        x2[rows - 1, at], w2[cout - 1, at] = float("inf"), float("nan")
        y2 = B.linear_forward(x2, w2, bias)
        ref = torch.mm(x2.double(), w2.double().T.contiguous()) + bias.double()
        assert torch.equal(torch.isnan(y2), torch.isnan(ref)) and torch.equal(torch.isinf(y2), torch.isinf(ref))
