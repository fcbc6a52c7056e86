"""The losses' forward kernels for few rows, each by its own rule (test_loss_paths.py pins which sizes take which), and rows that begin beyond 2^31
elements.  Tolerances are those of test_gpu_loss.py."""
import pytest

from tests.test_gpu_loss import DTYPES, U, Reference, _dt, _entropy_target, _randn, _t, _teacher_entries, _teacher_target, _within

pytestmark = pytest.mark.gpu


def _check(x, w, bias, name, top, smoothing, z_loss, seed):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    rows, classes = x.shape[0], w.shape[0]
    labels = torch.randint(0, classes, (rows,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()
    labels[0] = classes - 1
    if rows > 2:
        labels[1] = -1
    target, used = _entropy_target(labels, classes, smoothing)
    ref = Reference(name, x, w, bias, target, used, z_loss=z_loss)
    loss, lse = B.cross_entropy_forward(x, w, labels, bias, label_smoothing=smoothing, z_loss=z_loss)
    _within(lse, ref.lse, ref.lse_tol, "lse")
    _within(loss, ref.loss, ref.loss_tol, "loss")
    assert not bool(loss[~used].any())
    idx, t = _teacher_entries(rows, classes, top, seed + 1, torch.float32)
    idx[0, 0], t[0, 0] = classes - 1, 2.0
    target, used, entropy = _teacher_target(idx, t, classes, 2.0)
    ref = Reference(name, x, w, bias, target, used, tau=2.0, entropy=entropy)
    loss, lse = B.distillation_forward(x, w, idx, t, bias, temperature=2.0)
    _within(lse, ref.lse, ref.lse_tol, "lse of a teacher's")
    more = 20 * U * (target * (ref.s - ref.lse[:, None]).abs()).sum(1)
    _within(loss, ref.loss, ref.loss_tol + more, "loss against a teacher")
    assert not bool(loss[~used].any())


# (rows, in, classes): four wavefronts and eight; whole widths and the least of them; classes in one group, in as many as there are blocks and in several turns
@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,cin,classes", [(1, 4096, 5), (16, 4096, 900), (13, 3696, 9001), (1, 3688, 20011), (16, 4096, 33000), (9, 4088, 12289), (1, 2048, 16), (16, 1848, 24601), (2, 2048, 65537)])
def test_streamed_weights(rows, cin, classes, name):
    dt = _dt(name)
    x, w = _randn(rows, cin, seed=rows).to(dt), _randn(classes, cin, seed=classes, scale=2 * cin ** -0.5).to(dt)
    bias = _randn(classes, seed=3).float()
    _check(x, w, bias, name, 5, 0.1, 1e-2, 11)
    _check(x, w, None, name, 40, 0.0, 0.0, 12)


# off the alignment of 16 bytes, and fp32: 16, 32 and 64 rows, four to sixteen wavefronts
@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("rows,cin,classes", [(16, 4095, 900), (32, 2047, 5003), (33, 517, 40001), (64, 4097, 3001), (1, 7, 130), (48, 1025, 17000)])
def test_weights_as_they_lie(rows, cin, classes, name):
    dt = _dt(name)
    x, w = _randn(rows, cin, seed=rows).to(dt), _randn(classes, cin, seed=classes, scale=2 * cin ** -0.5).to(dt)
    _check(x, w, _randn(classes, seed=3).float(), name, 17, 0.1, 1e-2, 13)


@pytest.mark.parametrize("rows", [16, 530])
def test_rows_that_begin_beyond_32_bits(rows):
    """x, w, dx and dw with rows 2^22 - 8 elements apart: the same bits as where they lie together."""
    from paper_2105_00619_amd import binding as B
    torch = _t()
    ld, cin, classes = (1 << 22) - 8, 2048, 530
    apart = lambda n: torch.full(((n - 1) * ld + cin,), 7.5, dtype=torch.bfloat16, device="cuda").as_strided((n, cin), (ld, 1))  # noqa: E731
    x, w, dx, dw = apart(rows), apart(classes), apart(rows), apart(classes)
    assert (classes - 1) * ld > 1 << 31
    x.copy_(_randn(rows, cin, seed=1))
    w.copy_(_randn(classes, cin, seed=2, scale=2 * cin ** -0.5))
    labels = (torch.arange(rows, device="cuda") % classes).int()
    d = torch.rand(rows, device="cuda")
    near = [t.contiguous() for t in (x, w)]
    a, b = B.cross_entropy_forward(x, w, labels), B.cross_entropy_forward(*near, labels)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    B.cross_entropy_backward(d, x, w, labels, a[1], dx=dx, dw=dw, need=("dx", "dw"))
    want = B.cross_entropy_backward(d, *near, labels, a[1], need=("dx", "dw"))
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    assert float(torch.as_strided(dw, (classes - 1,), (ld,), cin).double().sub(7.5).abs().max()) == 0
