"""Layer norm at sizes whose kernels differ from the small ones': matrices beyond the last-level cache, rows of 8193 to 16384 columns of which a
block takes several, rows that begin beyond 2^31 elements.  Tolerances are those of test_gpu_norm.py."""
import pytest

from tests.test_gpu_norm import U, _column_adds, _dt, _randn, _row_adds, _t, _within

pytestmark = pytest.mark.gpu


def _rand_matrix(rows, cols, dt, ld, shift, seed, scale):
    """Random values made on the GPU, rows `ld` elements apart, `shift` elements off an aligned address; and all of the buffer."""
    torch = _t()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((shift + (rows - 1) * ld + cols + 8,), 7.5, dtype=dt, device="cuda")
    m = buf.as_strided((rows, cols), (ld, 1), shift)
    for a in range(0, rows, 65536):
        part = m[a:a + 65536]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
    return m, buf


def _check(rows, cols, name, ld, shift, residual, forward=True):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    dt = _dt(name)
    x, _ = _rand_matrix(rows, cols, dt, ld, shift, 1, 1.5)
    w, b = _randn(cols, seed=2, shift=1.0).float().cuda(), _randn(cols, seed=3).float().cuda()
    out, buf = _rand_matrix(rows, cols, dt, ld, shift, 4, 1.0)
    n, e = _row_adds(cols), torch.finfo(dt).eps / 2
    y, mean, rstd = B.layer_norm_forward(x, w, b, save_stats=True, out=out)
    if forward:
        for a in range(0, rows, 16384):
            v = x[a:a + 16384].double()
            m = v.mean(1, keepdim=True)
            d = v - m
            r = (d.square().mean(1, keepdim=True) + 1e-5) ** -0.5
            size, h = d.abs().mean(1, keepdim=True), d * r
            _within(mean[a:a + 16384], m[:, 0], U * m[:, 0].abs() + (n + 4) * U * size[:, 0], "mean")
            _within(rstd[a:a + 16384], r[:, 0], (n / 2 + 5) * U * r[:, 0], "rstd")
            ref = h * w.double() + b.double()
            fp32 = U * (w.double().abs() * ((n / 2 + 10) * h.abs() + (n + 4) * size * r) + 2 * (ref.abs() + b.double().abs()))
            _within(y[a:a + 16384], ref, e * (ref.abs() + fp32) + fp32, "y")
    dy, _ = _rand_matrix(rows, cols, dt, ld, shift, 5, 0.1)
    res = _rand_matrix(rows, cols, dt, ld, shift, 6, 0.1)[0] if residual else None
    before = buf.as_strided((rows - 1, ld - cols), (ld, 1), shift + cols).clone() if ld > cols and ld < 1 << 20 else None
    dx, dw, db = B.layer_norm_backward(dy, x, mean, rstd, w, residual=res, dx=out)
    if before is not None:
        assert torch.equal(buf.as_strided((rows - 1, ld - cols), (ld, 1), shift + cols), before), "values outside the result were written"
    sums = [torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(4)]
    for a in range(0, rows, 16384):
        k = slice(a, min(a + 16384, rows))
        r = rstd[k].double()[:, None]
        h = (x[k].double() - mean[k].double()[:, None]) * r
        g = dy[k].double()
        u = g * w.double()
        ref = r * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
        fp32 = U * r * (4 * u.abs() + (n + 6) * u.abs().mean(1, keepdim=True) + h.abs() * ((n + 10) * (u * h).abs().mean(1, keepdim=True)))
        full = ref + res[k].double() if residual else ref
        fp32 = fp32 + U * (ref.abs() + full.abs())
        _within(dx[k], full, e * (full.abs() + fp32) + fp32, "dx")
        for s, v in zip(sums, ((g * h), (g * h).abs(), g, g.abs())):
            s += v.sum(0)
    nr = _column_adds(rows, cols)
    _within(dw, sums[0], (nr + 4) * U * sums[1], "dweight")
    _within(db, sums[2], nr * U * sums[3], "dbias")
    if residual:
        B.layer_norm_backward(dy, x, mean, rstd, w, residual=res, dx=res, need=("dx",))
        assert torch.equal(res, dx), "dx in the residual's place"


# more than 384 MB in all: read past the caches.  One thread of a row to sixteen wavefronts of it, whole rows and odd ones, off their alignment
@pytest.mark.parametrize("name", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,pad,shift,residual", [(1100011, 50, 0, 0, True), (530003, 100, 3, 1, True), (98317, 517, 0, 0, True), (25003, 2027, 3, 1, True),
                                                          (17003, 4096, 0, 0, False), (7001, 7400, 8, 8, True), (3301, 15500, 0, 0, True), (5003, 16384, 3, 1, False)])
def test_matrices_beyond_the_caches(rows, cols, pad, shift, residual, name):
    assert rows * cols * 2 * (4 if residual else 3) > 384 << 20
    _check(rows, cols, name, cols + pad, shift, residual, forward=False)


@pytest.mark.parametrize("name", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1100, 8193, 3, 1), (1030, 8200, 0, 0), (1300, 12345, 0, 0), (1100, 16384, 8, 8)])
def test_blocks_that_walk_rows_of_two_pieces(rows, cols, pad, shift, name):
    _check(rows, cols, name, cols + pad, shift, True)


@pytest.mark.parametrize("cols", [520, 9000])
def test_rows_that_begin_beyond_32_bits(cols):
    ld = (1 << 22) - 8
    assert 519 * ld > 1 << 31
    _check(520, cols, "bf16", ld, 0, True)
