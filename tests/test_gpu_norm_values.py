"""Statistics of a layer norm's rows that hold a value that is not finite."""
import pytest

from tests.test_gpu_norm import DTYPES, _dt, _randn, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", DTYPES)
@pytest.mark.parametrize("cols", [5, 300, 4097, 9000, 20000])
@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_rstd_says_that_a_row_is_not_finite(eps, cols, name):
    from paper_2105_00619_amd import binding as B
    torch = _t()
    x = _randn(6, cols, seed=cols).to(_dt(name)).cuda()
    x[1, 3], x[2, cols - 1], x[4, 0] = float("inf"), float("nan"), -float("inf")
    y, mean, rstd = B.layer_norm_forward(x, eps=eps, save_stats=True)
    bad = [1, 2, 4]
    assert bool(torch.isnan(rstd[bad]).all()) and not bool(torch.isfinite(mean[bad]).any()) and bool(torch.isnan(y[bad]).all())
    assert bool(torch.isfinite(rstd[[0, 3, 5]]).all()) and bool(torch.isfinite(y[[0, 3, 5]]).all())
    # Equal values: the mean is off by at most 40 additions' rounding, 40 u 2.5 = 6e-6, and what the correction leaves of the variance by a few u of that
    # squared, 1e-17 (u = 2^-24).
    same = B.layer_norm_forward(torch.full((2, cols), 2.5, dtype=x.dtype, device="cuda"), eps=eps, save_stats=True)[2]
    assert bool((same >= 1e8).all()) if eps == 0 else bool(((same.double() * eps ** 0.5 - 1).abs() <= 8 * 2.0 ** -24).all())
