"""Layer norm's row statistics where they can be stated exactly."""
import math

import pytest
import torch

from tests.test_gpu_training_ops import TYPES, fa

pytestmark = pytest.mark.gpu

LONG = 20000                                   # columns of a row that does not fit registers


@pytest.mark.parametrize("cols", [2, LONG])
def test_rstd_is_the_rounded_reciprocal_of_the_deviation(cols):
    """Rows of v, -v and zeros: mean 0 and sum of squares 2 v^2, both exact for v of 11 bits.  With two columns and eps 0
    the variance is v^2, its root v, and rstd 1 / v rounded once."""
    v = torch.arange(1, 2049, device="cuda", dtype=torch.float32)
    x = torch.zeros(v.numel(), cols, device="cuda")
    x[:, 0], x[:, 1] = v, -v
    _, mean, rstd, _ = fa().fa_layer_norm_forward(x, eps=0.0)
    assert not mean.any()
    if cols == 2:
        assert torch.equal(rstd, (1.0 / v.double()).float())
    else:                                      # 2 v^2 / 20000 and the root are rounded: half a unit and a quarter, the reciprocal half
        assert ((rstd.double() * v.double() * math.sqrt(2.0 / cols)) - 1.0).abs().max() <= 1.25 * 2.0 ** -23


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 96, 768, 5000, 16384, LONG])
def test_means_of_rows_that_are_not_finite(dtype, cols):
    x = torch.ones(7, cols, device="cuda", dtype=TYPES[dtype])
    at = cols // 2
    x[1, at], x[2, at], x[3, at] = math.inf, -math.inf, math.nan
    x[4, 0], x[4, cols - 1] = math.inf, -math.inf
    x[5] = torch.finfo(x.dtype).max            # the sum runs over, its quotient with it
    y, mean, rstd, _ = fa().fa_layer_norm_forward(x)
    assert mean[0] == 1 and mean[6] == 1 and mean[1] == math.inf and mean[2] == -math.inf and torch.isnan(mean[3])
    assert torch.isnan(mean[4]) if cols > 1 else mean[4] == -math.inf
    if cols > 1:
        assert mean[5] == math.inf
    assert torch.isnan(rstd[1:4]).all() and torch.isnan(y[1:4]).all() and torch.isfinite(y[[0, 6]]).all()


@pytest.mark.parametrize("cols", [96, LONG])
def test_a_variance_that_runs_over_gives_a_zero_rstd(cols):
    """sqrt and reciprocal of Inf: rstd is 0, and y the bias."""
    x = torch.full((3, cols), 1e30, device="cuda")
    x[:, ::2] = -1e30
    bias = torch.linspace(-1, 1, cols, device="cuda")
    y, mean, rstd, _ = fa().fa_layer_norm_forward(x, bias=bias)
    assert not mean.any() and not rstd.any() and torch.equal(y, bias.expand(3, cols))


@pytest.mark.parametrize("cols", [96, LONG])
def test_gradient_rows_that_hold_an_infinity(cols):
    """mean(g) is Inf: dx is -Inf next to the infinite entry (which is Inf - Inf), in rows of any length."""
    dy = torch.ones(2, cols, device="cuda")
    dy[1, 5] = math.inf
    zero, one = torch.zeros(2, device="cuda"), torch.ones(2, device="cuda")
    x = torch.ones(2, cols, device="cuda")
    x[:, 1::2] = -1.0
    dx, _, db = fa().fa_layer_norm_backward(dy, None, zero, one, x=x)
    # h = x: mean(g h) is -Inf, so g - Inf + h Inf is NaN where h > 0 and -Inf where h < 0
    assert torch.isfinite(dx[0]).all() and torch.isnan(dx[1, 0::2]).all()
    others = torch.arange(1, cols, 2, device="cuda")
    others = others[others != 5]
    assert (dx[1, others] == -math.inf).all() and torch.isnan(dx[1, 5])
    assert db[5] == math.inf and torch.isfinite(db[6:]).all()
