"""Layer norm's row statistics where they can be stated exactly."""
import math

import pytest
import torch

from tests.test_gpu_training_ops import fa

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
