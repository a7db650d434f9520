"""Training operators over so many rows that every thread walks over several of them, the last turn ragged: the
next row's loads, stepped addresses, alternating buffers and sums over a thread's own rows, against 64 bits.

A layer norm kernel has at most 148 blocks of 768 threads; the sizes below take each number of chunks a thread, in
each direction and alignment, through at least three turns on a GPU of that size.

Tolerances, in units of 2^-24 of the magnitudes that enter: an output of a row as in test_gpu_training_ops (64 for
row sums, 128 and 192 for what is formed from them).  A column sum adds a thread's at most 10 rows, the block's at
most 96 teams, then 148 / 16 (GELU: 626 / 16) parts and 16 warps' sums: at most 162 additions of half a unit each,
81, and 8 more for the roundings of an addend: 96.
"""
import math

import pytest
import torch

from tests import training_reference as ref
from tests.test_gpu_training_ops import TYPES, empty_like_placed, fa, gen, outside_untouched, placed, randn

pytestmark = pytest.mark.gpu

PLACES = [(0, 0), (8, 8), (3, 5)]              # dense; aligned rows with gaps; rows that 16-byte loads cannot address
LN_SIZES = [(44011, 64), (9001, 328), (5003, 768), (4001, 1536), (3601, 2048), (1403, 4096), (601, 6144), (451, 16384),
            (1203, 9000)]


def inputs(rows, cols, T, seed):
    """Rows of different offsets; every 64th one zero, another constant."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda") * 2 + torch.randn(rows, 1, generator=g, device="cuda")
    x[63::64] = 0.0
    x[17::64] = 3.0
    return x.to(T), lambda *shape, scale=1.0: (torch.randn(*shape, generator=g, device="cuda") * scale).to(T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", LN_SIZES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("lead,gap", PLACES)
def test_layer_norm_forward_over_several_rows_a_thread(dtype, rows, cols, residual, lead, gap):
    T, eps = TYPES[dtype], 1e-5
    x, normal = inputs(rows, cols, T, rows + cols)
    r = placed(normal(rows, cols), lead, gap)[0] if residual else None
    w, b = normal(cols), normal(cols)
    y, ybuf = empty_like_placed(x, lead, gap)
    s_out, sbuf = empty_like_placed(x, lead, gap)
    ck_sum, ck_y = fa().new_checkpoint8(rows, cols, "cuda"), fa().new_checkpoint8(rows, cols, "cuda")
    _, mean, rstd, _ = fa().fa_layer_norm_forward(placed(x, lead, gap)[0], w, b, eps, residual=r, y=y, sum_out=s_out,
                                                  ck_sum=ck_sum, ck_y=ck_y)
    s = x.double() + (r.double() if residual else 0.0)
    ey, emean, erstd = ref.layer_norm(s, w.double(), b.double(), eps)
    big = s.abs().amax(1)
    ref.assert_close(mean, emean, big, 64, "mean")
    ref.assert_close(rstd, erstd, erstd * (1 + (big * erstd) ** 2 * 2.0 ** -12), 128, "rstd")
    h = (s - emean[:, None]).abs() * erstd[:, None]
    scale = (h * (1 + (big * erstd)[:, None] ** 2 * 2.0 ** -12) + (big * erstd)[:, None]) * w.double().abs() + b.double().abs()
    ref.assert_close(y, ey, scale, 192, "y")
    ref.assert_close(s_out, s, s.abs(), 1, "sum")
    assert outside_untouched(y, ybuf) and outside_untouched(s_out, sbuf)
    for ck, t in ((ck_sum, s_out), (ck_y, y)):
        for a, c in zip(ref.buffer_parts(ck, rows, cols), ref.buffer_parts(fa().fa_checkpoint8_store(t), rows, cols)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", LN_SIZES)
@pytest.mark.parametrize("source", ["x", "ck"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("lead,gap", PLACES)
def test_layer_norm_backward_over_several_rows_a_thread(dtype, rows, cols, source, residual, lead, gap):
    T = TYPES[dtype]
    x, normal = inputs(rows, cols, T, rows * 7 + cols)
    w, dy = normal(cols), normal(rows, cols, scale=0.1)
    r = placed(normal(rows, cols, scale=0.1), lead, gap)[0] if residual else None
    _, mean, rstd = ref.layer_norm(x.double(), None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    ck = fa().fa_checkpoint8_store(x) if source == "ck" else None
    x64 = x.double() if ck is None else ref.decode(ck, rows, cols).cuda()
    dx, dxbuf = empty_like_placed(x, lead, gap)
    row = torch.full((2 * cols + 16,), math.nan, device="cuda")
    fa().fa_layer_norm_backward(placed(dy, lead, gap)[0], w, mean, rstd, x=placed(x, lead, gap)[0] if ck is None else None,
                                ck=ck, residual_grad=r, dx=dx, dweight=row[3:3 + cols], dbias=row[3 + cols:3 + 2 * cols])
    edx, edw, edb = ref.layer_norm_grad(dy.double(), x64, mean.double(), rstd.double(), w.double(),
                                        r.double() if residual else None)
    rs = rstd.double()[:, None]
    spread = (x64.abs() + mean.double().abs()[:, None]) * rs
    gmag = dy.double().abs() * w.double().abs()
    hmag = spread.amax(1, keepdim=True)
    scale = rs * (gmag + gmag.mean(1, keepdim=True) + hmag * (gmag * spread).mean(1, keepdim=True)) + (r.double().abs() if residual else 0)
    ref.assert_close(dx, edx, scale, 128, "dx")
    ref.assert_close(row[3:3 + cols], edw, (dy.double().abs() * spread).sum(0), 96, "dweight")
    ref.assert_close(row[3 + cols:3 + 2 * cols], edb, dy.double().abs().sum(0), 96, "dbias")
    assert outside_untouched(dx, dxbuf) and torch.isnan(row[:3]).all() and torch.isnan(row[3 + 2 * cols:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", ["tanh", "erf"])
@pytest.mark.parametrize("rows,cols", [(40009, 40), (20011, 160), (5003, 1032), (1501, 8200)])
@pytest.mark.parametrize("source", ["x", "ck"])
@pytest.mark.parametrize("lead,gap", PLACES)
def test_gelu_backward_over_several_rows_a_thread(dtype, form, rows, cols, source, lead, gap):
    T = TYPES[dtype]
    x, normal = inputs(rows, cols, T, rows * 3 + cols)
    b = normal(cols) if source == "x" else None
    dy = normal(rows, cols)
    ck = fa().fa_checkpoint8_store(x) if source == "ck" else None
    z = ref.decode(ck, rows, cols).cuda() if ck is not None else x.double() + b.double()
    dx, dxbuf = empty_like_placed(x, lead, gap)
    row = torch.full((cols + 8,), math.nan, device="cuda")
    fa().fa_gelu_backward(placed(dy, lead, gap)[0], x=placed(x, lead, gap)[0] if ck is None else None, bias=b, ck=ck,
                          approximate=form, dx=dx, dbias=row[1:1 + cols])
    e = dy.double() * ref.gelu_slope(z, form)
    scale = dy.double().abs() * (1 + z.abs())
    ref.assert_close(dx, e, scale, 64, "dx")
    ref.assert_close(row[1:1 + cols], e.sum(0), scale.sum(0), 96 + 64, "dbias")
    assert outside_untouched(dx, dxbuf) and torch.isnan(row[:1]).all() and torch.isnan(row[1 + cols:]).all()
