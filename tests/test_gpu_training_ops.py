"""Training operators on the GPU against plain 64-bit statements of them (tests/training_reference.py).

Tolerances: an output is off by its rounding and by the fp32 arithmetic in front of it.  The latter is
bounded by `ulps` units of 2^-24 of the magnitudes that enter (`scale`): one unit per operation on the
longest chain of additions a value goes through.  For sums over a row of c columns the chain is at
most 8 K + 5 + 16 additions for register rows (K <= 4 chunks of 8 per thread, a shuffle tree, 16 warps),
8 * ceil(c / 4096) + 21 for longer ones; a sum over r rows adds a thread's rows first (at most r / 8 + 1
here), then 64 threads and 8 slices.  64 units per row sum and r / 8 + 128 per column sum cover all cases.
"""
import math

import pytest
import torch

from tests import training_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [(1, 1), (3, 7), (5, 32), (2, 33), (1, 768), (64, 40), (130, 768), (37, 1001), (9, 1024), (300, 1030),
         (17, 4096), (8, 16384), (5, 16392), (3, 20001)]


def fa():
    import paper_2302_05865_b200
    return paper_2302_05865_b200


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def placed(t, lead=0, gap=0):
    """t as rows of stride cols + gap, `lead` elements into a buffer that is NaN elsewhere."""
    rows, cols = t.shape
    buf = torch.full((lead + rows * (cols + gap) + 64,), math.nan, dtype=t.dtype, device=t.device)
    view = buf[lead:lead + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    view.copy_(t)
    return view, buf


def empty_like_placed(t, lead, gap):
    view, buf = placed(torch.zeros_like(t), lead, gap)
    view.fill_(math.nan)
    return view, buf


def outside_untouched(view, buf):
    """Whether everything of buf outside the view is still NaN."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool(torch.isnan(buf[mask]).all())


# ------------------------------------------------------------------------------- checkpoints

def special_rows(dtype):
    """Groups at the format's edges, one per row."""
    f = torch.finfo(dtype)
    rows = [[0.0] * 32, [127.0] + [0.5, 1.5, 2.5, -0.5, -1.5] * 6 + [0.0], [f.max, -f.max, f.tiny] + [1.0] * 29,
            [f.smallest_normal] * 32, [f.smallest_normal / 4, -f.smallest_normal / 2] * 16, [math.inf] + [1.0] * 31,
            [1.0] * 31 + [-math.inf], [1.0, math.nan] + [2.0] * 30, [2.0 ** -126 * 127] + [2.0 ** -127] * 31,
            [1.984375] + [0.0078125 * k for k in range(31)], [128.0, 127.0, 126.0, -127.0] * 8]
    edge = torch.tensor([127.0, 127.0 * 2.0 ** 20, 127.0 * 2.0 ** -40], dtype=dtype)
    above = torch.nextafter(edge, torch.full_like(edge, math.inf)) if dtype == torch.float32 else edge + edge / 128
    for v in torch.cat([edge, above]).tolist():
        rows.append([v, -v / 3, v / 254, v / 127 * 2.5] * 8)
    return torch.tensor(rows, dtype=torch.float64).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (4, 32), (3, 33), (7, 100), (5, 160), (2, 1001), (33, 768)])
@pytest.mark.parametrize("lead,gap", [(0, 0), (1, 0), (8, 8), (0, 3)])
def test_checkpoint_codes_scales_and_values(dtype, rows, cols, lead, gap):
    T = TYPES[dtype]
    g = gen(rows * 1000 + cols)
    x = (torch.randn(rows, cols, generator=g) * torch.exp(4 * torch.randn(rows, cols, generator=g))).to(T).cuda()
    xv, _ = placed(x, lead, gap)
    nbytes = fa().fa_checkpoint8_bytes(rows, cols)
    guard = torch.full((nbytes + 512,), 77, dtype=torch.uint8, device="cuda")
    ck = guard[256:256 + nbytes]
    fa().fa_checkpoint8_store(xv, ck=ck)
    codes, scales = ref.encode(x)
    got_codes, got_scales, padding = ref.buffer_parts(ck, rows, cols)
    assert torch.equal(got_codes, codes) and torch.equal(got_scales, scales) and not padding.any()
    assert (guard[:256] == 77).all() and (guard[256 + nbytes:] == 77).all()
    values = ref.decode(ck, rows, cols)
    for out_type in TYPES.values():
        out, buf = empty_like_placed(torch.zeros(rows, cols, dtype=out_type, device="cuda"), lead, gap)
        fa().fa_checkpoint8_load(ck, rows, cols, out=out)
        assert torch.equal(out.double().cpu(), values)          # exact in both types
        assert outside_untouched(out, buf)
    step = torch.exp2(scales.double() - 127.0).repeat_interleave(32, 1)[:, :cols]
    assert ((values - x.double().cpu()).abs() <= 0.5 * step).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_checkpoint_of_edge_values(dtype):
    x = special_rows(TYPES[dtype])
    ck = fa().fa_checkpoint8_store(x.cuda())
    codes, scales = ref.encode(x)
    got_codes, got_scales, _ = ref.buffer_parts(ck, *x.shape)
    assert torch.equal(got_scales, scales) and torch.equal(got_codes, codes)
    back = fa().fa_checkpoint8_load(ck, *x.shape, dtype=torch.float32).cpu().double()
    torch.testing.assert_close(back, ref.decode(ck, *x.shape), rtol=0, atol=0, equal_nan=True)
    broken = ~torch.isfinite(x).all(1)
    assert torch.isnan(back[broken]).all() and torch.isfinite(back[~broken]).all()


def test_row_strides_beyond_32_bits():
    """Rows 1.2e9 elements apart: offsets pass 2^31 elements and 2^32 bytes."""
    cols, ld = 96, 1_200_000_000
    buf = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, cols), (ld, 1))
    src = randn(gen(3), 3, cols, dtype=torch.bfloat16)
    x.copy_(src)
    assert torch.equal(fa().fa_checkpoint8_store(x)[:3 * cols], fa().fa_checkpoint8_store(src)[:3 * cols])
    y, mean, rstd, _ = fa().fa_layer_norm_forward(x)
    y2, mean2, rstd2, _ = fa().fa_layer_norm_forward(src)
    assert torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    dy = randn(gen(4), 3, cols, dtype=torch.bfloat16)
    for got, want in zip(fa().fa_layer_norm_backward(dy, None, mean, rstd, x=x),
                         fa().fa_layer_norm_backward(dy, None, mean, rstd, x=src)):
        assert torch.equal(got, want)
    for got, want in zip(fa().fa_gelu_backward(dy, x=x), fa().fa_gelu_backward(dy, x=src)):
        assert torch.equal(got, want)
    ck = fa().fa_checkpoint8_store(src)
    for got, want in zip(fa().fa_linear_weight_grad(x, ck, cols), fa().fa_linear_weight_grad(src, ck, cols)):
        assert torch.equal(got, want)


def test_checkpoint_of_more_than_2_to_the_31_values():
    rows, cols = 69_000, 32_000                                  # 2.2e9 values, 4.4 GB
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = randn(gen(9), 5, cols, dtype=torch.bfloat16)
    x[-5:] = tail
    ck = fa().fa_checkpoint8_store(x)
    out = fa().fa_checkpoint8_load(ck, rows, cols, out=x)
    small = fa().fa_checkpoint8_load(fa().fa_checkpoint8_store(tail), 5, cols)
    assert torch.equal(out[-5:], small) and not out[:-5].any()


# -------------------------------------------------------------------------------- layer norm

def norm_inputs(rows, cols, T, seed):
    g = gen(seed)
    x = (torch.randn(rows, cols, generator=g) * 2 + torch.randn(rows, 1, generator=g)).to(T).cuda()
    if rows > 2:
        x[1] = 0.0                                               # a row of padding
        x[2] = 3.0                                               # a constant row
    return g, x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("lead,gap", [(0, 0), (3, 5)])
def test_layer_norm_forward(dtype, rows, cols, residual, lead, gap):
    T = TYPES[dtype]
    eps = 1e-5
    g, x = norm_inputs(rows, cols, T, rows + cols)
    r = randn(g, rows, cols, dtype=T) if residual else None
    w, b = randn(g, cols, dtype=T), randn(g, cols, dtype=T)
    xv, _ = placed(x, lead, gap)
    y, ybuf = empty_like_placed(x, lead, gap)
    s_out, sbuf = empty_like_placed(x, lead, gap)
    ck_sum, ck_y = fa().new_checkpoint8(rows, cols, "cuda"), fa().new_checkpoint8(rows, cols, "cuda")
    got_y, mean, rstd, got_s = fa().fa_layer_norm_forward(xv, w, b, eps, residual=r, y=y, sum_out=s_out, ck_sum=ck_sum,
                                                          ck_y=ck_y)
    assert got_y is y and got_s is s_out
    s = x.double() + (r.double() if residual else 0.0)
    ey, emean, erstd = ref.layer_norm(s, w.double(), b.double(), eps)
    big = s.abs().amax(1)
    ref.assert_close(mean, emean, big, 64, "mean")
    # relative error of rstd: half of that of the variance, which centred values give to 64 units, and
    # twice the mean's error against the deviations where these are small (constant rows: eps decides)
    ref.assert_close(rstd, erstd, erstd * (1 + (big * erstd) ** 2 * 2.0 ** -12), 128, "rstd")
    h = (s - emean[:, None]).abs() * erstd[:, None]
    scale = (h * (1 + (big * erstd)[:, None] ** 2 * 2.0 ** -12) + (big * erstd)[:, None]) * w.double().abs() + b.double().abs()
    ref.assert_close(y, ey, scale, 192, "y")
    ref.assert_close(s_out, s, s.abs(), 1, "sum")
    assert outside_untouched(y, ybuf) and outside_untouched(s_out, sbuf)
    # the checkpoints are those of what was stored
    for ck, t in ((ck_sum, s_out), (ck_y, y)):
        for a, c in zip(ref.buffer_parts(ck, rows, cols), ref.buffer_parts(fa().fa_checkpoint8_store(t), rows, cols)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("pdtype", TYPES)
@pytest.mark.parametrize("which", ["none", "weight", "bias"])
def test_layer_norm_without_parameters_and_with_the_other_type(pdtype, which):
    g, x = norm_inputs(9, 264, torch.bfloat16, 5)
    w = randn(g, 264, dtype=TYPES[pdtype]) if which == "weight" else None
    b = randn(g, 264, dtype=TYPES[pdtype]) if which == "bias" else None
    y, mean, rstd, s = fa().fa_layer_norm_forward(x, w, b, 1e-6)
    assert s is x
    ey, _, _ = ref.layer_norm(x.double(), None if w is None else w.double(), None if b is None else b.double(), 1e-6)
    ref.assert_close(y, ey, 4000.0, 64, "y")        # (|x| + |mean|) rstd of the constant row: 3 * 1e3
    dy = randn(g, 9, 264, dtype=torch.bfloat16)
    dx, dw, db = fa().fa_layer_norm_backward(dy, w, mean, rstd, x=x, dbias=False)
    assert db is None and dw.dtype == torch.float32
    e = ref.layer_norm_grad(dy.double(), x.double(), mean.double(), rstd.double(), None if w is None else w.double(), None)
    ref.assert_close(dw, e[1], (dy.double().abs() * 8).sum(0), 128, "dweight")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gdtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES + [(1500, 136)])
@pytest.mark.parametrize("source", ["x", "ck"])
@pytest.mark.parametrize("residual,lead,gap", [(False, 0, 0), (True, 3, 5)])
def test_layer_norm_backward(dtype, gdtype, rows, cols, source, residual, lead, gap):
    T = TYPES[dtype]
    g, x = norm_inputs(rows, cols, T, rows * 7 + cols)
    w = randn(g, cols, dtype=T)
    dy = randn(g, rows, cols, dtype=T, scale=0.1)
    r = randn(g, rows, cols, dtype=T, scale=0.1) if residual else None
    x64 = x.double()
    ck = None
    if source == "ck":
        ck = fa().fa_checkpoint8_store(x)
        x64 = ref.decode(ck, rows, cols).cuda()
    _, mean, rstd = ref.layer_norm(x.double(), None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    dyv, _ = placed(dy, lead, gap)
    xv, _ = placed(x, lead, gap)
    dx, dxbuf = empty_like_placed(x, lead, gap)
    row = torch.full((2 * cols + 16,), math.nan, dtype=TYPES[gdtype], device="cuda")    # a worker's gradient row
    fa().fa_layer_norm_backward(dyv, w, mean, rstd, x=xv if ck is None else None, ck=ck, residual_grad=r, dx=dx,
                                dweight=row[3:3 + cols], dbias=row[3 + cols:3 + 2 * cols])
    edx, edw, edb = ref.layer_norm_grad(dy.double(), x64, mean.double(), rstd.double(), w.double(),
                                        r.double() if residual else None)
    rs = rstd.double()[:, None]
    spread = (x64.abs() + mean.double().abs()[:, None]) * rs          # magnitudes behind h
    gmag = dy.double().abs() * w.double().abs()
    hmag = spread.amax(1, keepdim=True)
    scale = rs * (gmag + gmag.mean(1, keepdim=True) + hmag * (gmag * spread).mean(1, keepdim=True)) + (r.double().abs() if residual else 0)
    ref.assert_close(dx, edx, scale, 128, "dx")
    units = rows / 8 + 128
    ref.assert_close(row[3:3 + cols], edw, (dy.double().abs() * spread).sum(0), units, "dweight")
    ref.assert_close(row[3 + cols:3 + 2 * cols], edb, dy.double().abs().sum(0), units, "dbias")
    assert outside_untouched(dx, dxbuf) and torch.isnan(row[:3]).all() and torch.isnan(row[3 + 2 * cols:]).all()


def test_layer_norm_gradient_against_differences():
    rows, cols, eps = 6, 200, 1e-5
    g = gen(11)
    x, w, b, up = (randn(g, *s) for s in ((rows, cols), (cols,), (cols,), (rows, cols)))
    _, mean, rstd, _ = fa().fa_layer_norm_forward(x, w, b, eps)
    dx, dw, db = fa().fa_layer_norm_backward(up, w, mean, rstd, x=x)

    def loss(x, w, b):
        return float((ref.layer_norm(x, w, b, eps)[0] * up.double()).sum())

    args = [x.double(), w.double(), b.double()]
    for k, grad in enumerate((dx, dw, db)):
        u = randn(g, *grad.shape).double()
        h = 1e-5
        plus, minus = [list(args) for _ in range(2)]
        plus[k], minus[k] = args[k] + h * u, args[k] - h * u
        slope = (loss(*plus) - loss(*minus)) / (2 * h)
        # differences: h^2 times third derivatives of order one and 1e-16 / h of the loss; gradient: fp32
        assert abs(slope - float((grad.double() * u).sum())) <= 1e-4 * float((grad.double() * u).abs().sum())


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_of_non_finite_rows(dtype):
    """A broken row stays broken and stays the only one; parameter gradients show it in their sums."""
    g, x = norm_inputs(5, 96, TYPES[dtype], 2)
    w = randn(g, 96, dtype=TYPES[dtype])
    x[3, 7], x[4, 9] = math.inf, math.nan
    y, mean, rstd, _ = fa().fa_layer_norm_forward(x, w)
    assert torch.isfinite(y[:3]).all() and torch.isnan(y[3:]).all()
    clean, _, _, _ = fa().fa_layer_norm_forward(x[:3].clone(), w)
    assert torch.equal(y[:3], clean)
    dy = randn(g, 5, 96, dtype=TYPES[dtype])
    ck = fa().fa_checkpoint8_store(x)
    dx, dw, db = fa().fa_layer_norm_backward(dy, w, mean, rstd, ck=ck)
    assert torch.isfinite(dx[:3]).all() and torch.isnan(dx[3:]).all() and torch.isnan(dw).all() and torch.isfinite(db).all()


# --------------------------------------------------------------------------------------- GELU

GELU_SIZES = [(1, 1), (3, 7), (2, 33), (64, 40), (1, 4096), (37, 1001), (300, 1032), (1030, 160), (5, 20001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", ["tanh", "erf"])
@pytest.mark.parametrize("rows,cols", GELU_SIZES)
@pytest.mark.parametrize("with_bias,lead,gap", [(False, 0, 0), (True, 3, 5)])
def test_gelu_forward(dtype, form, rows, cols, with_bias, lead, gap):
    T = TYPES[dtype]
    g = gen(rows + cols)
    x = randn(g, rows, cols, dtype=T, scale=2.0)
    b = randn(g, cols, dtype=T) if with_bias else None
    xv, _ = placed(x, lead, gap)
    y, ybuf = empty_like_placed(x, lead, gap)
    ck_x, ck_y = fa().new_checkpoint8(rows, cols, "cuda"), fa().new_checkpoint8(rows, cols, "cuda")
    fa().fa_gelu_forward(xv, b, approximate=form, y=y, ck_x=ck_x, ck_y=ck_y)
    z = x.double() + (b.double() if with_bias else 0.0)
    # the argument of the exponential is off by 4 units of its magnitude, |2u| <= 2 (|z| + |z|^3); tails decay
    ref.assert_close(y, ref.gelu(z, form), 1 + z.abs(), 64, "y")
    assert outside_untouched(y, ybuf)
    z32 = (x.float() + b.float()) if with_bias else x
    for ck, t in ((ck_x, z32), (ck_y, y)):
        for a, c in zip(ref.buffer_parts(ck, rows, cols), ref.buffer_parts(fa().fa_checkpoint8_store(t), rows, cols)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", ["tanh", "erf"])
@pytest.mark.parametrize("rows,cols", GELU_SIZES)
@pytest.mark.parametrize("source,gdtype,lead,gap", [("x", "f32", 0, 0), ("ck", "bf16", 0, 0), ("x", "bf16", 3, 5), ("ck", "f32", 3, 5)])
def test_gelu_backward(dtype, form, rows, cols, source, gdtype, lead, gap):
    T = TYPES[dtype]
    g = gen(rows * 3 + cols)
    x = randn(g, rows, cols, dtype=T, scale=2.0)
    b = randn(g, cols, dtype=T) if source == "x" and lead else None
    dy = randn(g, rows, cols, dtype=T)
    ck = fa().fa_checkpoint8_store(x) if source == "ck" else None
    z = ref.decode(ck, rows, cols).cuda() if ck is not None else x.double() + (b.double() if b is not None else 0.0)
    dyv, _ = placed(dy, lead, gap)
    xv, _ = placed(x, lead, gap)
    dx, dxbuf = empty_like_placed(x, lead, gap)
    row = torch.full((cols + 8,), math.nan, dtype=TYPES[gdtype], device="cuda")
    fa().fa_gelu_backward(dyv, x=xv if ck is None else None, bias=b, ck=ck, approximate=form, dx=dx, dbias=row[1:1 + cols])
    e = dy.double() * ref.gelu_slope(z, form)
    scale = dy.double().abs() * (1 + z.abs())
    ref.assert_close(dx, e, scale, 64, "dx")
    ref.assert_close(row[1:1 + cols], e.sum(0), scale.sum(0), rows / 8 + 128 + 64, "dbias")
    assert outside_untouched(dx, dxbuf) and torch.isnan(row[:1]).all() and torch.isnan(row[1 + cols:]).all()
    again, none = fa().fa_gelu_backward(dyv, x=xv if ck is None else None, bias=b, ck=ck, approximate=form, dbias=False)
    assert none is None and torch.equal(again, dx)


@pytest.mark.parametrize("form", ["tanh", "erf"])
def test_gelu_far_out_and_against_differences(form):
    z = torch.tensor([[0.0, -0.0, 30.0, -30.0, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38, 1e-30, -1e-30]], device="cuda")
    one = torch.ones_like(z)
    y = fa().fa_gelu_forward(z, approximate=form)
    ref.assert_close(y, torch.where(z > 1, z, torch.zeros_like(z)) + torch.where(z.abs() < 1, z / 2, torch.zeros_like(z)),
                     z.abs().clamp(max=1), 4, "far out")
    d, _ = fa().fa_gelu_backward(one, x=z, approximate=form, dbias=False)
    want = torch.where(z.abs() < 1, 0.5, (z > 0).double())
    ref.assert_close(d, want, 1.0, 4, "slope far out")
    x = torch.linspace(-6, 6, 1001, device="cuda")[None]
    d, _ = fa().fa_gelu_backward(torch.ones_like(x), x=x, approximate=form, dbias=False)
    h = 1e-5
    slope = (ref.gelu(x.double() + h, form) - ref.gelu(x.double() - h, form)) / (2 * h)
    assert (d.double() - slope).abs().max() <= 1e-5             # h^2 and fp32 are both far below


# --------------------------------------------------------------------- linear weight gradient

WGRAD_SIZES = [(1, 1, 1), (3, 5, 7), (16, 64, 32), (17, 130, 33), (64, 128, 128), (100, 8, 1000), (333, 250, 130),
               (257, 264, 520), (1024, 256, 128), (2049, 72, 136), (4100, 24, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gdtype", TYPES)
@pytest.mark.parametrize("rows,outs,ins", WGRAD_SIZES)
@pytest.mark.parametrize("lead,gap", [(0, 0), (1, 3)])
def test_linear_weight_grad(dtype, gdtype, rows, outs, ins, lead, gap):
    T = TYPES[dtype]
    g = gen(rows + outs + ins)
    dy = randn(g, rows, outs, dtype=T, scale=1e-2)
    ck = fa().fa_checkpoint8_store(randn(g, rows, ins, dtype=T, scale=2.0) + 0.5)
    x = ref.decode(ck, rows, ins).cuda()
    dyv, _ = placed(dy, lead, gap)
    row = torch.full((outs * (ins + 1) + 8,), math.nan, dtype=TYPES[gdtype], device="cuda")
    dw = row[1:1 + outs * ins].view(outs, ins)
    db = row[1 + outs * ins:1 + outs * (ins + 1)]
    got = fa().fa_linear_weight_grad(dyv, ck, ins, dweight=dw, dbias=db)
    assert got[0] is dw and got[1] is db
    # sums of 16 products enter an fp32 accumulator one after the other, each addition off by at most two
    # units whatever its rounding; parts of the sum (at most 32) are added at the end
    units = 2 * (rows / 16 + 34) + 16
    ref.assert_close(dw, dy.double().T @ x, dy.double().abs().T @ x.abs(), units, "dweight")
    ref.assert_close(db, dy.double().sum(0), dy.double().abs().sum(0), rows / 8 + 128, "dbias")
    assert torch.isnan(row[:1]).all() and torch.isnan(row[1 + outs * (ins + 1):]).all()


# more than 2^31 products: pairs of blocks and wider tiles; sums read out in several runs; narrow inputs
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gdtype", TYPES)
@pytest.mark.parametrize("rows,outs,ins", [(2100, 1030, 1100), (2300, 2310, 2330), (4200, 520, 1000), (33000, 300, 230),
                                           (70000, 300, 120), (2304, 4096, 512), (40001, 640, 256)])
def test_linear_weight_grad_of_many_products(dtype, gdtype, rows, outs, ins):
    T, G = TYPES[dtype], TYPES[gdtype]
    g = gen(rows + outs + ins)
    dy = randn(g, rows, outs, dtype=T, scale=1e-2)
    ck = fa().fa_checkpoint8_store(randn(g, rows, ins, dtype=T, scale=2.0) + 0.5)
    x = ref.decode(ck, rows, ins).cuda()
    row = torch.full((outs * (ins + 1) + 8,), math.nan, dtype=G, device="cuda")
    dw, db = row[1:1 + outs * ins].view(outs, ins), row[1 + outs * ins:1 + outs * (ins + 1)]
    fa().fa_linear_weight_grad(dy, ck, ins, dweight=dw, dbias=db)
    exact, mags = dy.double().T @ x, dy.double().abs().T @ x.abs()
    units = 2 * (rows / 16 + 34) + 16                            # as above
    ref.assert_close(dw, exact, mags, units, "dweight")
    if gdtype == "f32":      # summed in runs of at most 512 additions at two units, then at most rows / 512 + 34 more
        ref.assert_close(dw, exact, mags, 2 * (512 + rows / 512 + 34), "dweight in runs")
    ref.assert_close(db, dy.double().sum(0), dy.double().abs().sum(0), rows / 8 + 128, "dbias")
    assert torch.isnan(row[:1]).all() and torch.isnan(row[1 + outs * (ins + 1):]).all()
    only, none = fa().fa_linear_weight_grad(dy, ck, ins, dweight=torch.empty(outs, ins, dtype=G, device="cuda"), dbias=False)
    assert none is None and torch.equal(only, dw)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_weight_grad_keeps_broken_values_in_their_places(dtype):
    rows, outs, ins = 70, 48, 200
    g = gen(1)
    dy = randn(g, rows, outs, dtype=TYPES[dtype])
    x = randn(g, rows, ins, dtype=TYPES[dtype])
    x[69, 40] = math.nan                                         # its group of 32 inputs (32..63) reads back as NaN
    dy[5, 7] = math.inf
    dw, db = fa().fa_linear_weight_grad(dy, fa().fa_checkpoint8_store(x), ins)
    assert torch.isnan(dw[:, 32:64]).all()
    fine = torch.ones_like(dw, dtype=torch.bool)
    fine[:, 32:64] = False
    fine[7] = False
    assert torch.isfinite(dw[fine]).all() and not torch.isfinite(dw[7]).any()
    assert torch.isinf(db[7]) and torch.isfinite(db[:7]).all() and torch.isfinite(db[8:]).all()


def test_linear_weight_grad_of_exact_sums():
    """Small whole numbers: every product and sum is exact, so the result is, in each type."""
    rows, outs, ins = 1000, 136, 264
    g = gen(8)
    dy = torch.randint(-3, 4, (rows, outs), generator=g).float().cuda()
    x = torch.randint(-7, 8, (rows, ins), generator=g).float().cuda()
    x[:, ::32] = 64.0                                            # the scale of every group is 1
    ck = fa().fa_checkpoint8_store(x)
    for T in TYPES.values():
        dw, db = fa().fa_linear_weight_grad(dy.to(T), ck, ins)
        assert torch.equal(dw.double(), dy.double().T @ x.double()) and torch.equal(db.double(), dy.double().sum(0))


# ------------------------------------------------------------------------------ how it is called

def test_no_rows_and_shapes_with_more_dimensions():
    x = torch.zeros(0, 40, device="cuda")
    y, mean, rstd, _ = fa().fa_layer_norm_forward(x)
    assert y.shape == (0, 40) and mean.numel() == 0
    ck = fa().fa_checkpoint8_store(x)
    assert fa().fa_checkpoint8_load(ck, 0, 40).shape == (0, 40)
    dx, dw, db = fa().fa_layer_norm_backward(x, None, mean, rstd, x=x)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    dx, db = fa().fa_gelu_backward(x, x=x)
    assert dx.shape == (0, 40) and not db.any()
    dw, db = fa().fa_linear_weight_grad(torch.zeros(0, 24, device="cuda"), ck, 40)
    assert dw.shape == (24, 40) and not dw.any() and not db.any()
    g = gen(6)
    x = randn(g, 3, 5, 64)
    y = fa().fa_gelu_forward(x)
    assert y.shape == x.shape and torch.equal(y.view(15, 64), fa().fa_gelu_forward(x.view(15, 64)))
    part = randn(g, 3, 5, 80)[..., 8:72]                          # leading dimensions collapse, rows have gaps
    assert torch.equal(fa().fa_gelu_forward(part), fa().fa_gelu_forward(part.contiguous()))
    one = randn(g, 1, 64).expand(7, 64)                           # one row for all
    assert torch.equal(fa().fa_layer_norm_forward(one)[0], fa().fa_layer_norm_forward(one.contiguous())[0])


def run_all(dtype, rows=517, cols=776, outs=200):
    T = TYPES[dtype]
    g = gen(21)
    x, dy = randn(g, rows, cols, dtype=T), randn(g, rows, cols, dtype=T)
    w, b, dz = randn(g, cols, dtype=T), randn(g, cols, dtype=T), randn(g, rows, outs, dtype=T)

    def calls(stream=None):
        f = fa()
        ck_s, ck_y, ck_z = (f.new_checkpoint8(rows, cols, "cuda") for _ in range(3))
        y, mean, rstd, s = f.fa_layer_norm_forward(x, w, b, residual=dy, ck_sum=ck_s, ck_y=ck_y, stream=stream)
        a = f.fa_gelu_forward(y, b, ck_x=ck_z, stream=stream)
        out = [y, mean, rstd, s, a]
        out += f.fa_gelu_backward(dy, ck=ck_z, stream=stream)
        out += f.fa_layer_norm_backward(dy, w, mean, rstd, ck=ck_s, stream=stream)
        out += f.fa_linear_weight_grad(dz, ck_y, cols, stream=stream)
        return out + [f.fa_checkpoint8_load(ck_y, rows, cols, stream=stream)]
    return calls


@pytest.mark.parametrize("dtype", TYPES)
def test_same_bits_every_time_and_on_another_stream(dtype):
    calls = run_all(dtype)
    first = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for again in (calls(), calls(stream=side)):
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, again))


def test_calls_can_be_captured_in_a_graph():
    calls = run_all("bf16")
    want = calls()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_refusals_on_the_device():
    f = fa()
    x = torch.zeros(4, 64, device="cuda")
    ck = f.fa_checkpoint8_store(x)
    ones = torch.ones(4, device="cuda")
    with pytest.raises(ValueError, match="exactly one of x and ck"):
        f.fa_layer_norm_backward(x, None, ones, ones)
    with pytest.raises(ValueError, match="exactly one of x and ck"):
        f.fa_gelu_backward(x, x=x, ck=ck)
    with pytest.raises(ValueError, match="bias must be None"):
        f.fa_gelu_backward(x, ck=ck, bias=x[0])
    with pytest.raises(ValueError, match="approximate"):
        f.fa_gelu_forward(x, approximate="sigmoid")
    with pytest.raises(ValueError, match="at least .* bytes"):
        f.fa_checkpoint8_store(x, ck=ck[:100])
    with pytest.raises(ValueError, match="at least .* bytes"):
        f.fa_linear_weight_grad(x, ck, 4096)
    with pytest.raises(ValueError, match="64 elements"):
        f.fa_layer_norm_forward(x, weight=torch.ones(63, device="cuda"))
    with pytest.raises(ValueError, match="rows of 64"):
        f.fa_layer_norm_forward(x, residual=x[:3])
    with pytest.raises(ValueError, match="same dtype"):
        f.fa_layer_norm_forward(x, x[0], x[0].bfloat16())
    with pytest.raises(ValueError, match="dense along"):
        f.fa_gelu_forward(torch.zeros(64, 4, device="cuda").t())
    with pytest.raises(ValueError, match="collapse"):
        f.fa_gelu_forward(torch.zeros(3, 5, 64, device="cuda")[:, :4])
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        f.fa_gelu_forward(x.half())
    with pytest.raises(f.FaError, match="invalid argument"):
        f.fa_gelu_forward(x, y=x[:1].expand(4, 64))               # rows of the output lie on each other
    with pytest.raises(f.FaError, match="invalid argument"):
        f.fa_layer_norm_forward(x, eps=-1.0)
    with pytest.raises(f.FaError, match="misaligned"):
        f.fa_checkpoint8_load(torch.zeros(4096, dtype=torch.uint8, device="cuda")[1:], 4, 64)
    with pytest.raises(ValueError, match="at least"):
        f.fa_layer_norm_backward(x, None, ones, ones, x=x, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
