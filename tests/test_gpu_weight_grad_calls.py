"""Ways to call the weight gradient of a linear layer: one row of dy for all tokens, and how much workspace that takes."""
import pytest
import torch

from tests import training_reference as ref
from tests.test_gpu_training_ops import TYPES, fa, gen, randn

pytestmark = pytest.mark.gpu

OK, WORKSPACE = 0, -3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,outs,ins", [(1, 64, 40), (300, 64, 40), (1000, 264, 136)])
def test_one_row_of_dy_for_all_tokens(dtype, rows, outs, ins):
    """dy broadcast along its rows (stride 0), through the binding and the C ABI: the same bits as its copy."""
    f, T = fa(), TYPES[dtype]
    g = gen(rows + outs)
    dy = randn(g, 1, outs, dtype=T).expand(rows, outs)
    ck = f.fa_checkpoint8_store(randn(g, rows, ins, dtype=T))
    dw, db = f.fa_linear_weight_grad(dy, ck, ins)
    x = ref.decode(ck, rows, ins).cuda()
    # 1000 tokens: at most 63 additions at two units, and 34 of parts
    ref.assert_close(dw, dy.double().T @ x, dy.double().abs().T @ x.abs(), 2 * (rows / 16 + 34) + 16, "dweight")
    ref.assert_close(db, dy.double().sum(0), dy.double().abs().sum(0), rows / 8 + 128, "dbias")
    for got, want in zip(f.fa_linear_weight_grad(dy.contiguous(), ck, ins), (dw, db)):
        assert torch.equal(got, want)
    code = f.FA_BF16 if dtype == "bf16" else f.FA_F32
    raw_w, raw_b = torch.empty_like(dw), torch.empty_like(db)

    def call(nbytes):
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        return f._lib.fa_linear_weight_grad(dy.data_ptr(), 0, code, rows, outs, ck.data_ptr(), ins, raw_w.data_ptr(), raw_b.data_ptr(),
                                            f.FA_F32, ws.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)

    # a row stride below outs is not `aligned`, whatever it is a multiple of: dy is laid out in the workspace
    if dtype == "bf16":
        assert call(f.fa_linear_weight_grad_workspace_bytes(rows, outs, ins, T, aligned=True)) == WORKSPACE
    assert call(f.fa_linear_weight_grad_workspace_bytes(rows, outs, ins, T)) == OK
    assert torch.equal(raw_w, dw) and torch.equal(raw_b, db)


@pytest.mark.parametrize("scale", [1e-30, 1e-34, 1e-36, 1e-38, 1e-41])
def test_the_smallest_fp32_gradients_are_cut_off_at_a_multiple_of_2_to_the_minus_133(scale):
    rows, outs, ins = 256, 64, 64
    g = gen(3)
    dy = (torch.randn(rows, outs, generator=g, dtype=torch.float64) * scale).float().cuda()
    ck = fa().fa_checkpoint8_store(randn(g, rows, ins, scale=1e5))
    x = ref.decode(ck, rows, ins).cuda()
    dw, db = fa().fa_linear_weight_grad(dy, ck, ins)
    units = (2 * (rows / 16 + 34) + 16) * 2.0 ** -24              # of the sums, as in the other tests
    assert ((dw - dy.double().T @ x).abs() <= units * (dy.double().abs().T @ x.abs()) + 2.0 ** -133 * x.abs().sum(0)).all()
    assert ((db - dy.double().sum(0)).abs() <= (rows / 8 + 128) * 2.0 ** -24 * dy.double().abs().sum(0) + rows * 2.0 ** -133).all()
