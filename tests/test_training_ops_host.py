"""Host side of the training operators, without a GPU: sizes of buffers, refusals of the C ABI and of the
binding before anything is enqueued, and the tests' own 64-bit reference."""
import ctypes
import math

import pytest
import torch

from tests import training_reference as ref


@pytest.fixture(scope="module")
def fa():
    import __graft_entry__ as entry
    entry.build()
    import paper_2302_05865_b200 as fa
    return fa


F32, BF16 = 0, 1
OK, ARG, ALIGN, WORKSPACE = 0, -1, -2, -3


@pytest.mark.parametrize("rows,cols,want", [(0, 1, 0), (1, 1, 512), (3, 40, 512), (8, 32, 512), (9, 32, 768), (100, 768, 76800 + 2560)])
def test_checkpoint_bytes(fa, rows, cols, want):
    assert fa.fa_checkpoint8_bytes(rows, cols) == want


def test_size_limits(fa):
    size = ctypes.c_size_t(0)
    for rows, cols, code in ((-1, 8, ARG), (1, 0, ARG), (1, (1 << 23) + 1, ARG), ((1 << 40) + 1, 8, ARG), (1 << 40, 1 << 23, OK)):
        assert fa._lib.fa_checkpoint8_bytes(rows, cols, ctypes.byref(size)) == code
    assert fa._lib.fa_checkpoint8_bytes(1, 8, None) == ARG
    assert fa._lib.fa_linear_weight_grad_workspace_bytes(1, 8, 8, 5, 1, ctypes.byref(size)) == ARG
    # a bf16 dY on 16-byte boundaries needs no room of its own
    assert fa.fa_linear_weight_grad_workspace_bytes(4096, 4096, 1024, torch.bfloat16, True) < 4096 * 4096 * 2 <= \
        fa.fa_linear_weight_grad_workspace_bytes(4096, 4096, 1024, torch.bfloat16) < fa.fa_linear_weight_grad_workspace_bytes(4096, 4096, 1024, torch.float32, True)
    for rows in (0, 1, 100_000):
        assert 0 < fa.fa_layer_norm_backward_workspace_bytes(rows, 768) < 64 << 20
        assert 0 < fa.fa_gelu_backward_workspace_bytes(rows, 768) < 64 << 20


def test_refusals_of_the_c_abi(fa):
    """Addresses are made up: each call is refused before it reaches a device."""
    L, A, odd = fa._lib, 1 << 20, (1 << 20) + 1
    assert L.fa_checkpoint8_store(None, 8, F32, 4, 8, A, None) == ARG
    assert L.fa_checkpoint8_store(A, 8, 7, 4, 8, A, None) == ARG
    assert L.fa_checkpoint8_store(A, -8, F32, 4, 8, A, None) == ARG
    assert L.fa_checkpoint8_store(A, 8, F32, 4, 8, None, None) == ARG
    assert L.fa_checkpoint8_store(odd, 8, F32, 4, 8, A, None) == ALIGN
    assert L.fa_checkpoint8_store(A, 8, F32, 4, 8, A + 8, None) == ALIGN
    assert L.fa_checkpoint8_store(None, 8, F32, 0, 8, None, None) == OK
    assert L.fa_checkpoint8_load(A, F32, 4, 8, A, 7, None) == ARG               # output rows overlap
    assert L.fa_checkpoint8_load(A, BF16, 4, 8, odd, 8, None) == ALIGN
    gf = [A, 8, F32, 4, 8, A, F32, 1, A, 8, None, None, None]
    for k, v, code in ((0, None, ARG), (2, 3, ARG), (4, 0, ARG), (6, 9, ARG), (7, 2, ARG), (8, None, ARG), (9, 4, ARG), (5, odd, ALIGN), (10, odd, ALIGN)):
        assert L.fa_gelu_forward(*[v if i == k else a for i, a in enumerate(gf)]) == code, k
    gb = [A, 8, A, 8, None, F32, None, F32, 4, 8, 1, A, 8, A, F32, A, 1 << 20, None]
    for k, v, code in ((0, None, ARG), (2, None, ARG), (6, A, ARG), (11, None, ARG), (12, 0, ARG), (14, 2, ARG), (15, None, ARG), (16, 0, WORKSPACE),
                       (13, odd, ALIGN), (15, odd, ALIGN)):
        assert L.fa_gelu_backward(*[v if i == k else a for i, a in enumerate(gb)]) == code, k
    both = list(gb)
    both[2], both[6], both[4] = None, A, A                                       # a checkpoint and a bias
    assert L.fa_gelu_backward(*both) == ARG
    lf = [A, 8, None, 0, F32, 4, 8, A, A, F32, 1e-5, A, 8, None, 0, A, A, None, None, None]
    for k, v, code in ((0, None, ARG), (10, -1.0, ARG), (10, math.nan, ARG), (10, math.inf, ARG), (9, 4, ARG), (11, None, ARG), (6, 1 << 24, ARG),
                       (15, odd, ALIGN), (17, odd, ALIGN), (7, odd, ALIGN)):
        assert L.fa_layer_norm_forward(*[v if i == k else a for i, a in enumerate(lf)]) == code, k
    lb = [A, 8, A, 8, None, F32, 4, 8, A, F32, A, A, None, 0, A, 8, A, A, F32, A, 1 << 20, None]
    for k, v, code in ((0, None, ARG), (2, None, ARG), (4, A, ARG), (10, None, ARG), (14, None, ARG), (15, 7, ARG), (18, 5, ARG), (19, None, ARG),
                       (20, 8, WORKSPACE), (16, odd, ALIGN), (10, odd, ALIGN)):
        assert L.fa_layer_norm_backward(*[v if i == k else a for i, a in enumerate(lb)]) == code, k
    wg = [A, 8, BF16, 4, 8, A, 40, A, A, F32, A, 1 << 30, None]
    for k, v, code in ((0, None, ARG), (1, -1, ARG), (2, 2, ARG), (4, 0, ARG), (5, None, ARG), (6, 0, ARG), (7, None, ARG), (9, 2, ARG), (10, None, ARG),
                       (11, 0, WORKSPACE), (0, odd, ALIGN), (5, A + 8, ALIGN), (8, odd, ALIGN)):
        assert L.fa_linear_weight_grad(*[v if i == k else a for i, a in enumerate(wg)]) == code, k


def test_binding_refuses_cpu_tensors_and_wrong_types(fa):
    x = torch.zeros(4, 64)
    for call in (lambda: fa.fa_checkpoint8_store(x), lambda: fa.fa_gelu_forward(x), lambda: fa.fa_layer_norm_forward(x),
                 lambda: fa.fa_layer_norm_backward(x, None, x[0], x[0], x=x), lambda: fa.fa_gelu_backward(x, x=x),
                 lambda: fa.fa_linear_weight_grad(x, torch.zeros(4096, dtype=torch.uint8), 64),
                 lambda: fa.fa_checkpoint8_load(torch.zeros(4096, dtype=torch.uint8), 4, 64)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    for call in (lambda: fa.fa_gelu_forward(x.double()), lambda: fa.fa_checkpoint8_store([1.0]), lambda: fa.fa_checkpoint8_load([0], 1, 1)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="last dimension"):
        fa.fa_gelu_forward(torch.zeros(4, 0))


def test_row_strides_of_views(fa):
    from paper_2302_05865_b200.training import _row_stride
    t = torch.zeros(6, 5, 40)
    assert _row_stride(t[..., :32], "t") == 40 and _row_stride(t[:, :1, :32], "t") == 200 and _row_stride(t[0], "t") == 40
    assert _row_stride(t[:, 2], "t") == 200 and _row_stride(torch.zeros(1, 8).expand(3, 8), "t") == 0
    assert _row_stride(t[:1, :1, :8], "t") == 8
    for bad in (t[:, :3, :32], t.transpose(0, 1)):
        with pytest.raises(ValueError, match="collapse"):
            _row_stride(bad, "t")
    with pytest.raises(ValueError, match="dense"):
        _row_stride(t[..., ::2], "t")


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    x, w, b, up = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((4, 30), (30,), (30,), (4, 30)))
    _, mean, rstd = ref.layer_norm(x, w, b, 1e-5)
    dx, dw, db = ref.layer_norm_grad(up, x, mean, rstd, w, None)
    h = 1e-6
    for k, grad in enumerate((dx, dw, db)):
        u = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        f = lambda s: float((ref.layer_norm(*[t + s * u if i == k else t for i, t in enumerate((x, w, b))], 1e-5)[0] * up).sum())  # noqa: E731
        assert (f(h) - f(-h)) / (2 * h) == pytest.approx(float((grad * u).sum()), rel=1e-6, abs=1e-8)
    z = torch.linspace(-5, 5, 101, dtype=torch.float64)
    for form in ("tanh", "erf"):
        assert torch.allclose((ref.gelu(z + h, form) - ref.gelu(z - h, form)) / (2 * h), ref.gelu_slope(z, form), atol=1e-8)


def test_reference_codes_by_hand():
    codes, scales = ref.encode(torch.tensor([[127.0, -0.5, 1.5, 0.49] + [0.0] * 28, [254.0, 3.0, 1.0, -1.0] + [0.0] * 28]))
    assert scales.tolist() == [[127], [128]]
    assert codes[0, :4].tolist() == [127, 0, 2, 0] and codes[1, :4].tolist() == [127, 2, 0, 0]     # 1.5 -> 2, 0.5 -> 0
