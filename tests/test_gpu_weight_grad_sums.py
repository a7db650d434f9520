"""How exactly the weight gradient of a linear layer is summed, against 64 bits on the GPU.

The tensor cores cut a sum off after every 16 tokens instead of rounding it; the sums are therefore read out of their
accumulators in runs, and the runs added in fp32.  For inputs of random sign an accumulator of n additions is off by
at most n / 96 * 7e-7 of its result, and adding k runs in fp32 by sqrt(k) * 2^-25.
"""
import math

import pytest
import torch

from tests import training_reference as ref
from tests.test_gpu_training_ops import TYPES, fa

pytestmark = pytest.mark.gpu


def products(rows, outs, ins, T, positive, seed=5):
    """(dy, checkpoint of X, dy^T X in 64 bits)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    make = torch.rand if positive else torch.randn
    dy = (make(rows, outs, generator=g, device="cuda") * 1e-2).to(T)
    x = make(rows, ins, generator=g, device="cuda").to(T)
    ck = fa().fa_checkpoint8_store(x)
    read = fa().fa_checkpoint8_load(ck, rows, ins, dtype=torch.bfloat16)          # exact in bf16
    exact = torch.zeros(outs, ins, dtype=torch.float64, device="cuda")
    for r in range(0, rows, 16384):
        exact += dy[r:r + 16384].double().T @ read[r:r + 16384].double()
    return dy, ck, exact


def relative(got, exact):
    return float((got.double() - exact).norm() / exact.norm())


# tiles of 128 and 256 outputs, one and two accumulators, one and several splits, up to 22 runs
@pytest.mark.parametrize("rows,outs,ins,dtype", [(32768, 2048, 1024, "bf16"), (32768, 4096, 1024, "bf16"), (16384, 768, 768, "bf16"),
                                                 (40001, 640, 256, "bf16"), (8192, 640, 512, "f32"), (16384, 2048, 1024, "f32")])
def test_fp32_results_are_as_exact_as_documented(rows, outs, ins, dtype):
    dy, ck, exact = products(rows, outs, ins, TYPES[dtype], positive=False)
    dw, _ = fa().fa_linear_weight_grad(dy, ck, ins, dbias=False)
    # at most 7e-7 in runs of 24 steps (96 additions), of an fp32 dY with the small terms first 1.8e-7; half as much again
    assert relative(dw, exact) < (2.7e-7 if (dtype, rows) == ("f32", 8192) else 1.05e-6)


@pytest.mark.parametrize("rows,outs,ins,positive", [(32768, 4096, 1024, False), (16384, 4096, 4096, False), (16384, 768, 768, False),
                                                    (131072, 2048, 2048, True), (131072, 2048, 2048, False)])
def test_bf16_results_are_rounded_sums(rows, outs, ins, positive):
    """A result off by d of itself rounds another way for a share of d / 2^-7.5 of values, a few times that where sums
    cancel: below 1e-3 for sums in runs, whose error is less than 1e-6, but 3e-3 and more for sums that stay in one
    accumulator for half a thousand steps, and growing with their number."""
    dy, ck, exact = products(rows, outs, ins, torch.bfloat16, positive)
    dw = torch.empty(outs, ins, dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        fa().fa_linear_weight_grad(dy, ck, ins, dweight=dw, dbias=False)
        share = float((dw != exact.to(torch.float32).to(torch.bfloat16)).float().mean())
        assert share < 1e-3, share


@pytest.mark.parametrize("rows,outs,ins", [(32768, 4096, 1024), (16384, 4096, 4096), (20000, 1030, 2100)])
@pytest.mark.parametrize("gdtype", TYPES)
def test_results_in_several_runs_repeat_bit_for_bit(rows, outs, ins, gdtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.randn(rows, outs, generator=g, device="cuda", dtype=torch.bfloat16)
    ck = fa().fa_checkpoint8_store(torch.randn(rows, ins, generator=g, device="cuda", dtype=torch.bfloat16))
    calls = [fa().fa_linear_weight_grad(dy, ck, ins, dweight=torch.full((outs, ins), math.nan, dtype=TYPES[gdtype], device="cuda"))
             for _ in range(8)]
    for dw, db in calls[1:]:
        assert torch.equal(dw, calls[0][0]) and torch.equal(db, calls[0][1])
