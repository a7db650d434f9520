"""A wait inside the weight gradient's kernel that runs out ends the kernel with NaN in the results it concerns, and the
next call works.

Nothing is made to fail here.  The launch is a correct one; a test hook of the library (exported, not part of the C ABI in
include/fa.h) shortens the limit of the waits to one cycle, so the first wait for an operand gives up while it is still on
the way.  The waits that let copies and products in flight end before a block exits keep limits of their own.
"""
import ctypes

import pytest
import torch

from tests.test_gpu_training_ops import TYPES, fa, gen, randn

pytestmark = pytest.mark.gpu


# tiles of 128 outputs, of 256 by one block and by a pair, of 512; one and several splits, one and several runs; more
# steps than a ring has stages
@pytest.mark.parametrize("rows,outs,ins,dtype,gdtype", [(20000, 128, 128, "bf16", "f32"), (20000, 200, 136, "f32", "bf16"),
                                                       (70000, 300, 120, "bf16", "f32"), (2304, 1024, 1024, "f32", "f32"),
                                                       (6000, 2048, 4096, "bf16", "f32"), (16384, 2048, 4096, "bf16", "bf16")])
def test_a_wait_that_runs_out_leaves_nan_and_the_next_call_works(rows, outs, ins, dtype, gdtype):
    f = fa()
    lib = ctypes.CDLL(f.LIB_PATH)
    lib.fa_test_set_weight_grad_wait_cycles.argtypes = [ctypes.c_longlong]
    lib.fa_test_set_weight_grad_wait_cycles.restype = None
    g = gen(rows)
    dy = randn(g, rows, outs, dtype=TYPES[dtype])
    ck = f.fa_checkpoint8_store(randn(g, rows, ins, dtype=TYPES[dtype]))
    new = lambda *shape: torch.zeros(*shape, dtype=TYPES[gdtype], device="cuda")  # noqa: E731
    want = f.fa_linear_weight_grad(dy, ck, ins, dweight=new(outs, ins), dbias=new(outs))
    torch.cuda.synchronize()
    try:
        lib.fa_test_set_weight_grad_wait_cycles(1)
        dw, db = f.fa_linear_weight_grad(dy, ck, ins, dweight=new(outs, ins), dbias=new(outs))
        torch.cuda.synchronize()
    finally:
        lib.fa_test_set_weight_grad_wait_cycles(0)                # back to the default limit
    assert torch.isnan(dw).all()
    assert torch.equal(db, want[1])                               # the column sums wait for nothing
    for got, expected in zip(f.fa_linear_weight_grad(dy, ck, ins, dweight=new(outs, ins), dbias=new(outs)), want):
        assert torch.isfinite(expected).all() and torch.equal(got, expected)
