"""The example that runs the training operators and the aggregation together: its gradients against
automatic differentiation in 64 bits, and that training with broken workers reduces the error."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def test_gradients_in_a_row_of_G_match_automatic_differentiation():
    import train_mlp_block as ex
    import paper_2302_05865_b200 as fa
    width, hidden, tokens = 96, 200, 300
    block = ex.Block(width, hidden, torch.Generator().manual_seed(3))
    g = torch.Generator().manual_seed(4)
    x = torch.randn(tokens, width, generator=g).to(device="cuda", dtype=torch.bfloat16)
    d = torch.randn(tokens, width, generator=g).to(device="cuda", dtype=torch.bfloat16)
    ck = {k: fa.new_checkpoint8(tokens, n, "cuda") for k, n in (("x", width), ("y", width), ("z", hidden), ("a", hidden))}
    row = torch.empty_like(block.flat)
    block.forward(x, ck)
    dx = block.backward(d, ck, row)
    p = {k: v.double().requires_grad_() for k, v in block.p.items()}
    x64 = x.double().requires_grad_()
    y = torch.nn.functional.layer_norm(x64, (width,), p["norm_weight"], p["norm_bias"], 1e-5)
    a = torch.nn.functional.gelu(y @ p["w1"].T + p["b1"], approximate="tanh")
    ((x64 + a @ p["w2"].T + p["b2"]) * d.double()).sum().backward()
    # Every checkpointed value is off by at most 1/126 of its group's largest (2.5 to 3 times the root mean square of
    # normal values), evenly spread: 0.7 % of the root mean square each; bf16 adds 0.2 % per step.  The sums over the
    # tokens keep these shares; a gradient meets at most four of them, in quadrature.
    for name, got in block.views(row).items():
        want = p[name].grad
        assert float((got.double() - want).norm() / want.norm()) < 0.02, name
    assert float((dx.double() - x64.grad).norm() / x64.grad.norm()) < 0.02


def test_training_with_broken_workers_reduces_the_error():
    import train_mlp_block as ex
    before, after = ex.train(workers=7, byzantine=2, width=128, hidden=256, tokens=1024, steps=30)
    assert after < 0.7 * before, (before, after)
