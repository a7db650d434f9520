"""Robust data-parallel training of a transformer's MLP block, on one GPU.

p workers (their batches run one after the other here) learn to reproduce a fixed random block

    f(x) = x + W2 gelu(W1 norm(x) + b1) + b2

from noisy targets; some of them send garbage.  Each honest worker's forward pass keeps its
activations as 8-bit checkpoints only; its backward pass writes every parameter gradient where it
belongs in the worker's row of the gradient matrix G, and the Flag Aggregator turns G into one update.

    python examples/train_mlp_block.py [--workers 7 --byzantine 2 --width 256 --hidden 1024 --tokens 2048 --steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2302_05865_b200 as fa  # noqa: E402


class Block:
    """The block's parameters as one flat fp32 vector (its gradient is a row of G), and bf16 copies to compute with."""

    def __init__(self, width, hidden, generator):
        self.shapes = dict(norm_weight=(width,), norm_bias=(width,), w1=(hidden, width), b1=(hidden,), w2=(width, hidden), b2=(width,))
        self.flat = torch.zeros(sum(torch.Size(s).numel() for s in self.shapes.values()), device="cuda")
        for name, view in self.views(self.flat).items():
            if name == "norm_weight":
                view.fill_(1.0)
            elif name in ("w1", "w2"):
                view.copy_(torch.randn(view.shape, generator=generator) / view.shape[1] ** 0.5)
        self.refresh()

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def refresh(self):
        self.p = {k: v.to(torch.bfloat16) for k, v in self.views(self.flat).items()}

    def forward(self, x, checkpoints=None):
        p = self.p
        ck = checkpoints or {}
        y, mean, rstd, _ = fa.fa_layer_norm_forward(x, p["norm_weight"], p["norm_bias"], ck_sum=ck.get("x"), ck_y=ck.get("y"))
        ck["mean"], ck["rstd"] = mean, rstd
        a = fa.fa_gelu_forward(y @ p["w1"].T, p["b1"], ck_x=ck.get("z"), ck_y=ck.get("a"))
        return torch.addmm(p["b2"], a, p["w2"].T).add_(x)

    def backward(self, d, ck, row):
        """Gradients of sum(d * f(x)) with respect to the parameters into `row`; returns that of x."""
        p, g = self.p, self.views(row)
        fa.fa_linear_weight_grad(d, ck["a"], p["w2"].shape[1], dweight=g["w2"], dbias=g["b2"])
        dz, _ = fa.fa_gelu_backward(d @ p["w2"], ck=ck["z"], dbias=g["b1"])
        fa.fa_linear_weight_grad(dz, ck["y"], p["w1"].shape[1], dweight=g["w1"], dbias=False)
        dx, _, _ = fa.fa_layer_norm_backward(dz @ p["w1"], p["norm_weight"], ck["mean"], ck["rstd"], ck=ck["x"], residual_grad=d,
                                             dweight=g["norm_weight"], dbias=g["norm_bias"])
        return dx


def train(workers=7, byzantine=2, width=256, hidden=1024, tokens=2048, steps=40, rate=4.0, m=3, seed=0):
    """Mean squared error on held-out data before and after training."""
    generator = torch.Generator().manual_seed(seed)
    teacher, student = Block(width, hidden, generator), Block(width, hidden, generator)

    def batch():
        x = torch.randn(tokens, width, generator=generator).to(device="cuda", dtype=torch.bfloat16)
        noise = 0.05 * torch.randn(tokens, width, generator=generator).to(device="cuda", dtype=torch.bfloat16)
        return x, teacher.forward(x) + noise

    held_out = batch()

    def error():
        return float((student.forward(held_out[0]).float() - held_out[1].float()).square().mean())

    G = torch.empty(workers, student.flat.numel(), device="cuda")
    ck = {k: fa.new_checkpoint8(tokens, n, "cuda") for k, n in (("x", width), ("y", width), ("z", hidden), ("a", hidden))}
    ws = fa.new_workspace(G, m)
    before = error()
    for _ in range(steps):
        for w in range(workers):
            x, target = batch()
            d = (student.forward(x, ck) - target) * (2.0 / (tokens * width))
            student.backward(d, ck, G[w])
            if w < byzantine:
                G[w].copy_(torch.randn(G.shape[1], generator=generator) * 10.0 * G[w].abs().mean().cpu())
        student.flat.sub_(fa.fa_aggregate(G, m, 0.0, 10, ws=ws), alpha=rate)
        student.refresh()
    return before, error()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("workers", 7), ("byzantine", 2), ("width", 256), ("hidden", 1024), ("tokens", 2048), ("steps", 40)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    before, after = train(a.workers, a.byzantine, a.width, a.hidden, a.tokens, a.steps)
    print(f"mean squared error on held-out data: {before:.4f} -> {after:.4f}")


if __name__ == "__main__":
    main()
