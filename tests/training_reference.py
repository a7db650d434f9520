"""Plain 64-bit statements of the training operators, for their tests (torch, any device)."""
import math

import torch


def encode(x):
    """(codes int8 (rows, 32 * groups), scale bytes uint8 (rows, groups)) of x, by the definition, value by value."""
    rows, cols = x.shape
    groups = -(-cols // 32)
    v = torch.zeros(rows, groups * 32, dtype=torch.float64)
    v[:, :cols] = x.double().cpu()
    v = v.view(rows, groups, 32)
    codes = torch.zeros(rows, groups, 32, dtype=torch.int8)
    scales = torch.zeros(rows, groups, dtype=torch.uint8)
    for r in range(rows):
        for g in range(groups):
            amax = float(v[r, g].abs().max())
            if not all(math.isfinite(t) for t in v[r, g].tolist()):
                scales[r, g] = 255
                continue
            e = -127
            while 127.0 * 2.0 ** e < amax:
                e += 1
            scales[r, g] = e + 127
            top = 63 if e == 122 else 127                                   # 64 * 2^122 is no finite float
            codes[r, g] = torch.round(v[r, g] / 2.0 ** e).clamp(-top, top).to(torch.int8)    # half to even
    return codes.view(rows, -1), scales


def buffer_parts(ck, rows, cols):
    """(codes, scale bytes of the groups, scale bytes of the padding) of a checkpoint buffer."""
    groups = -(-cols // 32)
    pitch = -(-groups // 4) * 4
    start = -(-rows * groups * 32 // 256) * 256
    codes = ck[:rows * groups * 32].cpu().view(torch.int8).view(rows, groups * 32)
    scales = ck[start:start + rows * pitch].cpu().view(rows, pitch)
    return codes, scales[:, :groups], scales[:, groups:]


def decode(ck, rows, cols):
    codes, scales, _ = buffer_parts(ck, rows, cols)
    s = torch.exp2(scales.double() - 127.0)
    s[scales == 255] = math.nan
    return (codes.double().view(rows, -1, 32) * s[:, :, None]).reshape(rows, -1)[:, :cols]


def layer_norm(s, weight, bias, eps):
    mean = s.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((s - mean) ** 2).mean(1, keepdim=True) + eps)
    y = (s - mean) * rstd
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_grad(dy, s, mean, rstd, weight, residual_grad):
    h = (s - mean[:, None]) * rstd[:, None]
    g = dy if weight is None else dy * weight
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    if residual_grad is not None:
        dx = dx + residual_grad
    return dx, (dy * h).sum(0), dy.sum(0)


def gelu(z, form):
    if form == "erf":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def gelu_slope(z, form):
    if form == "erf":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)


def assert_close(got, exact, scale, ulps, what):
    """|got - exact| <= ulps * 2^-24 * scale, and the rounding to got's type (bf16: half a unit is 2^-9 of
    the value, taken twice for a value that fp32 noise moves across a rounding boundary)."""
    got64, exact = got.double().cpu(), exact.double().cpu()
    scale = torch.as_tensor(scale, dtype=torch.float64).cpu()
    bound = ulps * 2.0 ** -24 * scale + exact.abs() * (2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -23) + 1e-37
    bad = ~((got64 - exact).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(((got64 - exact).abs() / bound)[bad].nan_to_num(1e30).max()))
