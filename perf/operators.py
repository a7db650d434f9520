"""Cases of the training operators: layer norm with its gradient, activation checkpoints in 8 bits,
and the backward passes that read such checkpoints (layer norm, GELU, weight of a linear layer).

A worker of a data-parallel run calls these operators on its share of a batch; the parameter
gradients go to the worker's row of the gradient matrix that is aggregated afterwards, at the
element offset the parameter has in that row.

`run` computes a case in plain torch operations in 32 bits (`own` false) or through the framework
(`own` true); `exact` computes it in 64 bits from the definitions.

Checkpoint format: every row of d values is cut into groups of 32 (the last one filled up with
zeros).  A group has the scale 2^e, e the smallest integer >= -127 with 127 * 2^e >= its largest
magnitude; a value is held as the int8 code rint(v / 2^e).  The buffer holds the codes, rows x
32 * ceil(d / 32) bytes, and from the next multiple of 256 bytes the scales as bytes e + 127, rows x
(ceil(d / 32) rounded up to 4); the byte 255 marks a group with an Inf or NaN in it, all of which
reads back as NaN.
"""
import math

import torch

own = False

EPS = 1e-5
ROW_LEAD = 1237          # elements of a worker's gradient row in front of the parameters of a case: an odd offset


# ------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one token through a layer norm of GPT-2-small's width: nothing but the call's latency
        dict(name="ln_fwd_one_token", op="ln_fwd", rows=1, cols=768, dtype="bf16", residual=False, ck=False),
        # pre-norm block of a GPT-2-small-sized model, 16 sequences of 1024: residual add, norm, checkpoints
        # of the sum (for the norm's own backward pass) and of the output (for the next linear layer)
        dict(name="ln_fwd_residual_ck", op="ln_fwd", rows=16384, cols=768, dtype="bf16", residual=True, ck=True),
        # odd sizes in fp32 from the stored input itself: a small model trained in fp32
        dict(name="ln_bwd_f32_odd", op="ln_bwd", rows=1023, cols=1001, dtype="f32", ck=False, residual=False, grad="f32"),
        # wide model: backward from the 8-bit checkpoint, residual gradient added, parameter gradients into
        # a bf16 gradient row at an odd offset
        dict(name="ln_bwd_ck_wide", op="ln_bwd", rows=16384, cols=4096, dtype="bf16", ck=True, residual=True, grad="bf16"),
        # checkpoint of a short ragged fp32 activation and its way back
        dict(name="ck_f32_ragged", op="ck", rows=128, cols=1000, dtype="f32"),
        # checkpoint of a large activation of a wide model and its way back
        dict(name="ck_bf16_large", op="ck", rows=65536, cols=4096, dtype="bf16"),
        # activation of a 1024-wide model's MLP: bias, GELU, checkpoints of the input and of the output
        dict(name="gelu_fwd_ck", op="gelu_fwd", rows=16384, cols=4096, dtype="bf16", approx="tanh", ck=True),
        # a small odd-sized fp32 MLP with the erf form, input kept as it is
        dict(name="gelu_bwd_f32_odd", op="gelu_bwd", rows=257, cols=1111, dtype="f32", approx="erf", ck=False, grad="f32"),
        # the largest activation: backward from the checkpoint with the bias gradient
        dict(name="gelu_bwd_ck_large", op="gelu_bwd", rows=32768, cols=8192, dtype="bf16", approx="tanh", ck=True, grad="bf16"),
        # small ragged layer trained in fp32
        dict(name="wgrad_f32_ragged", op="wgrad", rows=333, outs=250, ins=130, dtype="f32", grad="f32"),
        # attention output projection of a GPT-2-small-sized model, 16 sequences of 1024: few tiles, a long sum
        dict(name="wgrad_768", op="wgrad", rows=16384, outs=768, ins=768, dtype="bf16", grad="f32"),
        # MLP projection of a 1024-wide model, into a bf16 gradient row
        dict(name="wgrad_wide", op="wgrad", rows=32768, outs=4096, ins=1024, dtype="bf16", grad="bf16"),
    ]


def _spread(rng, low, high):
    """A size between low and high, even over its logarithm; every other one odd."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    v = v | 1 if rng.random() < 0.5 else (v + 7) // 8 * 8
    return max(low, min(high, v if v != 3072 else v + 8))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "ck", "gelu_fwd", "gelu_bwd", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    case = dict(op=op, dtype=dtype)
    if op == "wgrad":
        outs, ins = _spread(rng, 64, 4096), _spread(rng, 64, 4096)
        # fp32 products cost three bf16 ones
        most = (1 << 37) // (outs * ins * (3 if dtype == "f32" else 1))
        case.update(rows=_spread(rng, 1, max(2, min(32768, most))), outs=outs, ins=ins, grad=rng.choice(["f32", "bf16"]))
        return case
    cols = _spread(rng, 33, 8192)
    case.update(rows=_spread(rng, 1, max(2, min(65536, (1 << 26) // cols))), cols=cols)
    if op != "ck":
        case["ck"] = rng.random() < 0.5
    if op in ("ln_fwd", "ln_bwd"):
        case["residual"] = rng.random() < 0.5
    if op in ("gelu_fwd", "gelu_bwd"):
        case["approx"] = rng.choice(["tanh", "erf"])
    if op in ("ln_bwd", "gelu_bwd"):
        case["grad"] = rng.choice(["f32", "bf16"])
    return case


# ----------------------------------------------------------------------------------------- inputs

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _checkpoint(v):
    """The checkpoint buffer of v, as the format above says."""
    rows, cols = v.shape
    groups = -(-cols // 32)
    pitch = -(-groups // 4) * 4
    codes, scales = _codes(v.float())
    start = -(-rows * groups * 32 // 256) * 256
    buf = torch.zeros(start + -(-rows * pitch // 256) * 256, dtype=torch.uint8, device=v.device)
    buf[:rows * groups * 32] = codes.to(torch.int8).view(torch.uint8).reshape(-1)
    buf[start:start + rows * pitch].view(rows, pitch)[:, :groups] = scales.to(torch.uint8)
    return buf


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, rows, dtype = case["op"], case["rows"], _type(case["dtype"])
    s = dict(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def stream(cols):
        """Hidden states: unit noise, an offset per column, a few columns that are ten times as large
        as the rest, and every 64th row zero (padding)."""
        scale = 1.0 + 9.0 * (torch.rand(cols, generator=g, device="cuda") < 0.02)
        x = (normal(rows, cols) + 0.5 * normal(cols)) * scale
        x[63::64] = 0.0
        return x.to(dtype)

    def upstream(cols):
        """Gradients from above: small, of a scale of its own per row, none for padding."""
        dy = normal(rows, cols) * (1e-3 * torch.exp(0.5 * normal(rows, 1)))
        dy[63::64] = 0.0
        return dy.to(dtype)

    if op == "wgrad":
        s["dy"] = upstream(case["outs"])
        s["ck"] = _checkpoint(stream(case["ins"]))
        s["row"] = torch.empty(ROW_LEAD + case["outs"] * (case["ins"] + 1), dtype=_type(case["grad"]), device="cuda")
        return s
    cols = case["cols"]
    s["x"] = stream(cols)
    if op == "ck":
        return s
    if op in ("ln_bwd", "gelu_bwd"):
        s["dy"] = upstream(cols)
        s["row"] = torch.empty(ROW_LEAD + 2 * cols, dtype=_type(case["grad"]), device="cuda")
    if op in ("ln_fwd", "ln_bwd"):
        s["weight"] = (1.0 + 0.2 * normal(cols)).to(dtype)
        s["bias"] = (0.1 * normal(cols)).to(dtype)
        s["other"] = (normal(rows, cols) if op == "ln_fwd" else upstream(cols).float()).to(dtype) if case["residual"] else None
    if op == "gelu_fwd":
        s["bias"] = (0.2 * normal(cols)).to(dtype)
    if op == "ln_bwd":
        x = s["x"].float()
        s["mean"] = x.mean(1)
        s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
    if op in ("ln_bwd", "gelu_bwd") and case["ck"]:
        s["ck"] = _checkpoint(s.pop("x"))
    return s


# ----------------------------------------------------------------------------- plain form, 32 bits

def _codes(v):
    """Codes (rows, groups, 32) and scale bytes (rows, groups) of v, fp32."""
    rows, cols = v.shape
    v = torch.nn.functional.pad(v, (0, -cols % 32)).view(rows, -1, 32)
    amax = v.abs().amax(2)
    m, k = torch.frexp(amax)
    e = torch.where(amax > 0, k - 7 + (m > 127.0 / 128.0), -127).clamp(min=-127)
    fine = torch.isfinite(amax)
    e = torch.where(fine, e, 128)
    codes = torch.where(fine[:, :, None], torch.round(torch.ldexp(v, -e[:, :, None])), 0.0)
    return codes, e + 127


def _values(codes, scales, cols):
    """What codes (rows, groups, 32) and scale bytes stand for, fp32."""
    e = scales.to(torch.int32) - 127
    scale = torch.where(e == 128, math.nan, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e))
    return (codes.float() * scale[:, :, None]).flatten(1)[:, :cols]


def _stored(v):
    """v after a way through a checkpoint, fp32."""
    return _values(*_codes(v), v.shape[1])


def _read(buf, rows, cols):
    """The values a checkpoint buffer holds, fp32."""
    groups = -(-cols // 32)
    pitch = -(-groups // 4) * 4
    start = -(-rows * groups * 32 // 256) * 256
    codes = buf[:rows * groups * 32].view(torch.int8).view(rows, groups, 32)
    return _values(codes, buf[start:start + rows * pitch].view(rows, pitch)[:, :groups], cols)


def _sigmoid_argument(z):
    """2u of gelu's tanh form z * (1 + tanh(u)) / 2 = z * sigmoid(2u), and its derivative."""
    c = 2.0 * math.sqrt(2.0 / math.pi)
    return c * (z + 0.044715 * z * z * z), c * (1.0 + 3.0 * 0.044715 * z * z)


def _plain(s):
    op, dtype = s["op"], _type(s["dtype"])
    if op == "ck":
        return _stored(s["x"].float()).to(dtype)
    if op == "ln_fwd":
        x = s["x"].float()
        if s["residual"]:
            x = x + s["other"].float()
        mean = x.mean(1)
        rstd = 1.0 / torch.sqrt((x - mean[:, None]).square().mean(1) + EPS)
        y = ((x - mean[:, None]) * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(dtype)
        out = [y, mean, rstd]
        total = x.to(dtype)
        if s["residual"]:
            out.append(total)
        if s["ck"]:
            out.append(_stored(total.float()).to(dtype))
            if dtype == torch.bfloat16:
                out.append(_stored(y.float()).to(dtype))
        return out
    if op == "ln_bwd":
        dy, grad = s["dy"].float(), _type(s["grad"])
        x = _read(s["ck"], *dy.shape) if "x" not in s else s["x"].float()
        rstd = s["rstd"][:, None]
        h = (x - s["mean"][:, None]) * rstd
        wdy = dy * s["weight"].float()
        dx = rstd * (wdy - wdy.mean(1, True) - h * (wdy * h).mean(1, True))
        if s["residual"]:
            dx = dx + s["other"].float()
        return dx.to(dtype), (dy * h).sum(0).to(grad), dy.sum(0).to(grad)
    if op == "gelu_fwd":
        z = s["x"].float() + s["bias"].float()
        if s["approx"] == "tanh":
            y = z * torch.sigmoid(_sigmoid_argument(z)[0])
        else:
            y = 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
        y = y.to(dtype)
        out = [y]
        if s["ck"]:
            out.append(_stored(z).to(dtype))
            if dtype == torch.bfloat16:
                out.append(_stored(y.float()).to(dtype))
        return out
    if op == "gelu_bwd":
        dy, grad = s["dy"].float(), _type(s["grad"])
        z = _read(s["ck"], *dy.shape) if "x" not in s else s["x"].float()
        if s["approx"] == "tanh":
            u, du = _sigmoid_argument(z)
            p = torch.sigmoid(u)
            d = p + z * p * (1.0 - p) * du
        else:
            d = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
        dz = dy * d
        return dz.to(dtype), dz.sum(0).to(grad)
    dy, grad = s["dy"].float(), _type(s["grad"])
    x = _read(s["ck"], s["rows"], s["ins"])
    return (dy.T @ x).to(grad), dy.sum(0).to(grad)


# ---------------------------------------------------------------------------------- the framework

def _own(s):
    import paper_2302_05865_b200 as fa
    op, dtype, rows = s["op"], _type(s["dtype"]), s["rows"]
    if op == "wgrad":
        outs, ins, row = s["outs"], s["ins"], s["row"]
        dweight = row[ROW_LEAD:ROW_LEAD + outs * ins].view(outs, ins)
        return fa.fa_linear_weight_grad(s["dy"], s["ck"], ins, dweight=dweight, dbias=row[ROW_LEAD + outs * ins:])
    cols = s["cols"]
    if op == "ck":
        ck = fa.fa_checkpoint8_store(s["x"])
        return fa.fa_checkpoint8_load(ck, rows, cols, dtype=dtype)
    if op == "ln_fwd":
        ck_sum = fa.new_checkpoint8(rows, cols, s["x"].device) if s["ck"] else None
        ck_y = fa.new_checkpoint8(rows, cols, s["x"].device) if s["ck"] and dtype == torch.bfloat16 else None
        y, mean, rstd, total = fa.fa_layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, residual=s["other"],
                                                        ck_sum=ck_sum, ck_y=ck_y)
        out = [y, mean, rstd] + ([total] if s["residual"] else [])
        return out + [fa.fa_checkpoint8_load(c, rows, cols, dtype=dtype) for c in (ck_sum, ck_y) if c is not None]
    if op == "gelu_fwd":
        ck_x = fa.new_checkpoint8(rows, cols, s["x"].device) if s["ck"] else None
        ck_y = fa.new_checkpoint8(rows, cols, s["x"].device) if s["ck"] and dtype == torch.bfloat16 else None
        y = fa.fa_gelu_forward(s["x"], s["bias"], approximate=s["approx"], ck_x=ck_x, ck_y=ck_y)
        return [y] + [fa.fa_checkpoint8_load(c, rows, cols, dtype=dtype) for c in (ck_x, ck_y) if c is not None]
    row = s["row"]
    first, second = row[ROW_LEAD:ROW_LEAD + cols], row[ROW_LEAD + cols:]
    if op == "ln_bwd":
        return fa.fa_layer_norm_backward(s["dy"], s["weight"], s["mean"], s["rstd"], x=s.get("x"), ck=s["ck"] if "x" not in s else None,
                                         residual_grad=s["other"], dweight=first, dbias=second)
    return fa.fa_gelu_backward(s["dy"], x=s.get("x"), ck=s["ck"] if "x" not in s else None, approximate=s["approx"], dbias=first)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what a pass must do

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    g = 2 if case.get("grad") == "bf16" else 4
    rows, op = case["rows"], case["op"]
    if op == "wgrad":
        outs, ins = case["outs"], case["ins"]
        return dict(bytes=rows * (outs * e + ins * 33 / 32) + outs * (ins + 1) * g, flops=2 * rows * outs * ins)
    cols = case["cols"]
    n, held = rows * cols, rows * cols * 33 / 32
    both = 2 if e == 2 else 1
    if op == "ck":                                     # values in, checkpoint out and in again, values out
        return dict(bytes=2 * n * e + 2 * held, flops=4 * n)
    if op == "ln_fwd":                                 # a checkpoint is written; its values come back as an output
        more = both * (held + n * e) if case["ck"] else 0
        return dict(bytes=n * e * (4 if case["residual"] else 2) + 8 * rows + 2 * cols * e + more, flops=8 * n)
    if op == "gelu_fwd":
        more = both * (held + n * e) if case["ck"] else 0
        return dict(bytes=2 * n * e + cols * e + more, flops=16 * n)
    stored = held if case["ck"] else n * e
    if op == "ln_bwd":
        return dict(bytes=n * e * (3 if case["residual"] else 2) + stored + 8 * rows + cols * e + 2 * cols * g, flops=14 * n)
    return dict(bytes=2 * n * e + stored + cols * g, flops=24 * n)


# ------------------------------------------------------------------------- definitions in 64 bits

def _through_checkpoint(v):
    """Each value of v rounded to a multiple of its group's power of two, v in 64 bits."""
    rows, cols = v.shape
    full = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=v.device)
    full[:, :cols] = v
    full = full.reshape(-1, 32)
    amax = full.abs().max(1, keepdim=True).values
    quantum = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=1e-300) / 127.0)).clamp(min=-127.0))
    quantum = torch.where(127.0 * quantum < amax, 2.0 * quantum, quantum)
    quantum = torch.where((63.5 * quantum >= amax) & (quantum > 2.0 ** -127), 0.5 * quantum, quantum)
    return (torch.round(full / quantum) * quantum).reshape(rows, -1)[:, :cols]


def _held(buf, rows, cols):
    """The values in a checkpoint buffer, in 64 bits."""
    width = -(-cols // 32) * 32
    pitch = -(-width // 128) * 4
    codes = buf[:rows * width].reshape(rows, width).to(torch.int16)
    codes = torch.where(codes > 127, codes - 256, codes).double()
    scales = buf[-(-rows * width // 256) * 256:][:rows * pitch].reshape(rows, pitch).double()
    return (codes * torch.exp2(scales - 127.0).repeat_interleave(32, 1)[:, :width])[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op, dtype = case["op"], _type(case["dtype"])
    if op == "ck":
        return _through_checkpoint(s["x"].double())
    if op == "wgrad":
        dy = s["dy"].double()
        return torch.einsum("to,ti->oi", dy, _held(s["ck"], case["rows"], case["ins"])), dy.sum(0)
    if op == "ln_fwd":
        x = s["x"].double()
        if case["residual"]:
            x += s["other"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = (x - mean[:, None]) * (rstd[:, None] * s["weight"].double()) + s["bias"].double()
        out = [y, mean, rstd] + ([x] if case["residual"] else [])
        if case["ck"]:
            out.append(_through_checkpoint(x.to(dtype).double()))
            if dtype == torch.bfloat16:
                out.append(_through_checkpoint(y.to(dtype).double()))
        return out
    if op == "gelu_fwd":
        z = s["x"].double() + s["bias"].double()
        if case["approx"] == "tanh":
            y = 0.5 * z * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
        else:
            y = 0.5 * z * torch.erfc(-z / 2.0 ** 0.5)
        out = [y]
        if case["ck"]:
            out.append(_through_checkpoint(z))
            if dtype == torch.bfloat16:
                out.append(_through_checkpoint(y.to(dtype).double()))
        return out
    dy = s["dy"].double()
    x = _held(s["ck"], *dy.shape) if case["ck"] else s["x"].double()
    if op == "ln_bwd":
        n, rstd = dy.shape[1], s["rstd"].double()
        h = (x - s["mean"].double()[:, None]) * rstd[:, None]
        wdy = dy * s["weight"].double()
        dx = (n * wdy - wdy.sum(1, keepdim=True) - h * (wdy * h).sum(1, keepdim=True)) * (rstd / n)[:, None]
        if case["residual"]:
            dx = dx + s["other"].double()
        return dx, torch.einsum("td,td->d", dy, h), dy.sum(0)
    if case["approx"] == "tanh":
        t = torch.tanh((2.0 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3))
        d = 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * (2.0 / math.pi) ** 0.5 * (1.0 + 3.0 * 0.044715 * x ** 2)
    else:
        d = 0.5 * torch.erfc(-x / 2.0 ** 0.5) + x * torch.exp(-0.5 * x ** 2) / (2.0 * math.pi) ** 0.5
    dz = dy * d
    return dz, dz.sum(0)
