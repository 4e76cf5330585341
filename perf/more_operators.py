"""Operators of the denoising step in 8-bit floating point (e4m3), as cases that can be timed and checked.

  norm      dc_rms_norm_f8: a sub-block's output added to the residual stream, RMS norm of the sum, and the
            normed rows as e4m3 codes with a scale to 128 features;
  quantize  dc_quantize_f8: rows as e4m3 codes with a scale to 128 features (activations), or to
            128 x 128 values (weights);
  linear    dc_linear_f8: the product of such rows and weights, with a block's epilogues;
  feed      a block's MLP of the three: norm, up with GELU, codes of the hidden rows, down with the gated residual.

Where `own` is false `run` computes the same in elementary torch operations in fp32.  Model shapes are the
framework's own (12 blocks of 1,152, 30 of 1,920) or generic.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
BLOCK = 128                     # features that share a scale; weights: 128 x 128 values
TOP = 448.0                     # largest e4m3 number
F8 = torch.float8_e4m3fn


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def _norm(name, rows, cols, x, residual, out, weight=True):
    """residual: its type, or "" for none; out: the written sum's type, or "" for none."""
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "x": x, "residual": residual, "out": out,
            "weight": weight, "major": "block"}


def _quantize(name, rows, cols, x, block_rows):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "x": x, "block_rows": block_rows,
            "major": "block"}


def _linear(name, m, k, n, out, **more):
    c = {"name": name, "op": "linear", "m": m, "k": k, "n": n, "out": out, "bias": True, "gelu": False,
         "residual": False, "gate": False, "major": "block"}
    c.update(more)
    return c


def listed():
    return [
        # One conditioning row through a norm: the smallest call, latency.
        _norm("norm 1x1920", 1, 1920, "bf16", "f32", "f32"),
        # A block's norm of the 12-block model on its fp32 residual stream.
        _norm("norm 3704x1152", 3704, 1152, "bf16", "f32", "f32"),
        # The 30-block model's at full length: twice per block in every refresh step.
        _norm("norm 17776x1920", 17776, 1920, "bf16", "f32", "f32"),
        # The hidden rows of the 30-block model's MLP, between its two products.
        _quantize("quantize 17776x7680", 17776, 7680, "bf16", 1),
        # A weight matrix taken from bf16 when a model is loaded.
        _quantize("quantize weight 7680x1920", 7680, 1920, "bf16", 128),
        # One conditioning row through MLP down: bound by the weights and by latency.
        _linear("linear 1x7680x1920", 1, 7680, 1920, "f32"),
        # The conditioning rows of a 50-step sample through the modulation projection.
        _linear("linear 50x1920x11520", 50, 1920, 11520, "f32"),
        # The fused QKV product of a short low-resolution clip: 1,556 tokens, a ragged last tile.
        _linear("linear 1556x1920x5760", 1556, 1920, 5760, "bf16"),
        # MLP up with GELU of the 30-block model at full length.
        _linear("linear 17776x1920x7680", 17776, 1920, 7680, "bf16", gelu=True),
        # MLP down with the gated residual at full length: the longest sums.
        _linear("linear 17776x7680x1920", 17776, 7680, 1920, "f32", residual=True, gate=True),
        # Rows and channels that no tile divides, a last block of 72 features, rows' scales side by side.
        _linear("linear 1001x1096x1003", 1001, 1096, 1003, "f32", major="row"),
        # The whole MLP of the 12-block model's clip, on a residual stream in bf16.
        {"name": "feed 3704x1152x4608", "op": "feed", "m": 3704, "d": 1152, "f": 4608, "major": "block"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A model's width half of the time (whole blocks), any other half of the time."""
    n = _log_int(rng, lo, hi)
    return BLOCK * -(-n // BLOCK) if rng.random() < 0.5 else n


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm", "quantize", "quantize", "linear", "linear", "linear", "feed"])
        rows = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 64, 17776), _log_int(rng, 64, 17776)])
        types = ["f32", "bf16"]
        if op == "norm":
            residual = rng.choice(["f32", "bf16", ""])
            c = _norm("", rows, _width(rng, 32, 8192), rng.choice(types), residual,
                      rng.choice(types) if residual else "", rng.random() < 0.8)
        elif op == "quantize":
            c = _quantize("", rows, _width(rng, 32, 8192), rng.choice(types), rng.choice([1, 1, 128]))
        elif op == "linear":
            c = _linear("", rows, _width(rng, 64, 7680), _width(rng, 32, 11520), rng.choice(types),
                        bias=rng.random() < 0.8)
            kind = rng.choice(["plain", "gelu", "residual", "gated"])
            c["gelu"], c["residual"], c["gate"] = kind == "gelu", kind in ("residual", "gated"), kind == "gated"
        else:
            d = BLOCK * _log_int(rng, 2, 16)
            c = {"name": "", "op": "feed", "m": rows, "d": d, "f": d * rng.choice([2, 3, 4])}
        c["major"] = rng.choice(["block", "block", "row"])
        del c["name"]
        w = work(c)
        most = [work(q) for q in listed() if q["op"] == op]
        if all(w[k] <= max(q[k] for q in most) for k in ("bytes", "flops")):
            return c


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
class _Draws:
    """Seeded normal draws on the GPU, in the order they are asked for."""

    def __init__(self, seed):
        self.g = torch.Generator(DEV)
        self.g.manual_seed(seed)

    def __call__(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device=DEV) * std


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _blocks(n):
    return -(-n // BLOCK)


def _scales(rows, blocks, major):
    """An empty [rows, blocks] tensor: a block's scales side by side ("block"), or a row's."""
    if major == "block":
        return torch.empty((blocks, rows), device=DEV).t()
    return torch.empty((rows, blocks), device=DEV)


def _codes(rows, cols):
    return torch.zeros((rows, BLOCK * _blocks(cols)), dtype=torch.uint8, device=DEV).view(F8)


def _activations(rnd, rows, cols):
    """Rows and features of different size, and a few large features, as a network's are."""
    x = rnd(rows, cols)
    x *= torch.exp(0.5 * rnd(rows, 1))
    x *= torch.exp(0.7 * rnd(cols))
    x[:, ::97] *= 8
    return x


def _weights(rnd, n, k):
    """A quantised [n, k] matrix: its codes, padded, and its scales."""
    codes, scale = _quantized(rnd(n, k, std=0.02) * torch.exp(0.3 * rnd(n, 1)), 128)
    return codes, scale


def prepare(case, seed):
    c, rnd = case, _Draws(seed)
    s = {"case": c}
    op = c["op"]
    if op == "norm":
        s["x"] = (0.3 * _activations(rnd, c["rows"], c["cols"])).to(_type(c["x"]))
        s["residual"] = rnd(c["rows"], c["cols"]).to(_type(c["residual"])) if c["residual"] else None
        s["out"] = torch.zeros((c["rows"], c["cols"]), dtype=_type(c["out"]), device=DEV) if c["out"] else None
        s["weight"] = 1 + rnd(c["cols"], std=0.2) if c["weight"] else None
        s["q"] = _codes(c["rows"], c["cols"])
        s["scale"] = _scales(c["rows"], _blocks(c["cols"]), c["major"])
    elif op == "quantize":
        s["x"] = _activations(rnd, c["rows"], c["cols"]).to(_type(c["x"]))
        s["q"] = _codes(c["rows"], c["cols"])
        rows = c["rows"] if c["block_rows"] == 1 else _blocks(c["rows"])
        s["scale"] = _scales(rows, _blocks(c["cols"]), c["major"])
    elif op == "linear":
        m, k, n = c["m"], c["k"], c["n"]
        s["x"], scale = _quantized(_activations(rnd, m, k), 1)
        s["x_scale"] = _scales(m, _blocks(k), c["major"]).copy_(scale)
        s["w"], s["w_scale"] = _weights(rnd, n, k)
        s["bias"] = rnd(n, std=0.02) if c["bias"] else None
        s["gate"] = rnd(n, std=0.3) if c["gate"] else None
        s["residual"] = rnd(m, n, std=0.5).to(_type(c["out"])) if c["residual"] else None
        s["out"] = torch.zeros((m, n), dtype=_type(c["out"]), device=DEV)
    else:
        m, d, f = c["m"], c["d"], c["f"]
        s["x"] = (0.3 * _activations(rnd, m, d)).to(torch.bfloat16)
        s["residual"] = rnd(m, d).to(torch.bfloat16)
        s["weight"] = 1 + rnd(d, std=0.2)
        s["up"], s["up_scale"] = _weights(rnd, f, d)
        s["down"], s["down_scale"] = _weights(rnd, d, f)
        s["up_bias"], s["down_bias"] = rnd(f, std=0.02), rnd(d, std=0.02)
        s["gate"] = rnd(d, std=0.3)
        s["h"], s["y"] = (torch.zeros((m, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        s["hidden"] = torch.zeros((m, f), dtype=torch.bfloat16, device=DEV)
        s["q"], s["hidden_q"] = _codes(m, d), _codes(m, f)
        s["scale"], s["hidden_scale"] = (_scales(m, _blocks(w), c["major"]) for w in (d, f))
    return s


# ----------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------
def _over(a, levels):
    """a / levels, one IEEE division (a Python number would be turned into a product)."""
    return a / torch.full_like(a, levels)


def _quantized(x, block_rows):
    """e4m3 codes of fp32 rows, padded with zeros to whole blocks, and the scales of the blocks."""
    rows, cols = x.shape
    r, b = -(-rows // block_rows), _blocks(cols)
    v = torch.zeros((r * block_rows, b * BLOCK), device=x.device)
    v[:rows, :cols] = x
    v = v.view(r, block_rows, b, BLOCK)
    scale = _over(v.abs().amax((1, 3)), TOP)
    step = scale[:, None, :, None]
    code = torch.where(step > 0, (v / step).clamp(-TOP, TOP), torch.zeros_like(v))
    return code.view(r * block_rows, b * BLOCK)[:rows].to(F8), scale


def _values(codes, scale, block_rows):
    """The numbers that codes with these scales stand for, in fp32, padding included."""
    rows = codes.shape[0]
    step = scale.repeat_interleave(block_rows, 0)[:rows] if block_rows > 1 else scale
    return codes.float() * step.repeat_interleave(BLOCK, 1)


def _gelu(z):
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def _plain_norm(x, residual, weight, out):
    """codes and scales of the normed sum, and the sum in out's type (None: not wanted)."""
    h = x.float()
    if residual is not None:
        h = h + residual.float()
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    if weight is not None:
        y = y * weight
    q, scale = _quantized(y, 1)
    return q, scale, None if out is None else h.to(out)


def _plain_linear(x, x_scale, w, w_scale, out, bias, gelu, gate, residual):
    y = _values(x, x_scale, 1) @ _values(w, w_scale, 128).t()
    if bias is not None:
        y = y + bias
    if gelu:
        y = _gelu(y)
    if gate is not None:
        y = gate * y
    if residual is not None:
        y = residual.float() + y
    return y.to(out)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        q, scale, h = _plain_norm(s["x"], s["residual"], s["weight"], _type(c["out"]) if c["out"] else None)
        return {"q": q, "scale": scale, "h": h}
    if op == "quantize":
        q, scale = _quantized(s["x"].float(), c["block_rows"])
        return {"q": q, "scale": scale}
    if op == "linear":
        return {"out": _plain_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], _type(c["out"]), s["bias"], c["gelu"],
                                     s["gate"], s["residual"])}
    q, scale, h = _plain_norm(s["x"], s["residual"], s["weight"], torch.bfloat16)
    hidden = _plain_linear(q, scale, s["up"], s["up_scale"], torch.bfloat16, s["up_bias"], True, None, None)
    q, scale = _quantized(hidden.float(), 1)
    y = _plain_linear(q, scale, s["down"], s["down_scale"], torch.bfloat16, s["down_bias"], False, s["gate"], h)
    return {"h": h, "y": y}


# ----------------------------------------------------------------------------
# the framework's calls
# ----------------------------------------------------------------------------
def _own(s):
    from paper_2608_16354_amd import api
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        api.dc_rms_norm_f8(s["x"], s["q"], s["scale"], weight=s["weight"], eps=EPS, residual=s["residual"], out=s["out"])
        return {"q": s["q"], "scale": s["scale"], "h": s["out"]}
    if op == "quantize":
        api.dc_quantize_f8(s["x"], s["q"], s["scale"], block_rows=c["block_rows"])
        return {"q": s["q"], "scale": s["scale"]}
    if op == "linear":
        api.dc_linear_f8(s["x"], s["x_scale"], s["w"], s["w_scale"], s["out"], bias=s["bias"], gelu=c["gelu"],
                         gate=s["gate"], residual=s["residual"])
        return {"out": s["out"]}
    api.dc_rms_norm_f8(s["x"], s["q"], s["scale"], weight=s["weight"], eps=EPS, residual=s["residual"], out=s["h"])
    api.dc_linear_f8(s["q"], s["scale"], s["up"], s["up_scale"], s["hidden"], bias=s["up_bias"], gelu=True)
    api.dc_quantize_f8(s["hidden"], s["hidden_q"], s["hidden_scale"])
    api.dc_linear_f8(s["hidden_q"], s["hidden_scale"], s["down"], s["down_scale"], s["y"], bias=s["down_bias"],
                     gate=s["gate"], residual=s["h"])
    return {"h": s["h"], "y": s["y"]}


def run(state):
    return _own(state) if own else _plain(state)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    c = case
    size = {"": 0, "f32": 4, "bf16": 2}
    if c["op"] == "norm":
        n = c["rows"] * c["cols"]
        moved = n * (size[c["x"]] + size[c["residual"]] + size[c["out"]] + 1)
        return {"bytes": moved + 4 * c["rows"] * _blocks(c["cols"]) + 4 * c["cols"] * c["weight"], "flops": 8 * n}
    if c["op"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (size[c["x"]] + 1) + 4 * _blocks(c["cols"]) * -(-c["rows"] // c["block_rows"]),
                "flops": 3 * n}
    if c["op"] == "linear":
        m, k, n = c["m"], c["k"], c["n"]
        moved = m * k + n * k + 4 * _blocks(k) * (m + _blocks(n)) + m * n * size[c["out"]] * (1 + c["residual"])
        return {"bytes": moved + 4 * n * (c["bias"] + c["gate"]), "flops": 2 * m * k * n}
    m, d, f = c["m"], c["d"], c["f"]
    moved = 8 * m * d + 2 * d * f + 8 * _blocks(d) * _blocks(f) + 4 * (3 * d + f)
    return {"bytes": moved, "flops": 4 * m * d * f}


# ----------------------------------------------------------------------------
# the same from the definitions in 64 bits
# ----------------------------------------------------------------------------
def _e4m3(v):
    """The nearest number of three fraction bits and exponents from -6 on, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.special.round(v / step) * step


def _exact_codes(v, block_rows=1):
    """Code numbers and scales, block by block; scales and the quotients that are rounded are fp32 numbers."""
    rows, cols = v.shape
    codes = torch.zeros((rows, BLOCK * _blocks(cols)), dtype=torch.float64, device=DEV)
    scale = torch.zeros((-(-rows // block_rows), _blocks(cols)), dtype=torch.float64, device=DEV)
    for j in range(_blocks(cols)):
        part = v[:, BLOCK * j: BLOCK * (j + 1)]
        top = part.abs().max(dim=1).values
        if block_rows > 1:
            top = torch.stack([t.max() for t in top.split(block_rows)])
        scale[:, j] = (top / 448).float().double()
        step = scale[:, j].repeat_interleave(block_rows)[:rows, None]
        code = _e4m3((part / step).float().double())
        codes[:, BLOCK * j: BLOCK * j + part.shape[1]] = torch.where(step > 0, code, 0.0)
    return codes, scale


def _exact_norm(s):
    h = s["x"].double()
    if s["residual"] is not None:
        h += s["residual"].double()
    y = h * (h.square().sum(1, keepdim=True) / h.shape[1] + EPS).rsqrt()
    if s["weight"] is not None:
        y *= s["weight"].double()
    return h, y


def _exact_linear(x, x_scale, w, w_scale, bias, gelu, gate, residual):
    m, n, k = x.shape[0], w.shape[0], x.shape[1]
    out = torch.empty((m, n), dtype=torch.float64, device=DEV)
    wide = w.double()
    for j in range(w_scale.shape[0]):
        wide[BLOCK * j: BLOCK * (j + 1)].view(-1, k // BLOCK, BLOCK).mul_(w_scale[j].double()[:, None])
    for r in range(0, m, 4096):
        rows = x[r: r + 4096].double().view(-1, k // BLOCK, BLOCK) * x_scale[r: r + 4096].double()[:, :, None]
        z = rows.view(-1, k) @ wide.t()
        if bias is not None:
            z += bias.double()
        if gelu:
            z = z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
        if gate is not None:
            z *= gate.double()
        out[r: r + 4096] = z if residual is None else residual[r: r + 4096].double() + z
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c, op = case, case["op"]
    if op == "norm":
        h, y = _exact_norm(s)
        q, scale = _exact_codes(y)
        return {"q": q, "scale": scale, "h": h if c["out"] else None}
    if op == "quantize":
        q, scale = _exact_codes(s["x"].double(), c["block_rows"])
        return {"q": q, "scale": scale}
    if op == "linear":
        return {"out": _exact_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], c["gelu"], s["gate"],
                                     s["residual"])}
    h, y = _exact_norm(s)
    q, scale = _exact_codes(y)
    hidden = _exact_linear(q, scale, s["up"], s["up_scale"], s["up_bias"], True, None, None).to(torch.bfloat16)
    q, scale = _exact_codes(hidden.double())
    # the stored sum is a bf16 number, and that is what the second product adds to
    y = _exact_linear(q, scale, s["down"], s["down_scale"], s["down_bias"], False, s["gate"], h.to(torch.bfloat16))
    return {"h": h, "y": y}
