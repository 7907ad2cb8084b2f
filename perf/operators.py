"""Measured cases of the layer operators in microscaled formats: quantisation to
4 and 8 bits, the product with 4-bit weights, and a layer's forward and backward
pass with its activations kept in 8 bits.

A microscaled row is cut into blocks of 32 values that share one power of two,
2^(c - 127) with c one byte: the smallest one with max |v| <= M 2^s, where M is
the largest value of the elements.  Elements are E2M1 ("mxfp4", M = 6) or E4M3
("mxfp8", M = 448), rounded to the nearest, ties to even; in mxfp8 a value other
than zero is never rounded to zero, so that the sign of a ReLU stays readable.
"""
import math

import torch

own = False

_LARGEST = {"mxfp4": 6.0, "mxfp8": 448.0}
_HIDDEN = 6          # hidden layers between a network's first layer and its head
_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the kept activations of one hidden layer for a 400 x 400 frame of rays
        {"name": "quantize_frame_mxfp8", "op": "quantize", "rows": 160000, "cols": 256, "fmt": "mxfp8", "type": "bf16", "pad": 0},
        # a wide layer's fp32 weights for serving, cut out of a longer row, with a ragged last block
        {"name": "quantize_weights_mxfp4", "op": "quantize", "rows": 2049, "cols": 4100, "fmt": "mxfp4", "type": "fp32", "pad": 12},
        # one token through a wide layer: the weights are read once for a single row
        {"name": "linear_one_token", "op": "linear", "rows": 1, "in": 4096, "out": 4096, "type": "bf16", "out_type": "bf16", "relu": False},
        # a handful of rays through a hidden layer: the smallest call
        {"name": "linear_few_rays", "op": "linear", "rows": 13, "in": 256, "out": 256, "type": "fp32", "out_type": "fp32", "relu": True},
        # a frame of rays through a hidden layer
        {"name": "linear_frame", "op": "linear", "rows": 160000, "in": 256, "out": 256, "type": "bf16", "out_type": "bf16", "relu": True},
        # a long prompt through a wide layer
        {"name": "linear_wide", "op": "linear", "rows": 8192, "in": 4096, "out": 4096, "type": "bf16", "out_type": "bf16", "relu": False},
        # the hidden layers of the shading network for a 400 x 400 frame of four samples per ray, in 4 bits throughout
        {"name": "hidden_layers_frame", "op": "hidden", "rows": 640000, "in": 256, "out": 256, "type": "bf16", "out_type": "bf16", "relu": True},
        # a small batch through the shading head's 283 inputs: odd sizes, odd strides
        {"name": "forward_small_odd", "op": "forward", "rows": 1021, "in": 283, "out": 100, "type": "bf16", "relu": True},
        # a hidden layer's forward pass over a frame of rays, its activations kept in 8 bits
        {"name": "forward_frame", "op": "forward", "rows": 160000, "in": 256, "out": 256, "type": "bf16", "relu": True},
        # the depth head's backward pass over a small batch
        {"name": "backward_small", "op": "backward", "rows": 1000, "in": 256, "out": 128, "type": "bf16", "relu": True},
        # a hidden layer's backward pass over a frame of rays
        {"name": "backward_frame", "op": "backward", "rows": 160000, "in": 256, "out": 256, "type": "bf16", "relu": True},
        # a wide layer's backward pass over a long batch
        {"name": "backward_wide", "op": "backward", "rows": 16384, "in": 2048, "out": 2048, "type": "bf16", "relu": True},
    ]


def _size(rng, lo, hi):
    """A size spread over its logarithm; two in three odd or ragged, one in three a multiple of 32 where it is long enough."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 1 / 3 and v >= 32:
        v -= v % 32
    return min(max(v, lo), hi)


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "hidden", "forward", "backward", "backward"])
    while True:
        if op == "quantize":
            case = {"op": op, "rows": _size(rng, 1, 160000), "cols": _size(rng, 32, 8192), "fmt": rng.choice(["mxfp4", "mxfp8"]),
                    "type": rng.choice(["fp32", "bf16"]), "pad": rng.choice([0, 0, 1, 12])}
        elif op == "hidden":
            wide = 256 if rng.random() < 0.5 else _size(rng, 64, 1024)
            case = {"op": op, "rows": _size(rng, 1, 640000), "in": wide, "out": wide, "type": "bf16", "out_type": "bf16", "relu": True}
        else:
            case = {"op": op, "rows": _size(rng, 1, 160000), "in": _size(rng, 32, 4096), "out": _size(rng, 16, 4096), "type": "bf16",
                    "relu": rng.random() < 0.5}
            if op == "linear":
                case |= {"type": rng.choice(["fp32", "bf16"]), "out_type": rng.choice(["fp32", "bf16"])}
        w = work(case)
        if w["flops"] <= 2.5e11 and w["bytes"] <= 5e8:
            return case


def _width(t):
    return 4 if t == "fp32" else 2


def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        held = n * (0.5 if case["fmt"] == "mxfp4" else 1.0) + n / 32
        # the values read, what holds them written and read back, the values that it stands for written
        return {"bytes": n * _width(case["type"]) + 2 * held + n * 2, "flops": 4.0 * n}
    m, k, n = case["rows"], case["in"], case["out"]
    if case["op"] in ("linear", "hidden"):
        layers = _HIDDEN if case["op"] == "hidden" else 1
        return {"bytes": m * k * _width(case["type"]) + layers * (n * k * (0.5 + 1 / 32) + 4 * n) + m * n * _width(case["out_type"]),
                "flops": 2.0 * m * n * k * layers}
    if case["op"] == "forward":
        # the checkpoint is written, read back and returned as values
        return {"bytes": 2 * m * k + 2 * n * k + 4 * n + 2 * m * n + 2 * m * n * (1 + 1 / 32) + 2 * m * n, "flops": 2.0 * m * n * k}
    return {"bytes": 2 * m * n + m * k * (1 + 1 / 32) + 2 * n * k + 2 * m * k + 4 * n * k + 4 * n, "flops": 4.0 * m * n * k}


# ---------------------------------------------------------------- the formats in plain operations

def _scaled(v, e):
    """v 2^e, exactly: by two factors, each with its exponent written into the type's bits (pow's rounding would move ties)."""
    bits, low, to = (torch.int32, 23, 127) if v.dtype == torch.float32 else (torch.int64, 52, 1023)
    half = e.to(bits) >> 1
    for h in (half, e.to(bits) - half):
        v = v * ((h + to) << low).view(v.dtype)
    return v


def _blocks(x):
    """fp32 values (rows, cols) as (rows, blocks, 32), the last block filled with zeros."""
    rows, cols = x.shape
    n = -(-cols // 32)
    if cols != 32 * n:
        x = torch.cat([x, x.new_zeros(rows, 32 * n - cols)], 1)
    return x.view(rows, n, 32)


def _scale_exp(blocks, fmt):
    """s of each block, (rows, blocks, 1) int32."""
    m, e = torch.frexp(blocks.abs().amax(2, keepdim=True))      # max = m 2^e, m in [1/2, 1)
    if fmt == "mxfp4":
        s = e - 3 + (m > 0.75)       # 6 = 0.75 * 2^3
    else:
        s = e - 9 + (m > 0.875)      # 448 = 0.875 * 2^9
    return torch.where(m == 0, torch.full_like(e, -127), s.clamp(min=-127))


def _elements(v, fmt):
    """|v| (already divided by its scale) rounded to the elements' values."""
    if fmt == "mxfp4":
        step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0))
        return torch.round(v / step) * step
    _, e = torch.frexp(v)
    step = _scaled(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return torch.where(v > 0, (torch.round(v / step) * step).clamp(min=2.0 ** -9), 0.0)


def _rounded(x, fmt):
    """fp32 (rows, cols) -> the values that its microscaled form stands for (fp32), and the scales' bytes."""
    b = _blocks(x)
    s = _scale_exp(b, fmt)
    v = _scaled(_elements(_scaled(b.abs(), -s), fmt), s)
    v = torch.copysign(v, b).reshape(x.shape[0], -1)[:, :x.shape[1]]
    return v, (s[:, :, 0] + 127).to(torch.uint8)


def _packed(x, fmt):
    """fp32 (rows, cols) -> codes and scales as the framework holds them: codes of a row in whole blocks of 32 (two to a byte
    in mxfp4, the even column low), scales in rows of a multiple of 8 bytes."""
    b = _blocks(x)
    s = _scale_exp(b, fmt)
    q = _elements(_scaled(b.abs(), -s), fmt)
    rows, n = b.shape[:2]
    sign = (torch.signbit(b)).to(torch.uint8)
    if fmt == "mxfp4":
        steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
        c = torch.bucketize(q, steps).to(torch.uint8) | (sign << 3)
        c = c.view(rows, n * 16, 2)
        codes = c[:, :, 0] | (c[:, :, 1] << 4)
    else:
        _, e = torch.frexp(q)
        e = (e - 1).clamp(min=-6)
        mant = _scaled(q, 3 - e).to(torch.int32)             # 8..15, below 8 for the smallest ones
        c = torch.where(mant >= 8, ((e + 7) << 3) + mant - 8, mant)
        codes = (c | (sign.to(torch.int32) << 7)).to(torch.uint8).view(rows, n * 32)
    scales = torch.zeros(rows, -(-n // 8) * 8, dtype=torch.uint8, device=x.device)
    scales[:, :n] = (s[:, :, 0] + 127).to(torch.uint8)
    return codes.contiguous(), scales


def _values(codes, scales, cols, fmt, dtype=torch.float32):
    """What codes and scales stand for."""
    if fmt == "mxfp4":
        table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=dtype, device=codes.device)
        c = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1).to(torch.int32)
        v = table[(c & 7).long()]
        v = torch.where(c >= 8, -v, v)
    else:
        c = codes.to(torch.int32)
        e, f = (c >> 3) & 15, c & 7
        mant = torch.where(e > 0, f + 8, f).to(dtype)
        v = _scaled(mant, torch.where(e > 0, e, torch.ones_like(e)) - 10)
        v = torch.where(c >= 128, -v, v)
    s = scales[:, :v.shape[1] // 32].to(torch.int32) - 127
    return _scaled(v.view(v.shape[0], -1, 32), s[:, :, None]).reshape(v.shape[0], -1)[:, :cols]


# ---------------------------------------------------------------- inputs

def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 11)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        x = normal(rows, cols + case["pad"]) * torch.exp2(3 * normal(rows, 1))    # rows of different magnitudes
        if case["fmt"] == "mxfp8":
            x = torch.relu(x)                                                     # activations behind a ReLU
        return {"x": x.to(_TYPES[case["type"]])[:, :cols]}
    m, k, n = case["rows"], case["in"], case["out"]
    bound = math.sqrt(6.0 / k)

    def weights():
        return (2 * torch.rand(n, k, generator=g, device="cuda") - 1) * bound

    if case["op"] in ("linear", "hidden"):
        x = normal(m, k)
        d = {"x": (torch.relu(x) if case["relu"] else x).to(_TYPES[case["type"]])}
        layers = _HIDDEN if case["op"] == "hidden" else 1
        d["w"] = [_packed(weights(), "mxfp4") for _ in range(layers)]
        d["b"] = [0.1 * normal(n) for _ in range(layers)]
        return d
    if case["op"] == "forward":
        return {"x": torch.relu(normal(m, k)).bfloat16(), "w": weights().bfloat16(), "b": 0.1 * normal(n)}
    x = normal(m, k)
    return {"dz": (normal(m, n) / m).bfloat16(), "x": _packed(torch.relu(x) if case["relu"] else x, "mxfp8"), "w": weights().bfloat16()}


_handle = None


def prepare(case, seed):
    global _handle
    state = _inputs(case, seed)
    state["case"] = case
    if own:
        from paper_2103_03231_amd import binding, inputs
        if _handle is None:      # whose device and stream the calls go to: a program keeps one
            _handle = binding.Renderer(binding.Config(), inputs.make_weights(128, 0))
        state |= {"b_": binding, "r": _handle}
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(case, state)


def _run_own(case, st):
    b, r = st["b_"], st["r"]
    op = case["op"]
    if op == "quantize":
        q = r.mx_quantize(st["x"], b.MXFP4 if case["fmt"] == "mxfp4" else b.MXFP8)
        return {"values": r.mx_dequantize(q, torch.bfloat16), "scales": q.scales[:, :-(-case["cols"] // 32)]}
    k, n = case["in"], case["out"]
    if op == "linear":
        w = b.MxTensor(*st["w"][0], k, b.MXFP4)
        return r.mx_linear(st["x"], w, st["b"][0], relu=case["relu"], out=_TYPES[case["out_type"]])
    if op == "hidden":
        ws = [b.MxTensor(*w, k, b.MXFP4) for w in st["w"]]
        h = st["x"]
        for w, bias in zip(ws[:-1], st["b"][:-1]):
            h = r.mx_linear(h, w, bias, relu=True, out=b.MXFP4)
        return r.mx_linear(h, ws[-1], st["b"][-1], relu=True, out=_TYPES[case["out_type"]])
    if op == "forward":
        y, kept = r.train_linear(st["x"], st["w"], st["b"], relu=case["relu"])
        return {"y": y, "kept": r.mx_dequantize(kept, torch.bfloat16)}
    dx, dw, db = r.train_linear_backward(st["dz"], b.MxTensor(*st["x"], k, b.MXFP8), st["w"], relu=case["relu"])
    return {"dx": dx, "dw": dw, "db": db}


def _run_plain(case, st):
    op = case["op"]
    if op == "quantize":
        v, s = _rounded(st["x"].float(), case["fmt"])
        return {"values": v.bfloat16(), "scales": s}
    k = case["in"]
    if op in ("linear", "hidden"):
        h = st["x"].float()
        for (codes, scales), bias in zip(st["w"], st["b"]):
            h = _rounded(h, "mxfp4")[0] @ _values(codes, scales, k, "mxfp4").t() + bias
            h = torch.relu(h) if case["relu"] else h
        return h.to(_TYPES[case["out_type"]])
    if op == "forward":
        z = st["x"].float() @ st["w"].float().t() + st["b"]
        z = torch.relu(z) if case["relu"] else z
        return {"y": z.bfloat16(), "kept": _rounded(z, "mxfp8")[0].bfloat16()}
    dz, x = st["dz"].float(), _values(*st["x"], k, "mxfp8")
    dx = dz @ st["w"].float()
    if case["relu"]:
        dx = torch.where(x != 0, dx, torch.zeros_like(dx))
    return {"dx": dx.bfloat16(), "dw": dz.t() @ x, "db": dz.sum(0)}


# ---------------------------------------------------------------- the same in 64 bits

def _grid(fmt, device):
    """All non-negative values of the elements, in order; a value's place is its code."""
    if fmt == "mxfp4":
        v = [0, .5, 1, 1.5, 2, 3, 4, 6]
    else:
        v = [f * 2.0 ** -9 for f in range(8)] + [(8 + f) * 2.0 ** (e - 10) for e in range(1, 16) for f in range(8)][:-1]
    return torch.tensor(v, dtype=torch.float64, device=device)


def _nearest(x, fmt):
    """fp64 (rows, cols) -> the values of its microscaled form, by search among the elements' values."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    top = x.abs().amax(2, keepdim=True)
    s = torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / _LARGEST[fmt]))
    s = torch.where(top > _LARGEST[fmt] * torch.exp2(s), s + 1, s)             # the logarithm's rounding next to a power of two
    s = torch.where(top <= _LARGEST[fmt] * torch.exp2(s - 1), s - 1, s)
    s = torch.where(top > 0, s.clamp(min=-127), torch.full_like(s, -127))
    scale = torch.exp2(s)
    grid = _grid(fmt, x.device)
    mid = (grid[1:] + grid[:-1]) / 2
    v = x.abs() / scale
    hi = torch.bucketize(v, mid, right=True)           # a tie goes up here
    lo = torch.bucketize(v, mid)                       # and down here
    code = torch.where((hi != lo) & (hi % 2 == 1), lo, hi)
    if fmt == "mxfp8":
        code = torch.where((v > 0) & (code == 0), torch.ones_like(code), code)
    out = torch.copysign(grid[code] * scale, x).view(rows, -1)[:, :cols]
    return out, (s[:, :, 0] + 127).to(torch.uint8)


def exact(case, seed):
    d = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        v, s = _nearest(d["x"].double(), case["fmt"])
        return {"values": v, "scales": s}
    k = case["in"]
    if op in ("linear", "hidden"):
        h = d["x"].double()
        for (codes, scales), bias in zip(d["w"], d["b"]):
            h = torch.addmm(bias.double(), _nearest(h, "mxfp4")[0], _values(codes, scales, k, "mxfp4", torch.float64).t())
            h = h.clamp(min=0) if case["relu"] else h
        return h
    if op == "forward":
        z = torch.addmm(d["b"].double(), d["x"].double(), d["w"].double().t())
        z = z.clamp(min=0) if case["relu"] else z
        return {"y": z, "kept": _nearest(z, "mxfp8")[0]}
    dz, x = d["dz"].double(), _values(*d["x"], k, "mxfp8", torch.float64)
    dx = torch.mm(dz, d["w"].double())
    return {"dx": dx * (x != 0) if case["relu"] else dx, "dw": torch.mm(dz.t(), x), "db": dz.sum(0)}
