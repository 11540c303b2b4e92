"""What the speed of the masked layer's operators is measured on: single calls as a program makes them that retrains or
serves a model whose projections carry transposable masks.

The operators work on scaled matrices: 8-bit floating point values (e4m3, row-major, rows padded with zeros to a multiple of
128) with a power of two (e8m0) for each row and 128 columns, kept as [column block][row] with 16-byte aligned blocks.  A case
is a dict of plain values:
  op "norm"      residual addition, root-mean-square norm, 8-bit output: h = x + r, y = g h / sqrt(mean(h^2) + eps); rows, cols,
                 dtype, residual; gain: type of g; keep_y: y comes back in the input's type too (the backward pass needs it);
                 backward: from h, g and dL/dy, and with residual the gradient that reaches h past the norm, dL/dh and dL/dg
  op "quantize"  a matrix into 8 bits: rows, cols, dtype; ld: columns of the matrix it is a column range of (0: all of it);
                 square: one scale for 128 x 128 (weights), otherwise for 128 values along the row (tokens, gradients);
                 masked: a 0/1 mask applies; ways: "rows", "columns" (the transposed matrix) or "both"
  op "product"   a b^T of two scaled matrices: m, n, k; weights: b has 128 x 128 scales (a layer's forward pass or input
                 gradient), otherwise both have scales along k (a weight gradient); masked: the result is kept where a 0/1 mask
                 says so.  The result is bf16: 8-bit operands are 2^-4 off, and the matrix cores line the products of 8-bit
                 values up with 16 bits below the largest of them, 1.6e-5 of the result for normal operands
  op "clip"      the global norm of all gradients of a model, and the gradients scaled down to a largest norm: layers, width,
                 inner, kv (columns of keys and values), dtype; active: whether the norm is above the largest
"""
from __future__ import annotations

import torch

own = False

EPS = 1e-5
BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, rows, cols, dtype="bf16", residual=True, gain="bf16", keep_y=False, backward=False):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual, "gain": gain,
            "keep_y": keep_y, "backward": backward}


def _quantize(name, rows, cols, dtype="bf16", ld=0, square=False, masked=False, ways="both"):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "ld": ld, "square": square,
            "masked": masked, "ways": ways}


def _product(name, m, n, k, weights=True, masked=False):
    return {"name": name, "op": "product", "m": m, "n": n, "k": k, "weights": weights, "masked": masked}


def _clip(name, layers, width, inner, kv, dtype="bf16", active=True):
    return {"name": name, "op": "clip", "layers": layers, "width": width, "inner": inner, "kv": kv, "dtype": dtype, "active": active}


def listed():
    return [
        # one token of a sequence that is being answered, at the width of an 8B model: the smallest call
        _norm("norm_1x4096", 1, 4096),
        # the tokens of a training step of a 70B model: the norm's output is kept for the weight gradient
        _norm("norm_4096x8192_keep", 4096, 8192, keep_y=True),
        # the backward pass over an odd number of tokens, in single precision
        _norm("norm_backward_2047x4096_f32", 2047, 4096, dtype="f32", gain="f32", backward=True),
        # the key projection of an 8B model with its mask, for the forward and the backward product
        _quantize("weights_1024x4096", 1024, 4096, square=True, masked=True),
        # activations or gradients of a ragged batch, along the tokens for the weight gradient too
        _quantize("tokens_1072x2928", 1072, 2928),
        # the largest projection of a 70B model from its single-precision weights: the largest call by bytes
        _quantize("weights_28672x8192_f32", 28672, 8192, dtype="f32", square=True, masked=True),
        # one token through an MLP projection of an 8B model: all of the weights for one row
        _product("product_1x14336x4096", 1, 14336, 4096),
        # a batch of sequences that are being answered, through the projection back
        _product("product_48x4096x14336", 48, 4096, 14336),
        # a prompt of odd length through that projection
        _product("product_1999x4096x14336", 1999, 4096, 14336),
        # the weight gradient of the MLP projection over the tokens of a training step: the largest call by operations
        _product("product_14336x4096x8192_masked", 14336, 4096, 8192, weights=False, masked=True),
        # the gradients of a small model: many small tensors
        _clip("clip_8_layers_of_512", 8, 512, 1431, 128, dtype="f32"),
        # one decoder layer of an 8B model
        _clip("clip_layer_of_4096", 1, 4096, 14336, 1024),
    ]


def _size(rng, low, high):
    """A whole number from 2^low to 2^high, spread over its logarithm; a third of them multiples of 16."""
    n = max(1, int(2.0 ** rng.uniform(low, high)))
    return n if n < 32 or rng.random() < 0.67 else n // 16 * 16


def draw(rng):
    op = rng.choice(("norm", "quantize", "product", "product", "clip"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        cols = _size(rng, 7, 14)
        rows = min(_size(rng, 0, 13), (1 << 25) // cols)
        c = _norm("", rows, cols, dtype, rng.random() < 0.7, rng.choice((dtype, "f32")), rng.random() < 0.4, rng.random() < 0.4)
        if c["backward"]:
            c["keep_y"] = False
    elif op == "quantize":
        square, cols = rng.random() < 0.5, _size(rng, 7, 14)
        rows = min(_size(rng, 7 if square else 0, 15), (1 << 27) // cols)
        c = _quantize("", rows, cols, dtype, cols + rng.choice((8, 24, 513)) if rng.random() < 0.25 else 0, square,
                      square and rng.random() < 0.7, rng.choice(("rows", "columns", "both", "both")))
    elif op == "product":
        weights = rng.random() < 0.7
        n, k = _size(rng, 8, 14.5), _size(rng, 7, 14)
        m = max(1, min(_size(rng, 0, 13) if weights else _size(rng, 8, 13), (1 << 38) // (n * k)))
        c = _product("", m, n, k, weights, not weights and rng.random() < 0.6)
    else:
        width = _size(rng, 6, 12)
        inner, kv = int(width * rng.uniform(2, 4)), max(1, int(width * rng.uniform(0.1, 1)))
        per_layer = 2 * width * width + 2 * kv * width + 3 * width * inner
        layers = max(1, min(_size(rng, 0, 5), (1 << 27) // per_layer))
        c = _clip("", layers, width, inner, kv, dtype, rng.random() < 0.8)
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _round_up(n, to):
    return -(-n // to) * to


def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _activations(gen, rows, cols):
    """Tokens as a layer sees them: a few columns are much larger than most."""
    return _normal(gen, rows, cols).mul_(torch.empty(cols, device="cuda").log_normal_(0.0, 0.7, generator=gen))


def _mask(gen, rows, cols):
    """8 of every 16 in rows and columns, in an order of its own for each block."""
    r, c = _round_up(rows, 16), _round_up(cols, 16)
    shift = torch.randint(0, 16, (r // 16, c // 16), device="cuda", generator=gen).repeat_interleave(16, 0).repeat_interleave(16, 1)
    at = torch.arange(r, device="cuda")[:, None] + torch.arange(c, device="cuda") + shift
    return (at % 16 < 8).to(torch.uint8)[:rows, :cols].contiguous()


def _scaled(x, square):
    """(values, scales) of a matrix as a program holds it that was handed 8-bit weights or tokens."""
    values, scales = _plain_quantize(x, square)
    rows = scales.shape[1]
    padded = torch.zeros(scales.shape[0], _round_up(rows, 16), dtype=torch.uint8, device="cuda")
    padded[:, :rows] = scales.view(torch.uint8)
    return values, padded.view(torch.float8_e8m0fnu)[:, :rows]


def _tensors(case):
    """Shapes of a model's gradients: the seven projections and the two norms of each layer."""
    w, f, kv = case["width"], case["inner"], case["kv"]
    return [(w, w), (kv, w), (kv, w), (w, w), (f, w), (f, w), (w, f), (w,), (w,)] * case["layers"]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "norm":
        rows, cols, dtype = case["rows"], case["cols"], TYPES[case["dtype"]]
        s["x"] = _activations(gen, rows, cols).to(dtype)
        s["gain"] = (1.0 + 0.2 * _normal(gen, cols)).to(TYPES[case["gain"]])
        s["past"] = _normal(gen, rows, cols).to(dtype) if case["residual"] else None
        s["dy"] = (1e-3 * _normal(gen, rows, cols)).to(dtype) if case["backward"] else None
        if case["backward"] and case["residual"]:
            s["past"] = (1e-3 * s["past"].float()).to(dtype)
    elif case["op"] == "quantize":
        rows, cols, ld = case["rows"], case["cols"], case["ld"] or case["cols"]
        x = _normal(gen, rows, ld).mul_(0.02) if case["square"] else _activations(gen, rows, ld)
        at = (ld - cols) // 16 * 8
        s["x"] = x.to(TYPES[case["dtype"]])[:, at:at + cols]
        s["mask"] = _mask(gen, rows, cols) if case["masked"] else None
    elif case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"] = _scaled(_activations(gen, m, k) if case["weights"] else 1e-3 * _normal(gen, m, k), False)
        if case["weights"]:
            s["b"] = _scaled(0.02 * _normal(gen, n, k) * _mask(gen, n, k), True)
        else:
            s["b"] = _scaled(_activations(gen, k, n).t().contiguous(), False)
        s["mask"] = _mask(gen, m, n) if case["masked"] else None
    else:
        s["grads"] = [(1e-3 * _normal(gen, *shape)).to(TYPES[case["dtype"]]) for shape in _tensors(case)]
        count = sum(g.numel() for g in s["grads"])
        # where each of them begins in one buffer of all, as a data-parallel program keeps them (the pieces 64 elements apart)
        s["begin"] = [0]
        for g in s["grads"]:
            s["begin"].append(s["begin"][-1] + _round_up(g.numel(), 64))
        s["largest"] = (0.1 if case["active"] else 10.0) * 1e-3 * count ** 0.5
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _plan(s)
    return s


def _plan(s):
    """The outputs, the workspace and the description of the call, which a program keeps from step to step."""
    from paper_2505_23949_amd import layer

    case = s["case"]
    if case["op"] == "norm":
        rows, cols = s["x"].shape
        if case["backward"]:
            s["out"] = {"dh": torch.empty_like(s["x"]), "dgain": torch.empty(cols, device="cuda")}
            s["problem"] = layer.make_norm_backward(s["x"], s["gain"], EPS, s["dy"], dh=s["out"]["dh"], dgain=s["out"]["dgain"],
                                                    dsum=s["past"])
            s["work"] = torch.empty(layer.tsenor_norm_backward_workspace_bytes(s["problem"]), dtype=torch.uint8, device="cuda")
            return
        y8 = layer.empty_scaled(rows, cols, "cuda")
        s["out"] = {"values": y8.values, "scales": y8.scales[:, :rows]}
        if case["residual"]:
            s["out"]["sum"] = torch.empty_like(s["x"])
        if case["keep_y"]:
            s["out"]["y"] = torch.empty_like(s["x"])
        s["problem"] = layer.make_norm(s["x"], s["gain"], EPS, residual=s["past"], out=y8, sum_out=s["out"].get("sum"),
                                       y_out=s["out"].get("y"))
    elif case["op"] == "quantize":
        rows, cols = s["x"].shape
        s["out"], ways = {}, {}
        if case["ways"] != "columns":
            ways["out"] = q = layer.empty_scaled(rows, cols, "cuda")
            s["out"].update(values=q.values, scales=q.scales[:, :rows])
        if case["ways"] != "rows":
            ways["out_t"] = q = layer.empty_scaled(cols, rows, "cuda")
            s["out"].update(values_t=q.values, scales_t=q.scales[:, :cols])
        s["problem"] = layer.make_quantize(s["x"], mask=s["mask"], square=case["square"], **ways)
    elif case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s["out"] = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        a, b = (layer.scaled_matrix(values, scales, k) for values, scales in (s["a"], s["b"]))
        s["problem"] = layer.make_product(a, b, out=s["out"], mask=s["mask"])
        s["work"] = torch.empty(layer.tsenor_product_workspace_bytes(s["problem"]), dtype=torch.uint8, device="cuda")
    else:
        s["out"] = {"grads": torch.zeros(s["begin"][-1], dtype=TYPES[case["dtype"]], device="cuda"), "norm": torch.empty(2, device="cuda")}
        pieces = [s["out"]["grads"][at:at + g.numel()].view(g.shape) for at, g in zip(s["begin"], s["grads"])]
        s["problem"] = layer.make_clip(s["grads"], s["largest"], out=pieces, norm_out=s["out"]["norm"])
        s["work"] = torch.empty(layer.tsenor_clip_workspace_bytes(s["problem"]), dtype=torch.uint8, device="cuda")


def _joined(grads):
    """One buffer of all tensors, zeros between them."""
    return torch.cat([torch.nn.functional.pad(g.reshape(-1), (0, -g.numel() % 64)) for g in grads])


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2505_23949_amd import layer

    op = s["case"]["op"]
    if op == "quantize":
        layer.tsenor_quantize(s["problem"])
    elif op == "product":
        layer.tsenor_product(s["problem"], s["work"])
    elif op == "clip":
        layer.tsenor_clip(s["problem"], s["work"])
    elif s["case"]["backward"]:
        layer.tsenor_norm_backward(s["problem"], s["work"])
    else:
        layer.tsenor_norm(s["problem"])
    return s["out"]


# ---- the operators in plain torch, 32 bits -------------------------------------------------------------------------------

def _plain_quantize(x, square):
    rows, cols = x.shape
    padded = torch.zeros(_round_up(rows, BLOCK) if square else rows, _round_up(cols, BLOCK), device=x.device)
    padded[:rows, :cols] = x
    blocks = padded.view(-1, BLOCK if square else 1, padded.shape[1] // BLOCK, BLOCK)
    largest = blocks.abs().amax((1, 3), keepdim=True)
    mantissa, exponent = torch.frexp(largest)
    exponent = (exponent - 9 + (mantissa > 0.875)).clamp(-126, 127)  # the largest 8-bit value is 448 = 0.875 * 2^9
    exponent = torch.where(largest == 0, 0, exponent)
    values = torch.ldexp(blocks, -exponent).reshape(padded.shape)[:rows].to(torch.float8_e4m3fn)
    scales = (exponent + 127).to(torch.uint8).expand(-1, blocks.shape[1], -1, 1).reshape(padded.shape[0], -1)[:rows]
    return values, scales.t().contiguous().view(torch.float8_e8m0fnu)


def _plain_values(q):
    values, scales = q
    exponent = scales.view(torch.uint8).t().to(torch.int32) - 127
    return torch.ldexp(values.float().view(values.shape[0], -1, BLOCK), exponent[:, :, None]).view(values.shape)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "norm":
        gain = s["gain"].float()
        if case["backward"]:
            h, dy = s["x"].float(), s["dy"].float()
            c = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
            a = gain * dy
            dh = c * a - h * (c * c * c) * (a * h).mean(1, keepdim=True)
            if s["past"] is not None:
                dh = dh + s["past"].float()
            return {"dh": dh.to(s["x"].dtype), "dgain": (dy * h * c).sum(0)}
        out, h = {}, s["x"]
        if s["past"] is not None:
            h = out["sum"] = (h.float() + s["past"].float()).to(h.dtype)
        h = h.float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * gain
        if case["keep_y"]:
            out["y"] = y.to(s["x"].dtype)
        out["values"], out["scales"] = _plain_quantize(y, False)
        return out
    if case["op"] == "quantize":
        x = s["x"].float()
        if s["mask"] is not None:
            x = torch.where(s["mask"] != 0, x, 0.0)
        out = {}
        if case["ways"] != "columns":
            out["values"], out["scales"] = _plain_quantize(x, case["square"])
        if case["ways"] != "rows":
            out["values_t"], out["scales_t"] = _plain_quantize(x.t(), case["square"])
        return out
    if case["op"] == "product":
        out = _plain_values(s["a"]) @ _plain_values(s["b"]).t()
        if s["mask"] is not None:
            out = torch.where(s["mask"] != 0, out, 0.0)
        return out.to(torch.bfloat16)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.where(norm > s["largest"], s["largest"] / norm, 1.0)
    return {"grads": _joined([(g.float() * factor).to(g.dtype) for g in s["grads"]]), "norm": torch.stack([norm, factor])}


# ---- bytes and operations ------------------------------------------------------------------------------------------------

def _scaled_bytes(rows, cols):
    return rows * (cols + -(-cols // BLOCK))


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "norm":
        rows, cols, b = case["rows"], case["cols"], size[case["dtype"]]
        one = rows * cols * b
        if case["backward"]:
            return {"bytes": (4 if case["residual"] else 3) * one + cols * (size[case["gain"]] + 4), "flops": 11 * rows * cols}
        return {"bytes": one * (1 + 2 * case["residual"] + case["keep_y"]) + cols * size[case["gain"]] + _scaled_bytes(rows, cols),
                "flops": 6 * rows * cols}
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        nbytes = rows * cols * (size[case["dtype"]] + case["masked"])
        if case["ways"] != "columns":
            nbytes += _scaled_bytes(rows, cols)
        if case["ways"] != "rows":
            nbytes += _scaled_bytes(cols, rows)
        return {"bytes": nbytes, "flops": 2 * rows * cols}
    if case["op"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": _scaled_bytes(m, k) + _scaled_bytes(n, k) + m * n * (2 + case["masked"]), "flops": 2 * m * n * k}
    count = 0
    for shape in _tensors(case):
        count += shape[0] * (shape[1] if len(shape) > 1 else 1)
    return {"bytes": 2 * count * size[case["dtype"]] + 8, "flops": 3 * count}


# ---- the definitions, 64 bits ---------------------------------------------------------------------------------------------

def _exact_scaled(x, square):
    """Values and scales of x in 64 bits: the nearest multiples of the 8-bit format's step, ties to even."""
    rows, cols = x.shape
    pad = (0, _round_up(cols, BLOCK) - cols, 0, _round_up(rows, BLOCK) - rows)
    x = torch.nn.functional.pad(x, pad)
    tall = x.shape[0] // BLOCK
    largest = x.abs().unflatten(1, (-1, BLOCK)).amax(2)
    if square:
        largest = largest.view(tall, BLOCK, -1).amax(1).repeat_interleave(BLOCK, 0)
    scale = torch.where(largest > 0, torch.exp2(torch.ceil(torch.log2(largest / 448.0)).clamp(min=-126.0)), 1.0)
    v = x / scale.repeat_interleave(BLOCK, 1)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(v / step) * step)[:rows], scale[:rows].t().contiguous()


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        h, gain = s["x"].double(), s["gain"].double()
        if case["backward"]:
            inverse = 1.0 / torch.sqrt((h * h).sum(1) / case["cols"] + EPS)
            unit = h * inverse[:, None]
            g = s["dy"].double() * gain
            dh = inverse[:, None] * (g - unit * ((g * unit).sum(1) / case["cols"])[:, None])
            if s["past"] is not None:
                dh = dh + s["past"].double()
            return {"dh": dh, "dgain": (s["dy"].double() * unit).sum(0)}
        out = {}
        if s["past"] is not None:
            out["sum"] = h + s["past"].double()
            h = out["sum"].to(s["x"].dtype).double()  # the norm is that of the sum as it is stored
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["cols"] + EPS) * gain
        if case["keep_y"]:
            out["y"] = y
        out["values"], out["scales"] = _exact_scaled(y, False)
        return out
    if case["op"] == "quantize":
        x = s["x"].double()
        if s["mask"] is not None:
            x = x.masked_fill(s["mask"] == 0, 0.0)
        out = {}
        if case["ways"] != "columns":
            out["values"], out["scales"] = _exact_scaled(x, case["square"])
        if case["ways"] != "rows":
            out["values_t"], out["scales_t"] = _exact_scaled(x.t(), case["square"])
        return out
    if case["op"] == "product":
        wide = []
        for values, scales in (s["a"], s["b"]):
            wide.append(values.double() * scales.double().t().repeat_interleave(BLOCK, 1))
        out = wide[0] @ wide[1].t()
        return out if s["mask"] is None else out.masked_fill(s["mask"] == 0, 0.0)
    total = 0.0
    for g in s["grads"]:
        total += float(g.double().pow(2).sum())
    norm = total ** 0.5
    factor = min(1.0, s["largest"] / norm)
    return {"grads": _joined([g.double() * factor for g in s["grads"]]), "norm": torch.tensor([norm, factor], dtype=torch.float64)}
