"""Performance cases of what a pre-norm feed-forward block needs beside its Matmuls: layer normalisation and its gradients for training,
and the block's weights in microscaled 4-bit floating point for serving.

    layer_norm        y = (x - mean) r w + b over each row of n, r = 1 / sqrt(var + eps); with `stats` also (mean, r)
    layer_norm_grad   h = (x - mean) r, g = grad w; dx = residual + r (g - mean(g) - h mean(g h)); dw, db: the sums of grad h
                      and grad over the rows
    mx_quantize       a tensor to blocks of 32 along k: a scale 2^e, e = floor(log2 max) - 2, and 32 values of
                      0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, the nearest ones (ties to the even code, at most 6); and
                      what they stand for, read back
    mx_linear         out = residual + f(Q lhs rhs + bias): rhs in blocks along k, Q lhs lhs in such blocks (quantised in the
                      call, or given so)

Quantised tensors are kept as the framework keeps them: `codes`, lines along k of two values a byte (the first in the low half), k filled
up to a multiple of 128 with zeros; `scales`, a byte e + 127 for each block, in the order in which sixteen-row matrix instructions
take them: block t = 4 s + g of line l = 64 G + 32 a + 8 b + 4 c + d is scales[G, s, g, 4 b + d, 2 a + c].
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ("none", "relu", "gelu", "silu")
EPS = 1e-5
LARGEST = 8192 * 2048 * 16384       # products of a pass
ELEMENTS = 8192 * 16384             # elements of a normalisation or quantisation


def _norm(name, op, m, n, dtype, **more):
    case = {"op": op, "b": 1, "m": m, "n": n, "dtype": dtype, "weight": "f32", "bias": "f32", "stats": False, "residual": False}
    case.update(more)
    return dict(case, name=name) if name else case


def _quantize(name, m, n, dtype, dim):
    case = {"op": "mx_quantize", "m": m, "n": n, "dtype": dtype, "dim": dim}
    return dict(case, name=name) if name else case


def _linear(name, m, k, n, dtype, out, **more):
    case = {"op": "mx_linear", "b": 1, "m": m, "k": k, "n": n, "dtype": dtype, "out": out, "batched": False, "quantized": False,
            "bias": False, "residual": False, "activation": "none"}
    case.update(more)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the normalisation in front of a block for one token: a launch
        _norm("norm_token", "layer_norm", 1, 2048, "bf16"),
        # and in a training step, statistics kept for the gradient
        _norm("norm_train", "layer_norm", 8192, 2048, "bf16", weight="bf16", bias="bf16", stats=True),
        # an odd width in f32, no bias
        _norm("norm_ragged_f32", "layer_norm", 1000, 4099, "f32", bias="none", stats=True),
        # the gradients of the training step, added to the residual stream's
        _norm("norm_grad_train", "layer_norm_grad", 8192, 2048, "bf16", weight="bf16", bias="bf16", residual=True),
        # of the widest rows (a normalisation inside a block, over its wide half)
        _norm("norm_grad_wide", "layer_norm_grad", 4096, 16384, "bf16"),
        # of a small layer with odd sizes in f32
        _norm("norm_grad_ragged_f32", "layer_norm_grad", 1000, 777, "f32"),
        # a prompt's activations, along their rows
        _quantize("quantize_rows", 8192, 2048, "bf16", -1),
        # a weight matrix of k x n, k from row to row, once when a model is loaded
        _quantize("quantize_weight_f32", 2048, 16384, "f32", -2),
        # a decoding step: the weights are read once, nothing else costs
        _linear("mx_token", 1, 2048, 16384, "bf16", "bf16"),
        # a few sequences that decode together, widths that are no multiple of anything
        _linear("mx_tokens_odd", 7, 2047, 1001, "bf16", "bf16", bias=True, residual=True, activation="gelu"),
        # a long prompt's first half of a feed-forward block
        _linear("mx_prompt_up", 8192, 2048, 16384, "bf16", "bf16", bias=True, activation="gelu"),
        # and the second half: activations that are quantised already, a long sum, f32 results
        _linear("mx_prompt_down", 4096, 16384, 2048, "bf16", "f32", quantized=True, bias=True, residual=True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A size: as it comes, or a multiple of 40, or a power of two (as most layers have them)."""
    size = _log_uniform(rng, lo, hi)
    kind = rng.choice(["any", "any", "multiple", "power"])
    if kind == "multiple" and size >= 40:
        return size // 40 * 40
    return 1 << (size.bit_length() - 1) if kind == "power" else size


def draw(rng):
    op = rng.choice(["layer_norm"] * 2 + ["layer_norm_grad"] * 3 + ["mx_quantize"] * 2 + ["mx_linear"] * 4)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "mx_linear":
        b = rng.choice([1, 1, 1, rng.randint(2, 16)])
        m, k, n = _log_uniform(rng, 1, 8192), _width(rng, 16, 16384), _width(rng, 16, 16384)
        while b * m * k * n > LARGEST:
            m = max(1, m // 2)
        return _linear(None, m, k, n, dtype, rng.choice([dtype, "bf16", "f32"]), b=b, batched=b > 1 and rng.random() < 0.5, quantized=rng.random() < 0.3,
                       bias=rng.random() < 0.7, residual=rng.random() < 0.4, activation=rng.choice(ACTIVATIONS))
    # (rows of two elements or so have a gradient of next to nothing, whatever the numbers)
    m, n = _log_uniform(rng, 1, 65536), _width(rng, 16, 16384)
    most = ELEMENTS // 2 if op == "layer_norm_grad" else ELEMENTS // 4
    while m * n > most:
        m = max(1, m // 2)
    if op == "mx_quantize":
        return _quantize(None, m, n, dtype, rng.choice([-1, -2])) if rng.random() < 0.5 else _quantize(None, n, m, dtype, rng.choice([-1, -2]))
    weight = rng.choice(["none", "f32", dtype, dtype])
    return _norm(None, op, m, n, dtype, weight=weight, bias=rng.choice(["none", "f32", dtype]), stats=op == "layer_norm" and rng.random() < 0.5,
                 residual=op == "layer_norm_grad" and rng.random() < 0.5)


def _shapes(case):
    """Shapes of lhs, rhs and out of a product."""
    lead = (case["b"],) if case["b"] > 1 or case["batched"] else ()
    return (lead + (case["m"], case["k"]), (lead if case["batched"] else ()) + (case["k"], case["n"]), lead + (case["m"], case["n"]))


# ---- quantised tensors in elementary operations

def _powers(e):
    """2^e in f32, e from -126 to 127."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _fill_up(x, multiple):
    """x with zeros behind its last dimension, up to a multiple."""
    k = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -k % multiple)) if k % multiple else x


def _blocks(lines):
    """(magnitudes of 0 to 6, signs, exponents) of the blocks of lines along k, f32: finite values."""
    x = _fill_up(lines.float(), 128)
    x = x.reshape(x.shape[:-1] + (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    e = torch.where(most > 0, torch.frexp(most).exponent - 3, -127).clamp_(min=-127)
    v = x.abs() * _powers(-e)
    v = torch.where(v < 2, torch.round(v * 2) / 2, torch.where(v < 4, torch.round(v), torch.round(v / 2) * 2)).clamp_(max=6.0)
    return v, torch.signbit(x), e


def _stored(lines):
    """(codes, scales) of lines along k."""
    v, negative, e = _blocks(lines)
    code = (torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8) | negative.to(torch.uint8) << 3).flatten(-2)
    codes = code[..., 0::2] | code[..., 1::2] << 4
    s = (e.squeeze(-1) + 127).to(torch.uint8)
    s = torch.nn.functional.pad(s, (0, 0, 0, -s.shape[-2] % 64))
    lead = s.shape[:-2]
    s = s.reshape(lead + (s.shape[-2] // 64, 2, 4, 2, 4, s.shape[-1] // 4, 4))         # G a b c d s g
    n = len(lead)
    s = s.permute(tuple(range(n)) + tuple(n + i for i in (0, 5, 6, 2, 4, 1, 3))).reshape(lead + (s.shape[n], s.shape[n + 5], 4, 16, 4))
    return codes.contiguous(), s.contiguous()


def _values(codes, scales, k, dtype):
    """What (codes, scales) stand for, lines along k."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=dtype, device=codes.device)
    lead, n = scales.shape[:-5], len(scales.shape) - 5
    s = scales.reshape(lead + scales.shape[n:n + 3] + (4, 4, 2, 2))                      # G s g b d a c
    s = s.permute(tuple(range(n)) + tuple(n + i for i in (0, 5, 3, 6, 4, 1, 2)))
    s = s.reshape(lead + (scales.shape[n] * 64, scales.shape[n + 1] * 4))[..., :codes.shape[-2], :]
    # (2^-127 is half of the least power that _powers has)
    power = torch.where(s > 0, _powers(s.int().clamp(min=1) - 127), _powers(torch.full_like(s, -126, dtype=torch.int32)) / 2).to(dtype)
    v = grid[code.long()].reshape(code.shape[:-1] + (-1, 32)) * power[..., None]
    return v.flatten(-2)[..., :k]


def prepare(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)

    def normal(shape, dtype, scale=1.0, shift=0.0):
        return (torch.randn(shape, generator=gen, device=device, dtype=torch.float32) * scale + shift).to(DTYPES[dtype])

    state = {"case": case}
    if case["op"] in ("layer_norm", "layer_norm_grad"):
        m, n = case["m"], case["n"]
        # channels of several scales and a shift, as a residual stream has them
        state["x"] = (normal((m, n), "f32") * torch.exp(normal((n,), "f32", 0.5)) + normal((n,), "f32", 0.3)).to(DTYPES[case["dtype"]])
        state["weight"] = normal((n,), case["weight"], 0.2, 1.0) if case["weight"] != "none" else None
        state["bias"] = normal((n,), case["bias"], 0.1) if case["bias"] != "none" else None
        if case["op"] == "layer_norm_grad":
            state["grad"] = normal((m, n), case["dtype"])
            state["residual"] = normal((m, n), case["dtype"]) if case["residual"] else None
            mean = state["x"].double().mean(-1, keepdim=True)
            var = (state["x"].double() - mean).square().mean(-1, keepdim=True)
            state["stats"] = torch.cat((mean, 1 / torch.sqrt(var + EPS)), -1).float()
        return state
    if case["op"] == "mx_quantize":
        shape = (case["m"], case["n"])
        state["x"] = (normal(shape, "f32") * torch.exp(normal((shape[1],), "f32", 0.5))).to(DTYPES[case["dtype"]])
        return state
    lhs, rhs, out = _shapes(case)
    state["lhs"] = normal(lhs, case["dtype"])
    if case["quantized"]:
        state["lhs"] = _stored(state["lhs"])
    # weights at the scale that keeps the sums near 1, in 4 bits as a program that serves keeps them
    state["rhs"] = _stored(normal(rhs[:-2] + (rhs[-1], rhs[-2]), "f32", case["k"] ** -0.5))
    state["bias"] = normal((case["n"],), case["dtype"], 0.1) if case["bias"] else None
    state["residual"] = normal(out, case["out"]) if case["residual"] else None
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2505_01637_amd import binding as B
    case = state["case"]
    if case["op"] == "layer_norm":
        return B.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS, stats=case["stats"])
    if case["op"] == "layer_norm_grad":
        return B.layer_norm_grad(state["grad"], state["x"], state["stats"], state["weight"], state["bias"], state["residual"])
    if case["op"] == "mx_quantize":
        return B.mx_dequantize(B.mx_quantize(state["x"], dim=case["dim"]))
    lhs = state["lhs"]
    if case["quantized"]:
        lhs = B.MX(lhs[0], lhs[1], case["k"], dtype=DTYPES[case["dtype"]])
    return B.mx_linear(lhs, B.MX(state["rhs"][0], state["rhs"][1], case["k"], dim=-2), state["bias"], state["residual"], activation=case["activation"],
                       dtype=DTYPES[case["out"]])


# ---- the plain form: torch, in 32 bits, rounded once at the end

def _activate(z, activation):
    if activation == "relu":
        return torch.clamp(z, min=0.0)
    if activation == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if activation == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _run_plain(state):
    case = state["case"]
    if case["op"] == "layer_norm":
        x = state["x"].float()
        mean = x.mean(-1, keepdim=True)
        centred = x - mean
        r = 1.0 / torch.sqrt(centred.square().mean(-1, keepdim=True) + EPS)
        y = centred * r
        if state["weight"] is not None:
            y = y * state["weight"].float()
        if state["bias"] is not None:
            y = y + state["bias"].float()
        y = y.to(state["x"].dtype)
        return (y, torch.cat((mean, r), -1)) if case["stats"] else y
    if case["op"] == "layer_norm_grad":
        grad, mean, r = state["grad"].float(), state["stats"][:, :1], state["stats"][:, 1:]
        h = (state["x"].float() - mean) * r
        g = grad * state["weight"].float() if state["weight"] is not None else grad
        dx = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
        if state["residual"] is not None:
            dx = dx + state["residual"].float()
        dw = (grad * h).sum(0).to(state["weight"].dtype) if state["weight"] is not None else None
        db = grad.sum(0).to(state["bias"].dtype) if state["bias"] is not None else None
        return dx.to(state["x"].dtype), dw, db
    if case["op"] == "mx_quantize":
        x = state["x"] if case["dim"] == -1 else state["x"].t()
        codes, scales = _stored(x)
        out = _values(codes, scales, x.shape[-1], torch.float32).to(x.dtype)
        return out if case["dim"] == -1 else out.t()
    codes, scales = state["lhs"] if case["quantized"] else _stored(state["lhs"])
    lhs = _values(codes, scales, case["k"], torch.float32)
    rhs = _values(*state["rhs"], case["k"], torch.float32).transpose(-1, -2).contiguous()
    z = torch.matmul(lhs, rhs)
    if state["bias"] is not None:
        z = z + state["bias"].float()
    out = _activate(z, case["activation"])
    if state["residual"] is not None:
        out = out + state["residual"].float()
    return out.to(DTYPES[case["out"]])


# ---- what a pass cannot do without

def work(case):
    size = {"f32": 4, "bf16": 2, "none": 0}
    if case["op"] in ("layer_norm", "layer_norm_grad"):
        m, n, s = case["m"], case["n"], size[case["dtype"]]
        vectors = n * (size[case["weight"]] + size[case["bias"]])
        if case["op"] == "layer_norm":
            return {"bytes": 2 * m * n * s + vectors + 8 * m * case["stats"], "flops": 8 * m * n}
        return {"bytes": (3 + case["residual"]) * m * n * s + 8 * m + n * (2 * size[case["weight"]] + size[case["bias"]]), "flops": 14 * m * n}
    if case["op"] == "mx_quantize":
        # read, written in 4.25 bits, those read, written
        values = case["m"] * case["n"]
        return {"bytes": int(values * (2 * size[case["dtype"]] + 2 * 17 / 32)), "flops": 6 * values}
    b, m, k, n = case["b"], case["m"], case["k"], case["n"]
    lhs, rhs, out = b * m * k, (b if case["batched"] else 1) * k * n, b * m * n
    return {"bytes": int(lhs * (17 / 32 if case["quantized"] else size[case["dtype"]]) + rhs * 17 / 32 + (n * size[case["dtype"]] if case["bias"] else 0)
                         + out * size[case["out"]] * (1 + case["residual"])), "flops": 2 * b * m * k * n}


# ---- the definition in 64 bits

def _two_to(e):
    """2^e in 64 bits (pow is not exact everywhere)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(lines):
    """Lines along k in blocks, read back: the nearest of the sixteen values, found by the borders between them."""
    k = lines.shape[-1]
    x = lines.double()
    x = torch.cat((x, x.new_zeros(x.shape[:-1] + (-k % 32,))), -1).unflatten(-1, (-1, 32))
    most = x.abs().max(-1, keepdim=True).values
    power = torch.where(most == 0, -127.0, torch.log2(most).floor() - 2)
    power = power + (most >= _two_to(power + 3)).double() - (most < _two_to(power + 2)).double()          # (where log2 was rounded over a whole number)
    step = _two_to(power.clamp(min=-127.0))
    scaled = x.abs() / step
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    index = torch.zeros(scaled.shape, dtype=torch.int64, device=x.device)
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        index += (scaled > border) if i % 2 == 0 else (scaled >= border)
    return (grid[index] * step * torch.sign(x)).flatten(-2)[..., :k]


def _read(codes, scales, k):
    """Stored lines read back one block position at a time."""
    lines, steps = codes.shape[-2], codes.shape[-1] // 64
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=codes.device)
    out = torch.empty(codes.shape[:-1] + (codes.shape[-1] * 2,), dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        nibble = (codes >> (4 * half)).long() % 16
        out[..., half::2] = grid[nibble % 8] * (1 - 2 * (nibble // 8))
    line = torch.arange(lines, device=codes.device)[:, None]
    block = torch.arange(4 * steps, device=codes.device)[None, :]
    inner = line % 64
    byte = scales[..., line // 64, block // 4, block % 4, inner // 8 % 4 * 4 + inner % 4, inner // 32 * 2 + inner // 4 % 2]
    return (out.unflatten(-1, (-1, 32)) * _two_to(byte.long() - 127)[..., None]).flatten(-2)[..., :k]


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] in ("layer_norm", "layer_norm_grad"):
        x, n = state["x"].double(), case["n"]
        weight = 1.0 if state["weight"] is None else state["weight"].double()
        if case["op"] == "layer_norm":
            mean = x.sum(-1) / n
            var = (x - mean[:, None]).pow(2).sum(-1) / n
            out = (x - mean[:, None]) / (var[:, None] + EPS).sqrt() * weight
            if state["bias"] is not None:
                out = out + state["bias"]
            return (out, torch.stack((mean, (var + EPS).rsqrt()), -1)) if case["stats"] else out
        grad, mean, r = state["grad"].double(), state["stats"][:, 0].double(), state["stats"][:, 1].double()
        h = (x - mean[:, None]) * r[:, None]
        g = grad * weight
        sums = torch.stack((g.sum(-1), (g * h).sum(-1))) / n
        dx = (g - sums[0][:, None] - h * sums[1][:, None]).mul_(r[:, None])
        if state["residual"] is not None:
            dx = dx + state["residual"]
        return dx, None if state["weight"] is None else torch.linalg.vecdot(grad, h, dim=0), None if state["bias"] is None else grad.sum(0)
    if case["op"] == "mx_quantize":
        return _nearest(state["x"]) if case["dim"] == -1 else _nearest(state["x"].t()).t()
    lhs = _read(*state["lhs"], case["k"]) if case["quantized"] else _nearest(state["lhs"])
    lhs, rhs = lhs.reshape(-1, case["m"], case["k"]), _read(*state["rhs"], case["k"]).reshape(-1, case["n"], case["k"])
    z = torch.stack([x @ rhs[i if case["batched"] else 0].t() for i, x in enumerate(lhs)]).reshape(_shapes(case)[2])
    if state["bias"] is not None:
        z = z + state["bias"].double()
    if case["activation"] == "relu":
        z = torch.where(z > 0, z, torch.zeros_like(z))
    elif case["activation"] == "silu":
        z = z * torch.sigmoid(z)
    elif case["activation"] == "gelu":      # (1 + tanh u) / 2 is the logistic function of 2 u
        z = z * torch.sigmoid(z.pow(3).mul_(0.044715).add_(z).mul_(2 * math.sqrt(2 / math.pi)))
    return z if state["residual"] is None else z + state["residual"].double()
