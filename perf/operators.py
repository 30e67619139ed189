"""Performance cases of the operators that the framework's Specs name, on data: the Matmul with bias, activation,
dropout and residual in its epilogue, its gradients, and dropout alone.

    linear        out = residual + D f(lhs rhs + bias), and z = lhs rhs + bias itself where `pre` is set
    linear_grad   dz = D f'(z) grad; dlhs = dz rhs^T, drhs = lhs^T dz, dbias = the sum of dz over the rows
    dropout       out = residual + D x
    dropout_grad  D grad

lhs is b x m x k, rhs k x n (or b x k x n with `batched`), row- or column-major.  f is the identity, ReLU, GELU in
its tanh form, or SiLU.  D is 0 where an element is dropped and 2^16 / (2^16 - T) elsewhere, T = round(p 2^16).  An
element is dropped if its 16 random bits are below T: the bits of element (i, j), i the row over all batches, are the
half (j % 2) of word (j % 8) / 2 of the Philox4x32 block of seven rounds (Salmon, Moraes, Dror, Shaw, 2011) with the
seed as key and the counter (j / 8, i, offset's low word, offset's high word).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ("none", "relu", "gelu", "silu")
LARGEST = 8192 * 2048 * 16384       # products of a pass in bf16 (a gradient has two Matmuls, so half of it)
LARGEST_F32 = LARGEST // 8          # and in f32, whose matrix rate is a sixteenth
ELEMENTS = 8192 * 16384             # elements of a dropout


def _linear(name, m, k, n, dtype, out, **more):
    case = {"op": "linear", "b": 1, "m": m, "k": k, "n": n, "dtype": dtype, "out": out, "batched": False, "rhs_columns": False,
            "bias": False, "residual": False, "activation": "none", "dropout": 0.0, "pre": False}
    case.update(more)
    return dict(case, name=name) if name else case


def _grad(name, m, k, n, dtype, **more):
    case = {"op": "linear_grad", "b": 1, "m": m, "k": k, "n": n, "dtype": dtype, "batched": False, "rhs_columns": False,
            "bias": True, "activation": "none", "dropout": 0.0}
    case.update(more)
    return dict(case, name=name) if name else case


def _dropout(name, op, m, n, dtype, p, residual=False):
    case = {"op": op, "m": m, "n": n, "dtype": dtype, "dropout": p, "residual": residual}
    return dict(case, name=name) if name else case


def listed():
    return [
        # a decoding step's vector-matrix product, 1 x 2048 x 16384, bf16 inputs and f32 results (logits, or the wide half of a
        # feed-forward block for one sequence): the weights are read once, nothing else costs
        _linear("linear_token", 1, 2048, 16384, "bf16", "f32", rhs_columns=True),
        # the smallest call: one row through one small fused layer; launches and the host's part
        _linear("linear_token_small", 1, 256, 256, "f32", "f32", bias=True, activation="relu"),
        # a few sequences that decode together, widths that are no multiple of anything
        _linear("linear_tokens_odd", 7, 2047, 1001, "bf16", "bf16", bias=True, residual=True, activation="gelu"),
        # the goal of the fused configuration, a 2048-cube in f32 with bias and ReLU
        _linear("linear_cube_f32", 2048, 2048, 2048, "f32", "f32", bias=True, activation="relu"),
        # a batch of small ragged Matmuls, each with its own right-hand side
        _linear("linear_batched_ragged", 100, 72, 56, "f32", "f32", b=16, batched=True, bias=True, activation="silu"),
        # a training step's (or long prompt's) first half of a feed-forward block, z kept for the gradient
        _linear("linear_train_up", 8192, 2048, 16384, "bf16", "bf16", bias=True, activation="gelu", pre=True),
        # and the second half: a long sum, dropout and residual in the epilogue
        _linear("linear_train_down", 4096, 16384, 2048, "bf16", "bf16", bias=True, residual=True, dropout=0.1),
        # the gradients of a training step's first half, dropout on its activations
        _grad("grad_train_up", 4096, 2048, 16384, "bf16", activation="gelu", dropout=0.1),
        # a small layer with odd sizes trained in f32
        _grad("grad_ragged_f32", 1000, 511, 777, "f32", activation="relu", dropout=0.25, rhs_columns=True),
        # one row of activations: a launch
        _dropout("dropout_row", "dropout", 1, 2048, "bf16", 0.1),
        # the largest activations of the training step above, added to the residual stream
        _dropout("dropout_residual", "dropout", 8192, 16384, "bf16", 0.1, residual=True),
        # a gradient of odd widths in f32
        _dropout("dropout_grad_ragged", "dropout_grad", 1000, 4099, "f32", 0.3),
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
    op = rng.choice(["linear"] * 5 + ["linear_grad"] * 3 + ["dropout", "dropout_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    p = rng.choice([0.1, 0.3, round(rng.uniform(0.01, 0.99), 3)])
    if op in ("dropout", "dropout_grad"):
        m, n = _log_uniform(rng, 1, 65536), _width(rng, 1, 16384)
        while m * n > ELEMENTS:
            m = max(1, m // 2)
        return _dropout(None, op, m, n, dtype, p, residual=op == "dropout" and rng.random() < 0.5)
    most = LARGEST if dtype == "bf16" else LARGEST_F32
    if op == "linear_grad":
        most //= 2
    b = rng.choice([1, 1, 1, rng.randint(2, 16)])
    m, k, n = _log_uniform(rng, 1, 8192), _width(rng, 16, 16384), _width(rng, 16, 16384)
    while b * m * k * n > most:
        m = max(1, m // 2)
    more = {"b": b, "batched": b > 1 and rng.random() < 0.5, "rhs_columns": rng.random() < 0.5, "bias": rng.random() < 0.7,
            "activation": rng.choice(ACTIVATIONS), "dropout": p if rng.random() < 0.4 else 0.0}
    if op == "linear_grad":
        return _grad(None, m, k, n, dtype, **more)
    out = rng.choice([dtype, dtype, "f32"])
    return _linear(None, m, k, n, dtype, out, residual=rng.random() < 0.4, pre=rng.random() < 0.3, **more)


def _shapes(case):
    """Shapes of lhs, rhs and out."""
    lead = (case["b"],) if case["b"] > 1 or case["batched"] else ()
    return (lead + (case["m"], case["k"]), (lead if case["batched"] else ()) + (case["k"], case["n"]), lead + (case["m"], case["n"]))


def prepare(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)

    def normal(shape, dtype, scale=1.0):
        return (torch.randn(shape, generator=gen, device=device, dtype=torch.float32) * scale).to(DTYPES[dtype])

    state = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 1) % (1 << 64), "offset": seed % 1000}
    if case["op"] in ("dropout", "dropout_grad"):
        shape = (case["m"], case["n"])
        state["x"] = normal(shape, case["dtype"])
        state["residual"] = normal(shape, case["dtype"]) if case["residual"] else None
        return state
    lhs, rhs, out = _shapes(case)
    dtype = case["dtype"]
    state["lhs"] = normal(lhs, dtype)
    # weights at the scale that keeps z near 1
    if case["rhs_columns"]:
        state["rhs"] = normal(rhs[:-2] + (rhs[-1], rhs[-2]), dtype, case["k"] ** -0.5).transpose(-1, -2)
    else:
        state["rhs"] = normal(rhs, dtype, case["k"] ** -0.5)
    state["bias"] = normal((case["n"],), dtype, 0.1) if case["bias"] else None
    if case["op"] == "linear":
        state["residual"] = normal(out, case["out"]) if case["residual"] else None
    else:
        state["grad"] = normal(out, dtype)
        state["pre"] = normal(out, dtype) if case["activation"] != "none" else None
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2505_01637_amd import binding as B
    case = state["case"]
    random = {"dropout": case["dropout"], "seed": state["seed"], "offset": state["offset"]}
    if case["op"] == "dropout":
        return B.dropout(state["x"], state["residual"], **random)
    if case["op"] == "dropout_grad":
        return B.dropout_grad(state["x"], **random)
    if case["op"] == "linear":
        return B.linear(state["lhs"], state["rhs"], state["bias"], state["residual"], activation=case["activation"],
                        dtype=DTYPES[case["out"]], pre=case["pre"], **random)
    return B.linear_grad(state["grad"], state["lhs"], state["rhs"], state["bias"], state["pre"], activation=case["activation"], **random)


# ---- the plain form: torch, in 32 bits, rounded once at the end

_LOW = 0xFFFFFFFF


def _scale(rows, cols, p, seed, offset, device):
    """D of a rows x cols tensor, f32."""
    threshold = int(p * 65536 + 0.5)
    if threshold == 0:
        return None
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, device=device, dtype=torch.int64).expand(rows, blocks)
    c1 = torch.arange(rows, device=device, dtype=torch.int64)[:, None].expand(rows, blocks)
    c2 = torch.full((), offset & _LOW, device=device, dtype=torch.int64)
    c3 = torch.full((), offset >> 32, device=device, dtype=torch.int64)
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57         # (products mod 2^64; the shift's sign bits are masked away)
        c0, c1, c2, c3 = (b >> 32 & _LOW) ^ c1 ^ k0, b & _LOW, (a >> 32 & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    bits = torch.stack([w.expand(rows, blocks) >> s & 0xFFFF for w in (c0, c1, c2, c3) for s in (0, 16)], dim=-1)
    keep = bits.reshape(rows, blocks * 8)[:, :cols] >= threshold
    return keep.to(torch.float32) * (65536.0 / (65536 - threshold) if threshold < 65536 else 0.0)


def _activate(z, activation):
    if activation == "relu":
        return torch.clamp(z, min=0.0)
    if activation == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if activation == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, activation):
    if activation == "relu":
        return (z > 0).to(z.dtype)
    if activation == "gelu":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _drop(x, state):
    """D x, over the last dimension's rows."""
    d = _scale(x.numel() // x.shape[-1], x.shape[-1], state["case"]["dropout"], state["seed"], state["offset"], x.device)
    return x if d is None else torch.where(d.reshape(x.shape) > 0, x * d.reshape(x.shape), 0.0)


def _run_plain(state):
    case = state["case"]
    if case["op"] in ("dropout", "dropout_grad"):
        out = _drop(state["x"].float(), state)
        if state["residual"] is not None:
            out = out + state["residual"].float()
        return out.to(state["x"].dtype)
    lhs, rhs = state["lhs"].float(), state["rhs"].float()
    if case["op"] == "linear":
        z = torch.matmul(lhs, rhs)
        if state["bias"] is not None:
            z = z + state["bias"].float()
        out = _drop(_activate(z, case["activation"]), state)
        if state["residual"] is not None:
            out = out + state["residual"].float()
        out = out.to(DTYPES[case["out"]])
        return (out, z.to(DTYPES[case["out"]])) if case["pre"] else out
    dz = _drop(state["grad"].float(), state)
    if state["pre"] is not None:
        dz = dz * _slope(state["pre"].float(), case["activation"])
    dlhs = torch.matmul(dz, rhs.transpose(-1, -2).contiguous())
    if case["batched"]:
        drhs = torch.matmul(lhs.transpose(-1, -2).contiguous(), dz)
    else:
        drhs = torch.matmul(lhs.reshape(-1, case["k"]).t(), dz.reshape(-1, case["n"]))
    dbias = dz.reshape(-1, case["n"]).sum(0).to(state["bias"].dtype) if state["bias"] is not None else None
    return dlhs.to(state["lhs"].dtype), drhs.to(state["rhs"].dtype), dbias


# ---- what a pass cannot do without

def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] in ("dropout", "dropout_grad"):
        tensors = 3 if case["residual"] else 2
        return {"bytes": tensors * case["m"] * case["n"] * size[case["dtype"]], "flops": 2 * case["m"] * case["n"]}
    b, m, k, n, s = case["b"], case["m"], case["k"], case["n"], size[case["dtype"]]
    lhs, rhs, out, bias = b * m * k, (b if case["batched"] else 1) * k * n, b * m * n, n if case["bias"] else 0
    if case["op"] == "linear":
        wide = size[case["out"]] * out * (1 + case["residual"] + case["pre"])
        return {"bytes": s * (lhs + rhs + bias) + wide, "flops": 2 * b * m * k * n}
    read = lhs + rhs + out * (1 if case["activation"] == "none" else 2)
    return {"bytes": s * (read + lhs + rhs + bias), "flops": 4 * b * m * k * n}


# ---- the definition in 64 bits

def _random_bits(rows, cols, seed, offset, device):
    """The 16 random bits of every element, by products of 16-bit halves."""
    def times(x, constant):
        xl, xh, cl, ch = x & 0xFFFF, x >> 16, constant & 0xFFFF, constant >> 16
        low, mid, high = xl * cl, xh * cl + (xl * cl >> 16), xl * ch
        mid2 = (mid & 0xFFFF) + high
        return xh * ch + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | low & 0xFFFF
    groups = -(-cols // 8)
    i = torch.arange(rows * groups, device=device, dtype=torch.int64)
    counter = [i % groups, i // groups, torch.full_like(i, offset % 2 ** 32), torch.full_like(i, offset // 2 ** 32)]
    for r in range(7):
        key = [(seed + r * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        h0, l0 = times(counter[0], 0xD2511F53)
        h1, l1 = times(counter[2], 0xCD9E8D57)
        counter = [h1 ^ counter[1] ^ key[0], l1, h0 ^ counter[3] ^ key[1], l0]
    out = torch.empty((rows * groups, 8), device=device, dtype=torch.int32)
    for w in range(4):
        out[:, 2 * w] = counter[w] % 65536
        out[:, 2 * w + 1] = counter[w] // 65536
    return out.view(rows, groups * 8)[:, :cols]


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] in ("dropout", "dropout_grad"):
        wide, cols = state["x"].double(), case["n"]
    else:
        wide, cols = None, case["n"]
    rows = case.get("b", 1) * case["m"]
    device = state["x"].device if wide is not None else state["lhs"].device
    dropped = math.floor(case["dropout"] * 65536 + 0.5)

    def masked(t):
        if dropped == 0:
            return t
        bits = _random_bits(rows, cols, state["seed"], state["offset"], device).reshape(t.shape)
        return torch.zeros_like(t) if dropped == 65536 else (t * (65536 / (65536 - dropped))).masked_fill(bits < dropped, 0.0)

    if wide is not None:
        out = masked(wide)
        return out if state["residual"] is None else out.add_(state["residual"])
    lhs = state["lhs"].double().reshape(-1, case["m"], case["k"])
    rhs = state["rhs"].double().reshape(-1, case["k"], case["n"])
    shared = not case["batched"]
    if shared:
        lhs = lhs.reshape(1, -1, case["k"])
    if case["op"] == "linear":
        z = torch.stack([x @ y for x, y in zip(lhs, rhs)]) if len(lhs) > 1 else (lhs[0] @ rhs[0])[None]
        if state["bias"] is not None:
            z = z + state["bias"].double()
        shape = _shapes(case)[2]
        z = z.reshape(shape)
        if case["activation"] == "none":
            f = z
        elif case["activation"] == "relu":
            f = torch.where(z > 0, z, torch.zeros_like(z))
        elif case["activation"] == "silu":
            f = z * torch.sigmoid(z)
        else:       # (1 + tanh u) / 2 is the logistic function of 2 u
            f = z * torch.sigmoid(z.pow(3).mul_(0.044715).add_(z).mul_(2 * math.sqrt(2 / math.pi)))
        out = masked(f)
        if state["residual"] is not None:
            out = out + state["residual"].double()
        return (out, z) if case["pre"] else out
    dz = masked(state["grad"].double())
    if case["activation"] != "none":
        z = state["pre"].double()
        if case["activation"] == "relu":
            dz = dz.masked_fill(z <= 0, 0.0)
        elif case["activation"] == "silu":
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        else:
            c = 2 * math.sqrt(2 / math.pi)
            u = c * (z + 0.044715 * z ** 3)
            dz = dz * (torch.sigmoid(u) + z * torch.sigmoid(u) * torch.sigmoid(-u) * c * (1 + 0.134145 * z ** 2))
    dz = dz.reshape(len(lhs), -1, case["n"])
    dlhs = torch.stack([d @ y.t() for d, y in zip(dz, rhs)]).reshape(_shapes(case)[0])
    drhs = torch.stack([x.t() @ d for x, d in zip(lhs, dz)]).reshape(_shapes(case)[1])
    return dlhs, drhs, (dz.sum((0, 1)) if case["bias"] else None)
