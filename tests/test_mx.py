"""Microscaled 4-bit floating point: quantisation, what it stands for, and products of such operands (binding.mx_quantize,
mx_dequantize, mx_linear) against plain implementations in 64 bits.

Codes and scales have to be equal.  A product of values that the blocks stand for is within (k + 2) u of the exact one times the sum of
magnitudes, u = 2^-24, as linear's (its products are exact in f32, and so are the sums within a block); the epilogue's part is linear's too.
"""
import ctypes as C

import numpy as np
import pytest

from paper_2505_01637_amd import binding as B
from test_operators import U, _torch, check, f64, f_of, strided

gpu = pytest.mark.gpu
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks_of(lines):
    """(codes, exponent bytes) of lines along k: one value and one block a place, k filled up to 128s."""
    k = lines.shape[-1]
    x = np.concatenate([lines, np.zeros(lines.shape[:-1] + (-k % 128,))], -1).reshape(lines.shape[:-1] + (-(-k // 128) * 4, 32))
    finite = np.isfinite(x).all(-1, keepdims=True)
    x = np.where(finite, x, 0.0)
    most = np.abs(x).max(-1, keepdims=True)
    e = np.where(most > 0, np.frexp(most)[1] - 3, -127).clip(-127)
    v = np.abs(x) / np.ldexp(1.0, e)
    # the nearest value; where two are as near, the one of even number
    far = np.abs(v[..., None] - GRID)
    near = far == far.min(-1, keepdims=True)
    first, last = near.argmax(-1), 7 - near[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, last) + 8 * np.signbit(x)
    return np.where(finite, code, 0).reshape(lines.shape[:-1] + (x.shape[-2] * 32,)), np.where(finite, e + 127, 255)[..., 0]


def read(codes, scales, k):
    """The values that codes and exponent bytes stand for."""
    v = GRID[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    power = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v.reshape(scales.shape + (32,)) * power[..., None]).reshape(codes.shape)[..., :k]


def stored(q):
    """(codes, exponent bytes) of an MX, line by line: the header's formula, one block at a time."""
    raw, s = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    codes = np.stack([raw & 15, raw >> 4], -1).reshape(raw.shape[:-1] + (2 * raw.shape[-1],)).astype(int)
    line, t = np.arange(raw.shape[-2])[:, None], np.arange(codes.shape[-1] // 32)[None, :]
    G, i, j, k, l = line // 64, line // 32 % 2, line // 8 % 4, line // 4 % 2, line % 4
    return codes, s[..., G, t // 4, t % 4, 4 * j + l, 2 * i + k]


def values(q):
    """What an MX stands for, lines along k."""
    return read(*stored(q), q.k)


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def case_quantize(x, dim):
    """x: a device tensor."""
    q = B.mx_quantize(x, dim=dim)
    assert q.shape == x.shape and q.dim == dim and q.dtype == x.dtype
    lines = f64(x) if dim == -1 else np.swapaxes(f64(x), -1, -2)
    codes, scales = blocks_of(lines)
    got = stored(q)
    assert same(got[1], scales) and same(got[0], codes)
    # lines that are not there have scales of 0
    raw = q.scales.cpu().numpy()
    n = lines.shape[-2]
    full = np.zeros(raw.shape[:-5] + (-(-n // 64) * 64, scales.shape[-1]), dtype=np.uint8)
    full[..., :n, :] = scales
    padded = full.reshape(raw.shape[:-5] + (raw.shape[-5], 2, 4, 2, 4, raw.shape[-4], 4))
    axes = tuple(range(raw.ndim - 5)) + tuple(raw.ndim - 5 + i for i in (0, 5, 6, 2, 4, 1, 3))
    assert same(padded.transpose(axes).reshape(raw.shape), raw)
    want = read(codes, scales, lines.shape[-1])
    torch, types = _torch()
    for dtype in types.values():
        back = B.mx_dequantize(q, dtype=dtype)
        assert back.dtype == dtype and back.shape == x.shape
        assert same(f64(back) if dim == -1 else np.swapaxes(f64(back), -1, -2), want)
    assert B.mx_dequantize(q).dtype == x.dtype
    return q


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [-1, -2])
@pytest.mark.parametrize("shape,gap,start", [((1, 1), 0, 0), ((1, 32), 0, 0), ((2, 31), 0, 0), ((3, 33), 1, 1), ((5, 128), 0, 0), ((64, 64), 8, 0), ((65, 130), 3, 1), ((130, 257), 0, 0),
                                             ((7, 2047), 0, 0), ((200, 1000), 24, 8), ((3, 20, 70), 0, 0), ((2, 65, 129), 1, 0), ((1, 5, 40), 0, 0), ((256, 512), 0, 0), ((129, 640), 0, 8)])
@pytest.mark.parametrize("columns", [False, True])
def test_quantize(shape, gap, start, dim, columns, dtype):
    rng = np.random.default_rng(1)
    x = rng.standard_normal(shape) * np.exp(2 * rng.standard_normal(shape[-1]))
    case_quantize(strided(x, dtype, columns, gap, start), dim)


@gpu
@pytest.mark.parametrize("dim", [-1, -2])
def test_quantize_every_bf16_value(dim):
    """Every bf16 value against block maxima of 1 to 8 times itself and beside its own negative, f32 values around the borders between codes."""
    torch, _ = _torch()
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    finite = bits[bits.isfinite()]
    with_max = torch.stack([(finite.float() * f).clamp(-3e38, 3e38).bfloat16() if i % 2 == 0 else finite
                            for i, f in enumerate([1, 0, 1.5, 0, 2, 0, 3, 0, 4, 0, 5, 0, 6, 0, 7, 0]) for _ in range(2)], -1)
    x = with_max.reshape(-1, 1024)
    case_quantize((x if dim == -1 else x.t()).cuda(), dim)
    rng = np.random.default_rng(2)
    e = rng.integers(-126, 124, (500, 1))
    edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.9])
    around = np.concatenate([edges * (1 + d * 2.0 ** -23) for d in (-1, 0, 1)])
    x = np.concatenate([np.full((500, 1), 7.0), np.broadcast_to(around, (500, 27))], 1) * np.ldexp(1.0, e)
    x = torch.from_numpy(x.astype(np.float32))
    case_quantize((x if dim == -1 else x.t().contiguous()).cuda(), dim)


@gpu
@pytest.mark.parametrize("dim", [-1, -2])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_extremes(dim, dtype):
    """Blocks of zeros, of the least and largest numbers, and with values that are not finite."""
    torch, types = _torch()
    inf, nan = float("inf"), float("nan")
    x = torch.zeros((9, 160))
    x[0, 0:32] = 0.0
    x[0, 33] = -0.0
    x[1, 3], x[1, 40], x[1, 70], x[1, 100], x[1, 130] = inf, -inf, nan, 3e38, -1e-45
    x[2, :] = 1e-40
    x[3, :] = 2.0 ** -126
    x[4, :] = torch.finfo(torch.float32).max if dtype == "f32" else torch.finfo(torch.bfloat16).max
    x[5, ::3] = 2.0 ** -133
    x[6, ::5] = -2.0 ** -125
    x[7, :] = torch.linspace(-2.0 ** -123, 2.0 ** -123, 160)
    x[8, :] = torch.logspace(-45, 38, 160)
    x = x.to(types[dtype]).cuda()
    q = case_quantize(x if dim == -1 else x.t(), dim)
    assert B.mx_dequantize(q).isnan().sum() == 96


def case_linear(b, m, k, n, dtype="bf16", out=None, batched=False, quantized=False, columns=False, bias=True, residual=True, activation="none", gap=0, start=0, seed=5):
    torch, types = _torch()
    out = out or dtype
    rng = np.random.default_rng(seed)
    lead = (b,) if b is not None else ()
    lhs = strided(rng.standard_normal(lead + (m, k)) * np.exp(rng.standard_normal(k)), dtype, columns, gap, start)
    rhs = strided(rng.standard_normal((lead if batched else ()) + (k, n)) * max(k, 1) ** -0.5, dtype)
    vec = torch.from_numpy(rng.standard_normal(n)).to(types[dtype]).cuda() if bias else None
    res = strided(rng.standard_normal(lead + (m, n)), out, gap=gap) if residual else None
    w = B.mx_quantize(rhs, dim=-2)
    x = B.mx_quantize(lhs) if quantized else lhs
    got = B.mx_linear(x, w, vec, res, activation=activation, dtype=types[out])
    L, R = values(B.mx_quantize(lhs)), np.swapaxes(values(w), -1, -2)
    S = np.abs(L) @ np.abs(R)
    z = L @ R
    if bias:
        z, S = z + f64(vec), S + np.abs(f64(vec))
    f = f_of(activation, z)
    bound = 1.13 * (k + 2) * U * S + (16 * (1 + np.abs(z)) * U * np.abs(f) + U if activation in ("gelu", "silu") else 0)
    want = f
    if residual:
        want = f + f64(res)
        bound = bound + 2 * U * np.abs(want)
    check(got, want, bound, out, (b, m, k, n))
    return x, w, vec, res, got


@gpu
@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 128, 64), (2, 31, 5), (1, 2048, 128), (7, 2047, 101), (16, 256, 64), (17, 300, 65), (33, 129, 40), (64, 1024, 64), (100, 72, 56), (130, 384, 200),
                                   (300, 1000, 300), (64, 8192, 72), (257, 640, 513), (1, 16384, 33), (48, 5000, 1000), (700, 512, 900), (1100, 1280, 1030)])
def test_linear_shapes(m, k, n, quantized):
    case_linear(None, m, k, n, quantized=quantized)


@gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
def test_linear_epilogues(dtype, out, activation, bias, residual):
    case_linear(None, 20, 200, 70, dtype, out, bias=bias, residual=residual, activation=activation)
    case_linear(None, 5, 400, 66, dtype, out, bias=bias, residual=residual, activation=activation)


@gpu
@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("batched", [False, True])
@pytest.mark.parametrize("b,m,k,n,columns,gap,start", [(3, 5, 70, 33, False, 0, 0), (2, 64, 200, 100, False, 0, 0), (4, 128, 96, 64, False, 8, 0), (3, 20, 100, 300, True, 0, 0), (1, 7, 64, 64, False, 0, 0),
                                                       (2, 70, 256, 65, True, 1, 1), (5, 1, 512, 130, False, 3, 0), (2, 260, 300, 270, False, 0, 0)])
def test_linear_batches_and_strides(b, m, k, n, columns, gap, start, batched, quantized):
    case_linear(b, m, k, n, batched=batched, quantized=quantized, columns=columns, gap=gap, start=start)


@gpu
@pytest.mark.parametrize("m,k,n", [(0, 8, 8), (8, 0, 8), (8, 8, 0), (1, 0, 5), (70, 0, 70)])
def test_linear_sizes_of_zero(m, k, n):
    case_linear(None, m, k, n)
    case_linear(None, m, k, n, quantized=True, activation="relu")
    case_linear(2, m, k, n, batched=True)


@gpu
def test_quantize_sizes_of_zero():
    torch, _ = _torch()
    for shape in ((0, 40), (40, 0), (0, 3, 4), (2, 0, 8), (2, 3, 0)):
        for dim in (-1, -2):
            q = B.mx_quantize(torch.ones(shape, device="cuda"), dim=dim)
            assert q.shape == shape and B.mx_dequantize(q).shape == shape


@gpu
@pytest.mark.parametrize("m", [3, 70, 300])
def test_linear_values_that_are_not_finite(m):
    """A block that stands for NaN makes its row (lhs) or column (rhs) NaN and touches no other."""
    torch, _ = _torch()
    k, n = 300, 140
    gen = torch.Generator(device="cuda").manual_seed(3)
    lhs, rhs = torch.randn((m, k), generator=gen, device="cuda").bfloat16(), torch.randn((k, n), generator=gen, device="cuda").bfloat16()
    clean = B.mx_linear(lhs, B.mx_quantize(rhs, dim=-2))
    lhs[1, 299], rhs[130, 70] = float("inf"), float("nan")
    out = B.mx_linear(lhs, B.mx_quantize(rhs, dim=-2))
    bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    bad[1], bad[:, 70] = True, True
    assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])


@gpu
def test_linear_same_bits_and_out():
    """The same bits every time, from a lhs that is quantised before as from one that the call quantises, and out may be the residual."""
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for m, k, n in ((1, 4096, 512), (5, 8192, 256), (130, 300, 140), (2000, 512, 1000), (64, 16384, 64)):
        lhs, rhs = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((m, k), (k, n)))
        w = B.mx_quantize(rhs, dim=-2)
        acc = torch.randn((m, n), generator=gen, device="cuda")
        first = B.mx_linear(lhs, w, residual=acc, dtype=torch.float32)
        for _ in range(5):
            assert torch.equal(B.mx_linear(lhs, w, residual=acc, dtype=torch.float32), first)
        assert torch.equal(B.mx_linear(B.mx_quantize(lhs), w, residual=acc, dtype=torch.float32), first)
        assert B.mx_linear(lhs, w, residual=acc, out=acc) is acc
        assert torch.equal(acc, first)


@gpu
def test_streams_graphs_and_workspaces():
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(7)
    for m, k, n in ((4, 8192, 320), (100, 700, 300)):
        lhs, rhs = torch.randn((m, k), generator=gen, device="cuda").bfloat16(), torch.randn((k, n), generator=gen, device="cuda")
        w = B.mx_quantize(rhs, dim=-2)
        want = B.mx_linear(lhs, w, activation="gelu")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        q = B.mx_quantize(rhs, dim=-2, stream=side)
        got = B.mx_linear(lhs, q, activation="gelu", stream=side)
        back = B.mx_dequantize(q, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(q.codes, w.codes) and torch.equal(got, want) and torch.equal(back, B.mx_dequantize(w))
        work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        inputs, graphs, results = [lhs.clone(), lhs.clone()], [], []
        for x in inputs:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                results.append((B.mx_linear(x, w, activation="gelu", workspace=work), B.mx_quantize(x)))
            graphs.append(graph)
        for turn in range(4):
            for x, graph, (out, q) in zip(inputs, graphs, results):
                x.copy_(torch.randn((m, k), generator=gen, device="cuda"))
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, B.mx_linear(x, w, activation="gelu")), turn
                again = B.mx_quantize(x)
                assert torch.equal(q.codes, again.codes) and torch.equal(q.scales, again.scales)
        into = B.MX(torch.full_like(w.codes, 77), torch.full_like(w.scales, 77), k, dim=-2)
        assert B.mx_quantize(rhs, dim=-2, out=into) is into and torch.equal(into.codes, w.codes) and torch.equal(into.scales, w.scales)
        with pytest.raises(B.MorelloError) as e:         # (few rows of neighbours along k may take none)
            B.mx_linear(lhs.t().contiguous().t(), w, workspace=work[:256])
        assert e.value.code == B.E_NOMEM


@gpu
def test_block_of_the_operators():
    """A pre-norm feed-forward block: trained in bf16 for two steps, its weights put into blocks, and served.  What is served
    is the formula on the values that the blocks stand for, within a rounding of each stored step."""
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(11)
    rows, width, hidden = 70, 192, 320
    make = lambda *s: torch.randn(s, generator=gen, device="cuda") * s[0] ** -0.5       # noqa: E731
    master = [1 + 0.1 * make(width), 0.1 * make(width), make(width, hidden), 0.1 * make(hidden), make(hidden, width), 0.1 * make(width)]
    x, want = make(rows, width) * 8, make(rows, width)
    x = x.bfloat16()
    for step in range(2):
        g, c, w1, b1, w2, b2 = p = [t.bfloat16() for t in master]
        y, stats = B.layer_norm(x, g, c, stats=True)
        h, z = B.linear(y, w1, b1, activation="gelu", pre=True, dropout=0.1, seed=1, offset=step)
        out = B.linear(h, w2, b2, x)
        grad = (out.float() - want).bfloat16()
        d_h, d_w2, d_b2 = B.linear_grad(grad, h, w2, b2)
        d_y, d_w1, d_b1 = B.linear_grad(d_h, y, w1, b1, z, activation="gelu", dropout=0.1, seed=1, offset=step)
        d_x, d_g, d_c = B.layer_norm_grad(d_y, x, stats, g, c, grad)
        mask = B.dropout(torch.ones((rows, hidden), device="cuda"), dropout=0.1, seed=1, offset=step).double()
        ps = [t.double().requires_grad_() for t in [x] + p]
        mean = ps[0].mean(-1, keepdim=True)
        n = (ps[0] - mean) / ((ps[0] - mean).square().mean(-1, keepdim=True) + 1e-5).sqrt() * ps[1] + ps[2]
        o = ps[0] + torch.nn.functional.gelu(n @ ps[3] + ps[4], approximate="tanh") * mask @ ps[5] + ps[6]
        o.backward(grad.double())
        # chained bf16 roundings (y, z, h, d_h, dz, d_y, the gradients): twelve units of 2^-8, of the norm, as they are independent
        grads = [d_g, d_c, d_w1, d_b1, d_w2, d_b2]
        for got, q in zip([d_x] + grads, ps):
            assert (got.double() - q.grad).norm() <= 12 * 2.0 ** -8 * q.grad.norm()
        for t, d in zip(master, grads):
            t.add_(d.float(), alpha=-0.01)
    g, c, w1, b1, w2, b2 = [t.bfloat16() for t in master]
    q1, q2 = B.mx_quantize(w1, dim=-2), B.mx_quantize(w2, dim=-2)
    for m in (1, rows):
        y = B.layer_norm(x[:m], g, c)
        h = B.mx_linear(y, q1, b1, activation="gelu")
        out = B.mx_linear(h, q2, b2, x[:m])
        # each step from the one before it, as stored: a rounding of 2^-8 of what it stores
        z = B.mx_dequantize(B.mx_quantize(y)).double() @ B.mx_dequantize(q1).double() + b1.double()
        assert (h.double() - torch.nn.functional.gelu(z, approximate="tanh")).norm() <= 2.0 ** -8 * h.double().norm()
        o = B.mx_dequantize(B.mx_quantize(h)).double() @ B.mx_dequantize(q2).double() + b2.double() + x[:m].double()
        assert (out.double() - o).norm() <= 2.0 ** -8 * o.norm()


@gpu
def test_blocks_that_batches_share():
    """The library's `shared`, which the binding sets for rhs alone: every batch of lhs the same blocks, of rhs too, and read back."""
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(9)
    b, m, k, n = 3, 70, 200, 50
    x, w = torch.randn((m, k), generator=gen, device="cuda").bfloat16(), torch.randn((b, k, n), generator=gen, device="cuda")
    q, many = B.mx_quantize(x), B.mx_quantize(w, dim=-2)
    one = B.mx_quantize(w[0], dim=-2)
    stream = torch.cuda.current_stream().cuda_stream
    for rhs, shared in ((many, 0), (one, 1)):
        out = torch.full((b, m, n), 7.0, device="cuda")
        d = B._MX_LINEAR.pack(b, m, k, n, *B._ABSENT, q.codes.data_ptr(), q.scales.data_ptr(), 1, 0, rhs.codes.data_ptr(), rhs.scales.data_ptr(), shared, 0,
                              *B._ABSENT, *B._ABSENT, out.data_ptr(), 0, 0, n, m * n, 0, 0)
        size = C.c_size_t()
        assert B.lib().mrl_mx_linear_bytes(d, C.addressof(size)) == 0
        work = torch.empty(size.value, dtype=torch.uint8, device="cuda")
        assert B.lib().mrl_mx_linear(d, work.data_ptr() if size.value else None, size.value, stream) == 0
        want = B.mx_linear(x.expand(b, m, k), many if shared == 0 else one, dtype=torch.float32)
        assert torch.equal(out, want)
    out = torch.full((b, m, k), 7.0, device="cuda")
    assert B.lib().mrl_mx_dequantize(B._MX.pack(b, m, k, 0, out.data_ptr(), 0, 0, k, m * k, q.codes.data_ptr(), q.scales.data_ptr(), 1, 0), stream) == 0
    assert torch.equal(out, B.mx_dequantize(q, dtype=torch.float32).expand(b, m, k))


@gpu
def test_operands_that_repeat():
    """Rows and batches that are the same memory again (strides of 0) are read as they are."""
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(10)
    row, rhs = torch.randn((1, 300), generator=gen, device="cuda").bfloat16(), torch.randn((300, 90), generator=gen, device="cuda")
    w = B.mx_quantize(rhs, dim=-2)
    want = B.mx_linear(row, w)
    for m in (2, 40, 200):
        assert torch.equal(B.mx_linear(row.expand(m, 300), w), want.expand(m, 90))
        assert torch.equal(B.mx_linear(row.expand(2, m, 300), w), want.expand(2, m, 90))
        assert torch.equal(B.mx_quantize(row.expand(m, 300)).codes, B.mx_quantize(row.expand(m, 300).contiguous()).codes)


@gpu
def test_beyond_32_bits():
    """Codes and values past 4 GB: 70,000 x 131,072 values."""
    torch, _ = _torch()
    lines, k, n = 70000, 131072, 3
    x = torch.empty((lines, k), device="cuda", dtype=torch.bfloat16)
    for part in x.split(10000):
        part.normal_()
    print("quantize beyond 4 GB", flush=True)
    q = B.mx_quantize(x)
    back = B.mx_dequantize(q)
    w = B.mx_quantize(torch.randn((k, n), device="cuda"), dim=-2)
    print("product beyond 4 GB", flush=True)
    out = B.mx_linear(q, w, dtype=torch.float32)
    R = np.swapaxes(values(w), -1, -2)
    for at in (0, 16384 - 2, 32768 - 2, 65536 - 2, lines - 4):
        lines_ = f64(x[at:at + 4])
        want = read(*blocks_of(lines_), k)
        assert same(f64(back[at:at + 4]), want)
        check(out[at:at + 4], want @ R, (k + 2) * U * (np.abs(want) @ np.abs(R)), "f32", at)


@gpu
def test_refusals_of_the_binding():
    torch, _ = _torch()
    x = torch.randn((40, 96), device="cuda").bfloat16()
    q, w = B.mx_quantize(x), B.mx_quantize(x.t(), dim=-2)

    def refused(f):
        with pytest.raises(B.MorelloError) as e:
            f()
        assert e.value.code == B.E_INVAL

    for f in (lambda: B.mx_quantize(x[0]), lambda: B.mx_quantize(x.half()), lambda: B.mx_quantize(x, dim=0), lambda: B.mx_quantize(x[:, ::2]), lambda: B.mx_quantize(x.cpu()),
              lambda: B.mx_quantize(x, out=w), lambda: B.mx_quantize(x, dim=-2, out=q), lambda: B.mx_dequantize(q, dtype=torch.float16),
              lambda: B.mx_linear(x, q), lambda: B.mx_linear(w, w), lambda: B.mx_linear(x[:, :95], w), lambda: B.mx_linear(x, w, bias=x[0]), lambda: B.mx_linear(x, w, residual=x),
              lambda: B.mx_linear(x, w, activation="tanh"), lambda: B.mx_linear(x, w, dtype=torch.float16), lambda: B.mx_linear(x, w, out=torch.empty((40, 41), device="cuda")),
              lambda: B.mx_linear(x.t().contiguous().t(), w, workspace=torch.empty((1 << 12, 2), dtype=torch.uint8, device="cuda").t()),
              lambda: B.MX(q.codes, q.scales, 129), lambda: B.MX(q.codes, q.scales, 96, dim=1), lambda: B.MX(q.codes.t(), q.scales, 96), lambda: B.MX(q.codes, q.scales[:, :0], 96),
              lambda: B.MX(q.codes.int(), q.scales, 96), lambda: B.MX(q.codes, q.scales, 96, dtype=torch.float64)):
        refused(f)
    assert "MX" in repr(q)


def test_refusals_of_the_library():
    """Host code: nothing is launched (the addresses are of nothing)."""
    P, lib = 1 << 20, B.lib()
    mat = lambda d=P, t=1, l=0, ld=256, batch=0: (d, t, l, ld, batch)       # noqa: E731
    mx = lambda codes=P, scales=P, shared=0: (codes, scales, shared, 0)     # noqa: E731

    def linear(b=1, m=4, k=256, n=16, lhs=mat(), blocks=(0, 0, 0, 0), rhs=mx(), out=mat(t=0, ld=16, batch=64), act=0, work=None, have=0):
        d, size = B._MX_LINEAR.pack(b, m, k, n, *lhs, *blocks, *rhs, *B._ABSENT, *B._ABSENT, *out, act, 0), C.c_size_t()
        return lib.mrl_mx_linear_bytes(d, C.addressof(size)) or lib.mrl_mx_linear(d, work, have, None)

    rows = lambda f, b=1, lines=4, k=256, x=mat(), q=mx(): f(B._MX.pack(b, lines, k, 0, *x, *q), None)       # noqa: E731
    for rc in (linear(rhs=mx(0)), linear(rhs=mx(P, 0)), linear(rhs=mx(P + 8)), linear(rhs=mx(P, P + 2)), linear(lhs=B._ABSENT), linear(blocks=mx()), linear(lhs=mat(t=3)),
               linear(k=(1 << 24) + 1, lhs=mat(ld=1 << 25)), linear(b=1 << 20, m=1 << 20), linear(out=mat(t=0, ld=15)), linear(act=4), linear(lhs=mat(P + 1)),
               rows(lib.mrl_mx_quantize, x=mat(0)), rows(lib.mrl_mx_quantize, q=mx(0)), rows(lib.mrl_mx_quantize, q=mx(P + 4)), rows(lib.mrl_mx_quantize, b=2, q=mx(shared=1)),
               rows(lib.mrl_mx_quantize, k=1 << 25), rows(lib.mrl_mx_quantize, lines=1 << 31), rows(lib.mrl_mx_dequantize, x=mat(l=1)), rows(lib.mrl_mx_dequantize, x=mat(ld=255)),
               rows(lib.mrl_mx_dequantize, x=mat(t=2)), rows(lib.mrl_mx_dequantize, b=2, x=mat(batch=256))):
        assert rc == B.E_INVAL, lib.mrl_last_error()
    # the workspace holds lhs in blocks where its neighbours along k are not adjacent: 4 lines of 128 bytes at least
    across = mat(l=1, ld=512)
    assert linear(lhs=across) == B.E_NOMEM and linear(lhs=across, work=P, have=100) == B.E_NOMEM
    assert linear(lhs=across, work=P + 16, have=1 << 30) == B.E_INVAL
    import torch
    blocks = B.MX(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((1, 1, 4, 16, 4), dtype=torch.uint8), 100, dim=-2)
    assert blocks.shape == (100, 4) and blocks.lines == 4
    for f in (lambda: B.mx_quantize(torch.ones(2, 4)), lambda: B.mx_dequantize(blocks), lambda: B.mx_linear(torch.ones(2, 100), blocks)):
        with pytest.raises(B.MorelloError) as e:
            f()
        assert "there is no CPU path" in str(e.value)


@gpu
def test_feed_forward_example_normed_and_served():
    """The example's block behind a normalisation: its gradients are autograd's of the formula in 64 bits, and what is served is the formula on
    the values that its weights' blocks stand for."""
    import os
    import sys
    torch, _ = _torch()
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import feed_forward as F
    model = F.Normed(F.FeedForward(64, 96, 0.0, seed=3))
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, g = (torch.randn(40, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    model.scale += 0.1 * torch.randn(64, generator=gen, device="cuda")
    out, saved = model.forward(x)
    d_x, grads = model.backward(g, saved)
    b = model.block
    ps = [p.double().requires_grad_() for p in (x, model.scale, model.shift, b.w1, b.b1, b.w2, b.b2)]
    y = torch.nn.functional.layer_norm(ps[0], (64,)) * ps[1] + ps[2]
    want = ps[0] + torch.nn.functional.gelu(y @ ps[3] + ps[4], approximate="tanh") @ ps[5] + ps[6]
    want.backward(g.double())
    # chained bf16 roundings (y, z, h, out, d_h, dz, d_y, the gradients): twelve units of 2^-8, of the norm, as they are independent
    for got, p in zip([d_x] + grads, ps):
        assert got.shape == p.shape and (got.double() - p.grad).norm() <= 12 * 2.0 ** -8 * p.grad.norm()
    assert (out.double() - want).norm() <= 4 * 2.0 ** -8 * want.norm()
    served = F.Served(model)
    for m in (1, 40):
        y = B.layer_norm(x[:m], model.scale, model.shift)
        h = B.mx_linear(y, served.w1, b.b1, activation="gelu")
        o = B.mx_dequantize(B.mx_quantize(h)).double() @ B.mx_dequantize(served.w2).double() + b.b2.double() + x[:m].double()
        assert (served.token(x[:m]).double() - o).norm() <= 2.0 ** -8 * o.norm()
