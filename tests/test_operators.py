"""The operators that Specs name, on data (binding.linear, linear_grad, dropout, dropout_grad), against plain
implementations in 64 bits.

Tolerances.  u = 2^-24 is f32's rounding unit.  A sum of k products and a bias in f32 is within
(k + 2) u of the exact one times S = sum |lhs| |rhs| + |bias|, in any order.  f's slope is below 1.13, and f's own evaluation is within
F (1 + |z|) u |f| + u; F = 16 covers an exponential of z (its argument rounded, once, at z log2 e: |z| u relative), a
reciprocal and four products.  Scale and residual add two roundings.  What is stored is rounded once more: u for f32, 2^-8 (eight bits of precision) for
bf16.  In a gradient dz is also rounded to the operands' type, which adds that unit times the sum of |products|.
"""
import math

import numpy as np
import pytest

from paper_2505_01637_amd import binding as B
from paper_2505_01637_amd import workloads as W

gpu = pytest.mark.gpu
U = 2.0 ** -24
UNIT = {"f32": U, "bf16": 2.0 ** -8}


def _torch():
    import torch
    return torch, {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- 64 bits

def random_bits(rows, cols, seed, offset, first_row=0):
    """The 16 bits of every element: the block function in 64-bit unsigned integers, for all blocks at once."""
    U64, M = np.uint64, np.uint64(0xFFFFFFFF)
    groups = (cols + 7) // 8
    c = [np.broadcast_to(np.arange(groups, dtype=U64), (rows, groups)), np.broadcast_to(np.arange(first_row, first_row + rows, dtype=U64)[:, None], (rows, groups)),
         np.full((rows, groups), offset & 0xFFFFFFFF, dtype=U64), np.full((rows, groups), offset >> 32, dtype=U64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        p0, p1 = U64(0xD2511F53) * c[0], U64(0xCD9E8D57) * c[2]         # (factors below 2^32: the products fit)
        c = [(p1 >> U64(32)) ^ c[1] ^ U64(k[0]), p1 & M, (p0 >> U64(32)) ^ c[3] ^ U64(k[1]), p0 & M]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = np.stack([w >> U64(s) & U64(0xFFFF) for w in c for s in (0, 16)], axis=-1)
    return halves.reshape(rows, groups * 8)[:, :cols].astype(np.int64)


def scale_of(shape, p, seed, offset):
    """D."""
    drop = B.drop_threshold(p)
    if drop == 0:
        return np.ones(shape)
    bits = random_bits(int(np.prod(shape[:-1])), shape[-1], seed, offset).reshape(shape)
    return np.where(bits < drop, 0.0, 65536.0 / max(1, 65536 - drop))


def f_of(act, z):
    if act == "relu":
        return np.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z / (1.0 + np.exp(-z)) if act == "silu" else z


def slope_of(act, z):
    if act == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if act == "gelu":
        u = math.sqrt(2.0 / math.pi)
        t = np.tanh(u * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * u * (1.0 + 3 * 0.044715 * z * z)
    s = 1.0 / (1.0 + np.exp(-z))
    return s * (1.0 + z * (1.0 - s)) if act == "silu" else np.ones_like(z)


def f64(t):
    return t.detach().double().cpu().numpy()


# ---- tensors of any stride inside storage whose other elements are NaN

def strided(values, dtype, columns=False, gap=0, start=0):
    """A device tensor of these values: row- or column-major, `gap` elements between lines, `start` elements into its storage."""
    torch, types = _torch()
    v = torch.from_numpy(np.ascontiguousarray(values)).to(types[dtype])
    if columns:
        v = v.transpose(-1, -2).contiguous()
    shape = list(v.shape)
    ld = shape[-1] + gap
    strides = [ld, 1] if v.dim() == 2 else [shape[-2] * ld + (3 if gap else 0), ld, 1]
    size = start + sum((n - 1) * s for n, s in zip(shape, strides)) + 1 if 0 not in shape else start + 1
    flat = torch.full((size + 5,), float("nan"), dtype=types[dtype])
    flat.as_strided(shape, strides, start).copy_(v)
    t = flat.cuda().as_strided(shape, strides, start)
    return t.transpose(-1, -2) if columns else t


def check(got, want, bound, dtype, what):
    got = f64(got)
    assert got.shape == want.shape
    allowed = bound + UNIT[dtype] * (np.abs(want) + bound) + 1e-37
    bad = np.argwhere(~(np.abs(got - want) <= allowed))
    assert bad.size == 0, (what, len(bad), bad[:4].tolist(), got[tuple(bad[0])], want[tuple(bad[0])], allowed[tuple(bad[0])])


def case_linear(b, m, k, n, dtype="f32", out=None, batched=False, lhs_columns=False, rhs_columns=False, bias=True, residual=True,
                activation="none", p=0.0, pre=True, gap=0, start=0, seed=5):
    torch, types = _torch()
    out = out or dtype
    rng = np.random.default_rng(seed)
    lead = (b,) if b is not None else ()
    lhs = strided(rng.standard_normal(lead + (m, k)), dtype, lhs_columns, gap, start)
    rhs = strided(rng.standard_normal((lead if batched else ()) + (k, n)) * max(k, 1) ** -0.5, dtype, rhs_columns, gap, start)
    bv = strided(rng.standard_normal((1, n)), dtype, start=start)[0] if bias else None
    rv = strided(rng.standard_normal(lead + (m, n)), out, False, gap, start) if residual else None
    kw = {"activation": activation, "dropout": p, "seed": 0x9E3779B97F4A7C15, "offset": (3 << 32) + 7}
    print("linear", b, m, k, n, dtype, out, batched, lhs_columns, rhs_columns, activation, p, gap, start, flush=True)
    got = B.linear(lhs, rhs, bv, rv, dtype=types[out], pre=pre, **kw)
    got, z_got = got if pre else (got, None)
    L, R = f64(lhs), f64(rhs)
    z, S = L @ R, np.abs(L) @ np.abs(R)
    if bias:
        z, S = z + f64(bv), S + np.abs(f64(bv))
    zb = (k + 2) * U * S
    if pre:
        check(z_got, z, zb, out, "pre")
    f, d = f_of(activation, z), scale_of(z.shape, p, kw["seed"], kw["offset"])
    fb = 1.13 * zb + (16 * (1 + np.abs(z)) * U * np.abs(f) + U if activation in ("gelu", "silu") else 0.0)
    want, wb = f * d, d * fb + 2 * U * np.abs(f * d)
    if residual:
        want = want + f64(rv)
        wb = wb + U * (np.abs(want) + wb)
    check(got, want, wb, out, "out")
    return lhs, rhs, bv, rv, kw, got, z_got


SHAPES = [(None, 1, 1, 1), (None, 1, 8, 8), (None, 1, 2048, 129), (None, 3, 5, 7), (None, 17, 64, 64), (None, 64, 33, 65), (None, 130, 200, 257),
          (None, 257, 65, 100), (2, 31, 40, 70), (5, 1, 100, 33)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lhs_columns,rhs_columns", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("b,m,k,n", SHAPES)
def test_linear_shapes_and_layouts(b, m, k, n, dtype, lhs_columns, rhs_columns):
    case_linear(b, m, k, n, dtype, lhs_columns=lhs_columns, rhs_columns=rhs_columns)


@gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("bias,residual,pre,p", [(False, False, False, 0.0), (True, False, True, 0.3), (False, True, False, 0.9), (True, True, True, 0.0)])
def test_linear_epilogues(dtype, out, activation, bias, residual, pre, p):
    case_linear(None, 45, 72, 83, dtype, out, activation=activation, bias=bias, residual=residual, pre=pre, p=p)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lhs_columns,rhs_columns", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("gap,start", [(1, 0), (8, 0), (8, 1), (3, 5)])
@pytest.mark.parametrize("b,batched", [(None, False), (3, False), (3, True)])
def test_linear_strides(dtype, lhs_columns, rhs_columns, gap, start, b, batched):
    """Lines with gaps (NaN in them), storage that starts anywhere, batches with gaps and a shared rhs."""
    case_linear(b, 37, 72, 40, dtype, batched=batched, lhs_columns=lhs_columns, rhs_columns=rhs_columns, gap=gap, start=start, p=0.2)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(1, 2048, 1024), (1, 4096, 16), (2, 1000, 512), (7, 2047, 1001), (16, 512, 512), (33, 8192, 64), (300, 256, 520), (512, 512, 512),
                                   (264, 96, 1032), (1, 16384, 1), (16385, 8, 1), (1000, 1, 9)])
@pytest.mark.parametrize("rhs_columns", [False, True])
def test_linear_sizes_of_every_path(dtype, m, k, n, rhs_columns):
    """Single rows, few rows over long sums, whole and ragged tiles of every size."""
    case_linear(None, m, k, n, dtype, rhs_columns=rhs_columns, activation="gelu", p=0.1 if m * n < 20000 else 0.0)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lhs_columns,rhs_columns", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("b,batched,m,k,n,gap", [(None, False, 1029, 1543, 1031, 0), (None, False, 2057, 263, 3001, 3), (None, False, 1024, 1001, 2048, 0),
                                                 (None, False, 1001, 1024, 2056, 0), (3, True, 515, 1030, 777, 0), (3, False, 515, 1030, 777, 8),
                                                 (None, False, 2000, 3, 2000, 0), (None, False, 3, 2000, 2000, 5)])
def test_large_operands_of_any_alignment(dtype, lhs_columns, rhs_columns, b, batched, m, k, n, gap):
    """Large products with one operand or both at odd strides or sizes (NaN in the gaps)."""
    case_linear(b, m, k, n, dtype, batched=batched, lhs_columns=lhs_columns, rhs_columns=rhs_columns, gap=gap, activation="silu", residual=False, pre=False)


@gpu
@pytest.mark.parametrize("m,k,n", [(0, 8, 8), (8, 0, 8), (8, 8, 0), (0, 0, 0)])
@pytest.mark.parametrize("b", [None, 0, 2])
def test_sizes_of_zero(b, m, k, n):
    """Nothing to compute, and sums over nothing: out is then residual + D f(bias), a gradient 0."""
    torch, _ = _torch()
    lhs, rhs, bias, res, kw, out, z = case_linear(b, m, k, n, "bf16", activation="silu", p=0.5)
    grad = torch.ones_like(out)
    d_lhs, d_rhs, d_bias = B.linear_grad(grad, lhs, rhs, bias, z, **kw)
    assert d_lhs.shape == lhs.shape and d_rhs.shape == rhs.shape and d_bias.shape == bias.shape
    if 0 in (m, n, b):
        assert not d_rhs.any() and not d_bias.any() and not d_lhs.any()


def plain_grad(grad, lhs, rhs, z, act, d):
    dz = grad * d * slope_of(act, z)
    return dz, dz @ np.swapaxes(rhs, -1, -2), np.swapaxes(lhs, -1, -2) @ dz


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lhs_columns,rhs_columns", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("activation,p", [("none", 0.0), ("none", 0.4), ("relu", 0.0), ("gelu", 0.25), ("silu", 0.0)])
@pytest.mark.parametrize("b,batched,m,k,n,gap", [(None, False, 1, 64, 40, 0), (None, False, 70, 33, 90, 1), (None, False, 130, 136, 264, 8), (3, False, 33, 40, 24, 0),
                                                 (3, False, 33, 40, 24, 8), (3, True, 33, 40, 24, 0), (2, True, 65, 17, 9, 3), (None, False, 131, 1027, 1501, 0)])
def test_gradients_of_the_formula(dtype, lhs_columns, rhs_columns, activation, p, b, batched, m, k, n, gap):
    torch, _ = _torch()
    rng = np.random.default_rng(11)
    lead = (b,) if b is not None else ()
    lhs = strided(rng.standard_normal(lead + (m, k)), dtype, lhs_columns, gap)
    rhs = strided(rng.standard_normal((lead if batched else ()) + (k, n)) * k ** -0.5, dtype, rhs_columns, gap)
    bias = strided(rng.standard_normal((1, n)), "f32")[0]
    grad = strided(rng.standard_normal(lead + (m, n)), dtype, False, gap)
    z = strided(rng.standard_normal(lead + (m, n)), dtype, False, gap)
    kw = {"activation": activation, "dropout": p, "seed": 99, "offset": 1 << 40}
    print("linear_grad", b, batched, m, k, n, dtype, lhs_columns, rhs_columns, activation, p, gap, flush=True)
    d_lhs, d_rhs, d_bias = B.linear_grad(grad, lhs, rhs, bias, z, **kw)
    G, L, R, Z = f64(grad), f64(lhs), f64(rhs), f64(z)
    d = scale_of(G.shape, p, 99, 1 << 40)
    dz, want_l, want_r = plain_grad(G, L, R, Z, activation, d)
    if b is not None and not batched:
        want_r = want_r.sum(0)
    # dz before it is rounded: the slope's evaluation is within 64 (1 + |z|)^3 u of it (two terms, each with an exponential, z^3 in GELU's), then two products
    db = np.abs(G * d) * (64 * (1 + np.abs(Z)) ** 3 * U if activation in ("gelu", "silu") else 0.0) + 2 * U * np.abs(dz)
    rounded = db + UNIT[dtype] * (np.abs(dz) + db)
    s_l = rounded @ np.abs(np.swapaxes(R, -1, -2)) + (n + 2) * U * (np.abs(dz) @ np.abs(np.swapaxes(R, -1, -2)))
    s_r = np.swapaxes(np.abs(L), -1, -2) @ rounded + ((b or 1) * m + 2) * U * (np.swapaxes(np.abs(L), -1, -2) @ np.abs(dz))
    if b is not None and not batched:
        s_r = s_r.sum(0)
    check(d_lhs, want_l, s_l, dtype, "d_lhs")
    check(d_rhs, want_r, s_r, dtype, "d_rhs")
    axes = tuple(range(G.ndim - 1))
    check(d_bias, dz.sum(axes), db.sum(axes) + ((b or 1) * m + 2) * U * np.abs(dz).sum(axes), "f32", "d_bias")
    # one wanted at a time: the same bits
    only, none, no_bias = B.linear_grad(grad, lhs, rhs, None, z, need_rhs=False, **kw)
    assert torch.equal(only, d_lhs) and none is None and no_bias is None
    none, only, _ = B.linear_grad(grad, lhs, rhs, None, z, need_lhs=False, **kw)
    assert torch.equal(only, d_rhs) and none is None
    none, none2, only = B.linear_grad(grad, lhs, rhs, bias, z, need_lhs=False, need_rhs=False, **kw)
    assert none is None and none2 is None and torch.equal(only, d_bias)


@gpu
@pytest.mark.parametrize("activation,p", [("gelu", 0.3), ("silu", 0.0), ("none", 0.5)])
def test_gradients_against_differences(activation, p):
    """d/dt of sum(grad * linear(lhs + t v, rhs + t w, bias + t c)) at 0 by a central difference in 64 bits of the formula, against the
    gradients' products with v, w, c.  The difference's own error is t^2 / 6 times a third derivative of order 1 per element: with t = 1e-4
    below 1e-7 of the sum of magnitudes; the gradients' is that of f32."""
    torch, _ = _torch()
    rng = np.random.default_rng(3)
    m, k, n, t = 20, 30, 25, 1e-4
    L, R, c0 = rng.standard_normal((m, k)), rng.standard_normal((k, n)) * k ** -0.5, rng.standard_normal(n)
    L, R, c0 = (x.astype(np.float32).astype(np.float64) for x in (L, R, c0))
    v, w, c, G = rng.standard_normal((m, k)), rng.standard_normal((k, n)) * k ** -0.5, rng.standard_normal(n), rng.standard_normal((m, n)).astype(np.float32)
    kw = {"activation": activation, "dropout": p, "seed": 4, "offset": 2}
    d = scale_of((m, n), p, 4, 2)
    value = lambda s: (G * d * f_of(activation, (L + s * v) @ (R + s * w) + c0 + s * c)).sum()
    slope = (value(t) - value(-t)) / (2 * t)
    dev = lambda x: torch.from_numpy(x.astype(np.float32)).cuda()
    lhs, rhs, bias, grad = dev(L), dev(R), dev(c0), dev(G)
    out, z = B.linear(lhs, rhs, bias, pre=True, **kw)
    d_lhs, d_rhs, d_bias = (f64(x) for x in B.linear_grad(grad, lhs, rhs, bias, z, **kw))
    parts = (d_lhs * v).sum(), (d_rhs * w).sum(), (d_bias * c).sum()
    size = np.abs(d_lhs * v).sum() + np.abs(d_rhs * w).sum() + np.abs(d_bias * c).sum()
    assert abs(sum(parts) - slope) <= 2e-5 * size


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 2048), (3, 7), (64, 8), (33, 4099), (2, 5, 9), (300, 1)])
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 1.0])
def test_dropout(dtype, shape, p):
    torch, _ = _torch()
    rng = np.random.default_rng(8)
    x, res = strided(rng.standard_normal(shape), dtype), strided(rng.standard_normal(shape), dtype)
    print("dropout", dtype, shape, p, flush=True)
    out = B.dropout(x, res, dropout=p, seed=(1 << 64) - 1, offset=5)
    d = scale_of(shape, p, (1 << 64) - 1, 5)
    want = f64(x) * d + f64(res)
    check(out, want, 3 * U * (np.abs(f64(x) * d) + np.abs(want)), dtype, "dropout")
    g = B.dropout_grad(x, dropout=p, seed=(1 << 64) - 1, offset=5)
    check(g, f64(x) * d, 2 * U * np.abs(f64(x) * d), dtype, "dropout_grad")
    # in place, over rows with gaps
    wide = torch.zeros(shape[:-1] + (shape[-1] + 3,), dtype=x.dtype, device=x.device)
    part = wide[..., :shape[-1]]
    part.copy_(x)
    B.dropout(part, res, dropout=p, seed=(1 << 64) - 1, offset=5, out=part)
    assert torch.equal(part, out) and not wide[..., shape[-1]:].any()


@gpu
def test_dropout_share_and_independence():
    """2^20 elements: the share that is dropped is binomial, 6 standard deviations; other seeds and offsets drop others."""
    torch, _ = _torch()
    x = torch.ones((1024, 1024), device="cuda")
    kept = [B.dropout(x, dropout=0.3, seed=s, offset=o) != 0 for s, o in ((1, 0), (2, 0), (1, 1), (1 + (1 << 32), 0))]
    q = 1 - B.drop_threshold(0.3) / 65536
    for a in kept:
        assert abs(a.double().mean().item() - q) < 6 * math.sqrt(q * (1 - q) / 2 ** 20)
    for i, a in enumerate(kept):
        for b in kept[:i]:
            both = (a & b).double().mean().item()
            assert abs(both - q * q) < 6 * math.sqrt(q * q * (1 - q * q) / 2 ** 20)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_with_dropout_is_linear_then_dropout(dtype):
    torch, types = _torch()
    gen = torch.Generator(device="cuda").manual_seed(2)
    lhs, rhs = (torch.randn(s, generator=gen, device="cuda").to(types[dtype]) for s in ((3, 50, 64), (64, 99)))
    res = torch.randn((3, 50, 99), generator=gen, device="cuda")
    kw = {"dropout": 0.37, "seed": 77, "offset": 12}
    whole = B.linear(lhs, rhs, residual=res, dtype=torch.float32, **kw)
    parts = B.dropout(B.linear(lhs, rhs, dtype=torch.float32), res, **kw)
    assert torch.equal(whole == res, parts == res)
    assert (whole - parts).abs().max().item() <= 4 * U * (whole.abs() + res.abs()).max().item()


@gpu
def test_operands_beyond_32_bits():
    """Offsets past 4 GB: the last rows of a product over 4.6 GB, a gradient that sums over them, a dropout of as much; every part
    against 64 bits.  (d_rhs adds 1,130,000 products: u times their number times the sum of magnitudes bounds it.)"""
    torch, _ = _torch()
    m, k, n = 1130000, 2048, 24
    gen = torch.Generator(device="cuda").manual_seed(1)
    lhs = torch.empty((m, k), device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    rhs = torch.randn((k, n), generator=gen, device="cuda").bfloat16()
    grad = torch.randn((m, n), generator=gen, device="cuda").bfloat16()
    print("linear beyond 4 GB", flush=True)
    out = B.linear(lhs, rhs, dtype=torch.float32)
    for at in (0, 524288 - 50, 1048576 - 50, m - 100):          # around 2 GB, around 4 GB, the end
        L, R = f64(lhs[at:at + 100]), f64(rhs)
        check(out[at:at + 100], L @ R, (k + 2) * U * (np.abs(L) @ np.abs(R)), "f32", at)
    _, d_rhs, _ = B.linear_grad(grad, lhs, rhs, need_lhs=False)
    want = sum(a.double().t() @ g.double() for a, g in zip(lhs.split(100000), grad.split(100000)))
    size = sum(a.abs().double().t() @ g.abs().double() for a, g in zip(lhs.split(100000), grad.split(100000)))
    check(d_rhs, f64(want), f64(size) * (m + 2) * U, "bf16", "d_rhs")
    assert (d_rhs.double() - want).norm() <= 2.0 ** -8 * want.norm()
    d_lhs, _, _ = B.linear_grad(grad, lhs, rhs, need_rhs=False)
    G = f64(grad[-100:])
    check(d_lhs[-100:], G @ f64(rhs).T, (n + 2) * U * (np.abs(G) @ np.abs(f64(rhs)).T), "bf16", "d_lhs")
    dropped = B.dropout(lhs, dropout=0.25, seed=9)
    bits = random_bits(3, k, 9, 0, first_row=m - 3)
    want = np.where(bits < 16384, 0.0, f64(lhs[-3:]) * 65536 / 49152)
    check(dropped[-3:], want, 2 * U * np.abs(want), "bf16", "dropout")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite(dtype):
    """Infinities and NaN go where the formula takes them; where an element is dropped there is the residual, whatever was dropped."""
    torch, types = _torch()
    k, n = 64, 48
    lhs = torch.ones((4, k), device="cuda", dtype=types[dtype])
    rhs = torch.ones((k, n), device="cuda", dtype=types[dtype])
    lhs[1, 3], lhs[2, 5], lhs[3, 7] = float("inf"), float("-inf"), float("nan")
    inf = float("inf")
    want = {"none": [64.0, inf, -inf], "relu": [64.0, inf, 0.0], "gelu": [64.0, inf, 0.0], "silu": [64.0, inf, 0.0]}
    for act, (one, plus, minus) in want.items():
        out = B.linear(lhs, rhs, activation=act).float()
        assert (out[0] == one).all() and (out[1] == plus).all() and (out[2] == minus).all() and out[3].isnan().all(), act
    res = torch.full((4, n), 2.0, device="cuda", dtype=types[dtype])
    assert torch.equal(B.linear(lhs, rhs, residual=res, dropout=1.0), res)
    out = B.linear(lhs, rhs, residual=res, dropout=0.5, seed=6).float()
    dropped = torch.from_numpy(scale_of((4, n), 0.5, 6, 0) == 0).cuda()
    assert (out[dropped] == 2.0).all() and not out[1:][~dropped[1:]].isfinite().any()
    x = torch.full((4, n), float("nan"), device="cuda", dtype=types[dtype])
    out = B.dropout(x, res, dropout=0.5, seed=6).float()
    assert (out[dropped] == 2.0).all() and out[~dropped].isnan().all()
    # a slope where z is infinite: 1 or 0, no NaN
    z = torch.tensor([[inf, -inf, 0.0, 1e30, -1e30, 300.0, -300.0, 88.0]], device="cuda", dtype=types[dtype])
    grad = torch.ones_like(z)
    eye = torch.eye(8, device="cuda", dtype=types[dtype])
    for act, at0 in (("relu", 0.0), ("gelu", 0.5), ("silu", 0.5)):
        d_lhs, _, _ = B.linear_grad(grad, eye[:1], eye, None, z, activation=act, need_rhs=False)
        assert d_lhs.float().tolist() == [[1.0, 0.0, at0, 1.0, 0.0, 1.0, 0.0, 1.0]], act


@gpu
def test_nan_beside_the_operands_does_not_reach_the_sums():
    """k that ends inside a step along k: what lies behind it in memory, NaN here, counts nothing."""
    for k in (1, 7, 8, 31, 33, 63, 65, 120, 127):
        for dtype in ("f32", "bf16"):
            for lc in (False, True):
                for rc in (False, True):
                    case_linear(None, 66, k, 70, dtype, lhs_columns=lc, rhs_columns=rc, gap=8, pre=False, seed=k)


@gpu
def test_same_bits_every_time_and_out_may_be_the_residual():
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for m, k, n in ((1, 4096, 512), (5, 8192, 256), (130, 300, 140)):
        lhs, rhs = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((m, k), (k, n)))
        acc = torch.randn((m, n), generator=gen, device="cuda")
        first = B.linear(lhs, rhs, residual=acc, dtype=torch.float32, dropout=0.1)
        for _ in range(5):
            assert torch.equal(B.linear(lhs, rhs, residual=acc, dtype=torch.float32, dropout=0.1), first)
        assert B.linear(lhs, rhs, residual=acc, out=acc, dropout=0.1) is acc
        assert torch.equal(acc, first)


@gpu
def test_streams_graphs_and_workspaces():
    """On another stream; captured into a graph and replayed with other inputs; with a workspace the caller keeps."""
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(7)
    m, k, n = 4, 4096, 640
    lhs, rhs = torch.randn((m, k), generator=gen, device="cuda"), torch.randn((k, n), generator=gen, device="cuda") * 0.02
    bias = torch.randn((n,), generator=gen, device="cuda")
    kw = {"activation": "gelu", "dropout": 0.2, "seed": 3}
    want, z = B.linear(lhs, rhs, bias, pre=True, **kw)
    grads = B.linear_grad(want, lhs, rhs, bias, z, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = B.linear(lhs, rhs, bias, stream=side, **kw)
    side.synchronize()
    assert torch.equal(out, want)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    assert torch.equal(B.linear(lhs, rhs, bias, workspace=ws, **kw), want)
    with pytest.raises(B.MorelloError) as e:
        B.linear_grad(want, lhs, rhs, bias, z, workspace=ws[:16], **kw)
    assert e.value.code == B.E_NOMEM
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g_out, g_z = B.linear(lhs, rhs, bias, pre=True, **kw)
        g_grads = B.linear_grad(g_out, lhs, rhs, bias, g_z, **kw)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(g_out, want)
        for a, b in zip(g_grads, grads):
            assert torch.equal(a, b)
        lhs.mul_(0.5)
        want, z = B.linear(lhs, rhs, bias, pre=True, **kw)
        grads = B.linear_grad(want, lhs, rhs, bias, z, **kw)


@gpu
def test_operator_of_a_spec():
    """Table.apply: the fused configuration's goal and a Matmul's Spec with layouts, on data."""
    torch, _ = _torch()
    target, tabs = B.solve_config(W.config(5, max_size=16))
    gen = torch.Generator(device="cuda").manual_seed(1)
    lhs, rhs, bias = (torch.randn(s, generator=gen, device="cuda") for s in ((8, 16), (4, 16), (4,)))
    rhs = rhs.t()
    x = tabs["F"].coord_of_spec((1, 8, 16, 4), (3, 3, 3, 3, 3), layouts=(0, 1, 0, 0))
    out = tabs["F"].apply(x, lhs, rhs, bias)
    want = np.maximum(f64(lhs) @ f64(rhs) + f64(bias), 0)
    assert np.abs(f64(out) - want).max() < 20 * U * (np.abs(f64(lhs)) @ np.abs(f64(rhs)) + np.abs(f64(bias))).max()
    y = tabs["M"].coord_of_spec((1, 8, 16, 4), (3, 3, 3), layouts=(0, 1, 0))
    acc = torch.ones((8, 4), device="cuda")
    assert tabs["M"].apply(y, lhs, rhs, out=acc) is acc
    assert np.abs(f64(acc) - 1 - f64(lhs) @ f64(rhs)).max() < 20 * U * (1 + np.abs(f64(lhs)) @ np.abs(f64(rhs))).max()
    for bad in (lambda: tabs["F"].apply(x, lhs, rhs),                               # no bias
                lambda: tabs["M"].apply(y, lhs, rhs, bias),                         # one too many
                lambda: tabs["M"].apply(y, lhs[:4], rhs),                           # another shape
                lambda: tabs["M"].apply(y, lhs, rhs.contiguous()),                  # another layout
                lambda: tabs["M"].apply(y, lhs.bfloat16(), rhs.bfloat16()),         # another type
                lambda: tabs["E"].apply(x, lhs, rhs, bias)):                        # no Matmul
        with pytest.raises(B.MorelloError):
            bad()


@gpu
def test_refusals_of_the_binding():
    torch, _ = _torch()
    a, b = torch.zeros((4, 8), device="cuda"), torch.zeros((8, 6), device="cuda")
    for bad in (lambda: B.linear(a, b.bfloat16()), lambda: B.linear(a, b[:7]), lambda: B.linear(a.double(), b.double()),
                lambda: B.linear(a.cpu(), b), lambda: B.linear(a, b.cpu()), lambda: B.linear(a, b, activation="tanh"),
                lambda: B.linear(a, b, dropout=1.5), lambda: B.linear(a, b, dropout=float("nan")), lambda: B.linear(a, b, dropout=0.1, seed=1 << 64),
                lambda: B.linear(a, b, offset=-1), lambda: B.linear(a, b, torch.zeros(5, device="cuda")),
                lambda: B.linear(a, b, residual=torch.zeros((4, 5), device="cuda")), lambda: B.linear(a, b, out=torch.zeros((6, 4), device="cuda").t()),
                lambda: B.linear(torch.zeros((4, 16), device="cuda")[:, ::2], torch.zeros((8, 6), device="cuda")),
                lambda: B.linear(a, b, out=torch.zeros((1, 6), device="cuda").expand(4, 6)),
                lambda: B.linear(a[None].expand(3, 4, 8), b[None].expand(2, 8, 6)), lambda: B.linear_grad(torch.zeros((4, 6), device="cuda"), a, b, activation="gelu"),
                lambda: B.linear_grad(torch.zeros((4, 5), device="cuda"), a, b), lambda: B.dropout(a[0], dropout=0.1),
                lambda: B.dropout(a.t(), dropout=0.1), lambda: B.dropout(torch.zeros((2, 3, 8), device="cuda")[:, :2], dropout=0.1)):
        with pytest.raises(B.MorelloError) as e:
            bad()
        assert e.value.code == B.E_INVAL


# ---- the C entry points' own refusals: no device work, no GPU needed

def _linear_desc(b=1, m=4, k=8, n=6, act=0, drop=0, **mats):
    def mat(name, ld, layout=0, dtype=0, batch=0, data=256):
        return tuple(mats.get(name, (data, dtype, layout, ld, batch)))
    none = (0, 0, 0, 0, 0)
    return B._LINEAR.pack(b, m, k, n, *mat("lhs", k, batch=m * k), *mat("rhs", n), *mats.get("bias", none), *mats.get("residual", none),
                          *mat("out", n, batch=m * n), *mats.get("pre", none), act, drop, 0, 0)


def test_refusals_of_the_library():
    import ctypes as C
    lib = B.lib()
    size = C.c_size_t()

    def linear(raw):
        return lib.mrl_linear(raw, None, C.c_size_t(0), None), lib.mrl_last_error().decode()
    assert lib.mrl_linear(None, None, C.c_size_t(0), None) == B.E_INVAL
    assert lib.mrl_linear_bytes(None, C.byref(size)) == B.E_INVAL
    assert lib.mrl_linear_grad(None, None, C.c_size_t(0), None) == B.E_INVAL
    assert lib.mrl_dropout(None, None) == B.E_INVAL
    for part, raw in (("unknown activation", _linear_desc(act=4)), ("above 65536", _linear_desc(drop=65537)), ("2^31", _linear_desc(m=1 << 31)),
                      ("2^31", _linear_desc(b=1 << 16, m=1 << 15)), ("lhs is NULL", _linear_desc(lhs=(0, 0, 0, 8, 0))),
                      ("two types", _linear_desc(lhs=(256, 1, 0, 8, 0))), ("not aligned", _linear_desc(lhs=(258, 0, 0, 8, 0))),
                      ("layout", _linear_desc(out=(256, 0, 1, 4, 0))), ("overlap", _linear_desc(out=(256, 0, 0, 5, 0))),
                      ("overlap", _linear_desc(b=2, out=(256, 0, 0, 6, 6))), ("negative", _linear_desc(lhs=(256, 0, 0, -8, 0))),
                      ("unknown type", _linear_desc(out=(256, 2, 0, 6, 0))), ("bias is not aligned", _linear_desc(bias=(257, 1, 0, 1, 0)))):
        rc, message = linear(raw)
        assert rc == B.E_INVAL and part in message, (part, message)
    # a workspace that is too small, or not there
    raw = _linear_desc(m=1, k=1 << 16, n=64, out=(256, 0, 0, 64, 0), lhs=(256, 0, 0, 1 << 16, 0), rhs=(256, 0, 0, 64, 0))
    assert lib.mrl_linear_bytes(raw, C.byref(size)) == B.OK
    if size.value:
        assert lib.mrl_linear(raw, C.c_void_p(256), C.c_size_t(size.value - 1), None) == B.E_NOMEM
        assert lib.mrl_linear(raw, None, size, None) == B.E_INVAL
        assert lib.mrl_linear(raw, C.c_void_p(264), size, None) == B.E_INVAL


def test_drop_threshold():
    assert [B.drop_threshold(p) for p in (0.0, 1e-6, 1 / 65536, 0.1, 0.5, 1.0)] == [0, 0, 1, 6554, 32768, 65536]
    for p in (-0.1, 1.1, float("nan"), float("inf")):
        with pytest.raises(B.MorelloError):
            B.drop_threshold(p)


def test_operators_refuse_the_cpu():
    torch, _ = _torch()
    a = torch.zeros((2, 2))
    for call in (lambda: B.linear(a, a), lambda: B.linear_grad(a, a, a), lambda: B.dropout(a, dropout=0.1), lambda: B.dropout_grad(a, dropout=0.1)):
        with pytest.raises(B.MorelloError) as e:
            call()
        assert e.value.code == B.E_INVAL and "no CPU path" in str(e.value)
