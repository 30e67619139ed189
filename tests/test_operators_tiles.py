"""Every kernel that the operators' products are made of, at sizes that the rule takes it for: which one is launched (on the CPU, on a
runtime that launches nothing but counts: fake_hip.c), and what it computes against 64 bits, in every layout, with sums and tiles
that end inside a step, splits, segments and copies.

The tolerances are those of test_operators.py, with its derivation: (k + 2) u sum |products| for a sum in any order, f's slope
below 1.13 and 16 (1 + |z|) u for its evaluation, one rounding to what is stored, one of dz to the operands' type."""
import math

import pytest

from test_host_part import run_on_fake_hip
from test_operators import U, UNIT
from test_operators_edges import HOST

gpu = pytest.mark.gpu
LAYOUTS = [(0, 0), (0, 1), (1, 0), (1, 1)]

# kernel: what its mangled name holds behind the type and the layouts
KERNELS = {"256": "fast_kernelI%sELi256ELi256ELi2ELi4ELi2E", "256x128": "fast_kernelI%sELi256ELi128ELi4ELi2ELi3E", "128": "fast_kernelI%sELi128ELi128ELi2ELi4ELi2E",
           "128 alone": "fast_kernelI%sELi128ELi128ELi2ELi4ELi4E", "64": "fast_kernelI%sELi64ELi64ELi2ELi2ELi4E", "rows": "11rows_kernelI%sELi",
           "rows wide": "rows_wide_kernelI%sELi", "wide 128": "product_kernelI%sELi128ELi128ELi2ELi2ELb1E", "wide 64": "product_kernelI%sELi64ELi64ELi2ELi2ELb1E"}
TYPES = {"f32": "f", "bf16": "DF16b"}

# kernel, type, b (each batch with its own rhs), m, k, n, whether the sum is split, whether operands are copied
LINEAR = [
    ("256", "bf16", 1, 4088, 1000, 4088, False, False), ("256", "f32", 1, 4088, 1000, 4088, False, False),
    ("256", "bf16", 1, 4040, 520, 4040, False, False), ("256", "f32", 1, 1176, 456, 12536, False, False),
    ("256", "bf16", 40, 1320, 576, 160, False, False), ("256", "f32", 40, 448, 448, 720, False, False),
    ("256", "bf16", 40, 160, 14080, 168, True, False), ("256", "f32", 1, 504, 1640, 10544, True, False), ("256", "f32", 7, 496, 1744, 1472, True, False),
    ("256", "bf16", 1, 5001, 2401, 9003, False, True), ("256", "f32", 1, 5001, 2401, 9003, False, True), ("256", "f32", 1, 3457, 1771, 1481, True, True),
    ("256x128", "bf16", 1, 4088, 2536, 2040, False, False), ("256x128", "bf16", 1, 2288, 2536, 1824, False, False),
    ("256x128", "bf16", 7, 208, 2288, 2376, False, False), ("256x128", "bf16", 1, 1000, 9928, 2072, True, False),
    ("256x128", "f32", 1, 6656, 3872, 1616, True, False), ("256x128", "bf16", 1, 2373, 2281, 1753, False, True), ("256x128", "bf16", 1, 1291, 9863, 1029, True, True),
    ("128", "bf16", 1, 3000, 264, 3000, False, False), ("128", "f32", 1, 4088, 2536, 2040, False, False), ("128", "f32", 1, 976, 256, 6344, False, False),
    ("128", "bf16", 40, 208, 272, 424, False, False), ("128", "bf16", 1, 144, 5544, 5536, True, False), ("128", "f32", 1, 2280, 9848, 80, True, False),
    ("128", "bf16", 1, 3001, 1001, 3003, False, True), ("128", "f32", 1, 4701, 2303, 4097, False, True),
    ("128 alone", "bf16", 1, 2000, 264, 2040, False, False), ("128 alone", "f32", 1, 2000, 264, 2040, False, False),
    ("128 alone", "bf16", 1, 2048, 2048, 2048, False, False), ("128 alone", "f32", 1, 2048, 2048, 2048, False, False),
    ("128 alone", "bf16", 1, 136, 11848, 904, True, False), ("128 alone", "f32", 1, 2360, 1616, 400, True, False),
    ("128 alone", "bf16", 1, 2001, 4001, 2003, False, True), ("128 alone", "f32", 1, 2001, 4001, 2003, False, True),
    ("64", "bf16", 1, 1032, 200, 1032, False, False), ("64", "f32", 1, 1032, 200, 1032, False, False),
    ("64", "bf16", 1, 504, 9928, 504, True, False), ("64", "f32", 1, 504, 9928, 504, True, False), ("64", "bf16", 1, 1177, 3001, 1177, False, True),
    ("rows", "bf16", 1, 264, 4104, 264, False, False), ("rows", "f32", 1, 264, 4104, 264, True, False), ("rows", "f32", 1, 1032, 1032, 1032, False, False),
    ("rows wide", "bf16", 1, 301, 5001, 303, False, False), ("rows wide", "f32", 1, 301, 5001, 303, True, False),
    ("wide 128", "bf16", 1, 3001, 301, 3003, False, False), ("wide 128", "bf16", 7, 263, 1841, 259, True, False),
    ("wide 128", "f32", 40, 203, 361, 745, False, False), ("wide 128", "f32", 1, 367, 2237, 6937, True, False),
    ("wide 64", "bf16", 1, 1001, 777, 1011, False, False), ("wide 64", "f32", 1, 1001, 777, 1011, False, False),
    ("wide 64", "bf16", 1, 9387, 2371, 11, True, False), ("wide 64", "f32", 1, 9387, 2371, 11, True, False),
]

# kernel of d_rhs, type, b (sharing rhs, with gaps between the batches: a sum of b segments), m, k, n, activation, whether d_rhs's sum is split
SEGMENTS = [
    ("256", "bf16", 5, 200, 4088, 4088, 0, False), ("256", "f32", 5, 104, 4088, 4088, 0, False), ("256", "bf16", 7, 328, 4072, 4080, 1, False),
    ("256", "f32", 3, 136, 4072, 4080, 1, False), ("256", "f32", 6, 600, 504, 10544, 0, True), ("256x128", "bf16", 5, 520, 4088, 2040, 0, False),
    ("256x128", "bf16", 5, 520, 4088, 2040, 1, False), ("128", "bf16", 3, 88, 3000, 3000, 0, False), ("128", "f32", 5, 504, 4088, 2040, 0, False),
    ("128 alone", "bf16", 5, 72, 2000, 2040, 1, False), ("128 alone", "f32", 5, 72, 2000, 2040, 0, False), ("64", "bf16", 9, 24, 1032, 1032, 0, False),
    ("64", "f32", 9, 24, 1032, 1032, 1, False), ("wide 64", "f32", 7, 101, 1001, 1011, 0, False), ("wide 128", "bf16", 5, 61, 3001, 3003, 0, False),
]

LAUNCHED = HOST + r"""
import itertools
TYPES, KERNELS, LINEAR, SEGMENTS, LAYOUTS = eval(sys.argv[3])

def kernels():
    # all products' kernels that were launched: (kernel, type, whether lhs and rhs are adjacent along k)
    n = []
    for (name, part), (dtype, t), kc in itertools.product(KERNELS.items(), TYPES.items(), itertools.product("01", "01")):
        n += [(name, dtype, kc)] * hip.fake_launches_of((part % ("%sLb%sELb%s" % (t, *kc))).encode())
    return n

bad = []
for name, dtype, b, m, k, n, split, copied in LINEAR:
    for lhs, rhs in LAYOUTS:
        kernels(), took("copy_kernel", "rest_kernel")
        run("mrl_linear", linear(m, k, n, int(dtype == "bf16"), b, lhs, rhs, shared=b == 1))
        got = kernels(), took("copy_kernel", "rest_kernel")
        want = [(name, dtype, ("01"[not lhs], "01"[rhs]))], dict([("copy_kernel", 1)] * copied + [("rest_kernel", 1)] * split)
        if got != want: bad.append((got, want, b, m, k, n, lhs, rhs))

def with_gap(rows, columns, dtype, layout, e):
    ld = (rows if layout else columns) + e
    return P, dtype, layout, ld, (columns if layout else rows) * ld + e

for name, dtype, b, m, k, n, act, split in SEGMENTS:
    t, e = int(dtype == "bf16"), 8
    for lhs, d_rhs in LAYOUTS:
        kernels(), took("copy_kernel", "rest_kernel")
        mats = (with_gap(m, n, t, 0, e), with_gap(m, k, t, lhs, e), mat(k, n, t, d_rhs, shared=True), with_gap(m, n, t, 0, e) if act else NONE, NONE, mat(k, n, t, d_rhs, shared=True), NONE)
        run("mrl_linear_grad", B._LINEAR_GRAD.pack(b, m, k, n, *(v for x in mats for v in x), act, 0, 0, 0))
        got = kernels(), took("copy_kernel", "rest_kernel")
        kc = ("0", "01"[lhs]) if d_rhs else ("01"[lhs], "0")
        want = [(name, dtype, kc)], dict([("rest_kernel", 1)] * split)
        if got != want: bad.append((got, want, b, m, k, n, act, lhs, d_rhs))
assert not bad, "\n".join(map(str, bad))
print("done")
"""


def test_sizes_take_the_kernels_they_are_for(tmp_path):
    run_on_fake_hip(tmp_path, LAUNCHED, repr((TYPES, KERNELS, LINEAR, SEGMENTS, LAYOUTS)))


def test_every_kernel_is_aimed_at():
    """In both types, in 2 stages and 4, split and whole."""
    assert {(c[0], c[1]) for c in LINEAR} == {(name, dtype) for name in KERNELS for dtype in TYPES}
    for name in KERNELS:
        assert {c[6] for c in LINEAR if c[0] == name} == {False, True}


# ---- values

def _types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def on_gpu(gen, shape, dtype, columns=False, gap=0, scale=1.0):
    """A normal tensor, row- or column-major, with `gap` elements between its lines and its batches, NaN in them."""
    import torch
    shape = list(shape)
    if columns:
        shape[-2:] = shape[:-3:-1]
    ld = shape[-1] + gap
    strides = ([shape[-2] * ld + gap] if len(shape) == 3 else []) + [ld, 1]
    flat = torch.full((shape[0] * strides[0] + (0 if len(shape) == 3 else gap),), float("nan"), device="cuda", dtype=_types()[dtype])
    t = flat.as_strided(shape, strides)
    t.copy_(torch.randn(shape, generator=gen, device="cuda") * scale)
    return t.transpose(-1, -2) if columns else t


def product(a, b):
    """In 64 bits, batch by batch."""
    import torch
    if a.dim() == 2:
        return a.double() @ b.double()
    return torch.stack([x.double() @ (b if b.dim() == 2 else b[i]).double() for i, x in enumerate(a)])


def within(got, want, bound, dtype, what):
    import torch
    assert got.shape == want.shape
    got = got.double()
    off = ~((got - want).abs() <= bound + UNIT[dtype] * (want.abs() + bound) + 1e-37)
    assert not off.any(), (what, int(off.sum()), off.nonzero()[:4].tolist(), got[off][:4].tolist(), want[off][:4].tolist(), torch.broadcast_to(bound, want.shape)[off][:4].tolist())


@gpu
@pytest.mark.parametrize("lhs_columns,rhs_columns", LAYOUTS)
@pytest.mark.parametrize("kernel,dtype,b,m,k,n,split,copied", LINEAR)
def test_linear_of_every_kernel(kernel, dtype, b, m, k, n, split, copied, lhs_columns, rhs_columns):
    """The sum, and GELU, dropout, bias and residual behind it, z beside it."""
    import torch
    from paper_2505_01637_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    lead = (b,) if b > 1 else ()
    lhs = on_gpu(gen, lead + (m, k), dtype, lhs_columns)
    rhs = on_gpu(gen, lead + (k, n), dtype, rhs_columns, scale=k ** -0.5)
    bias, residual = on_gpu(gen, (1, n), dtype)[0], on_gpu(gen, lead + (m, n), dtype)
    kw = {"dropout": 0.25, "seed": 17, "offset": 1 << 33}
    print("linear", kernel, dtype, b, m, k, n, lhs_columns, rhs_columns, flush=True)
    out, z = B.linear(lhs, rhs, bias, residual, activation="gelu", pre=True, **kw)
    want = product(lhs, rhs) + bias.double()
    bound = (k + 2) * U * (product(lhs.abs(), rhs.abs()) + bias.double().abs())
    within(z, want, bound, dtype, "z")
    f = 0.5 * want * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (want + 0.044715 * want ** 3)))
    bound = 1.13 * bound + 16 * (1 + want.abs()) * U * f.abs() + U
    d = B.dropout(torch.ones(z.shape, device="cuda"), **kw).double()
    want, bound = f * d, d * bound + 2 * U * (f * d).abs()
    want = want + residual.double()
    within(out, want, bound + U * (want.abs() + bound), dtype, "out")
    # the sum alone is z without a bias, also where f32 is stored
    got = B.linear(lhs, rhs, dtype=torch.float32)
    within(got, product(lhs, rhs), (k + 2) * U * product(lhs.abs(), rhs.abs()), "f32", "sum")


@gpu
@pytest.mark.parametrize("lhs_columns,rhs_columns", LAYOUTS)
@pytest.mark.parametrize("kernel,dtype,b,m,k,n,act,split", SEGMENTS)
def test_gradients_over_segments_of_every_kernel(kernel, dtype, b, m, k, n, act, split, lhs_columns, rhs_columns):
    """Batches with gaps (NaN in them) that share rhs: d_rhs is one sum over all of them."""
    import torch
    from paper_2505_01637_amd import binding as B
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    gap = 8
    grad, lhs = on_gpu(gen, (b, m, n), dtype, False, gap), on_gpu(gen, (b, m, k), dtype, lhs_columns, gap)
    rhs = on_gpu(gen, (k, n), dtype, rhs_columns, scale=k ** -0.5)
    z = on_gpu(gen, (b, m, n), dtype, False, gap) if act else None
    print("linear_grad", kernel, dtype, b, m, k, n, act, lhs_columns, rhs_columns, flush=True)
    d_lhs, d_rhs, d_bias = B.linear_grad(grad, lhs, rhs, torch.ones(n, device="cuda"), z, activation=("none", "relu")[act])
    dz = grad.double() if z is None else torch.where(z > 0, grad.double(), 0.0)       # (exact in the operands' type)
    turned = rhs.t()
    within(d_lhs, product(dz, turned), (n + 2) * U * product(dz.abs(), turned.abs()), dtype, "d_lhs")
    columns = lhs.transpose(-1, -2)
    within(d_rhs, product(columns, dz).sum(0), (b * m + 2) * U * product(columns.abs(), dz.abs()).sum(0), dtype, "d_rhs")
    within(d_bias, dz.sum((0, 1)), (b * m + 2) * U * dz.abs().sum((0, 1)), "f32", "d_bias")
    assert d_rhs.stride() == rhs.stride()
