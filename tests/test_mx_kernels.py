"""Every kernel of mx_linear by its launch (without a GPU, on a runtime that counts) and by values, with edges and sums that are split; what
layer_norm and the quantisation launch; results that are stored past the caches (11 to 32 MB, or 256 and more), at any alignment."""
import pytest

from paper_2505_01637_amd import binding as B
from test_host_part import run_on_fake_hip
from test_operators import U, UNIT

gpu = pytest.mark.gpu

# (kernel, m, k, n, sums are split)
KERNELS = [
    ("mx_tile_kernelILi256ELi256E", 4000, 700, 4090, False), ("mx_tile_kernelILi256ELi256E", 2040, 12288, 2050, True),
    ("mx_tile_kernelILi256ELi128E", 2000, 9000, 4090, False),
    ("mx_tile_kernelILi128ELi128ELi2ELi2E", 4100, 300, 4100, False), ("mx_tile_kernelILi128ELi128ELi2ELi2E", 3000, 32768, 250, True),
    ("mx_tile_kernelILi128ELi128ELi2ELi4E", 2000, 600, 2040, False), ("mx_tile_kernelILi128ELi128ELi2ELi4E", 1000, 16384, 1020, True),
    ("mx_tile_kernelILi64E", 700, 500, 900, False), ("mx_tile_kernelILi64E", 300, 16400, 301, True),
    ("mx_rows_kernel", 3, 1000, 1000, False), ("mx_rows_kernel", 16, 4100, 4096, False), ("mx_rows_kernel", 300, 1000, 300, False), ("mx_rows_kernel", 1, 20000, 100, True),
]

BODY = r"""
import ctypes as C, sys
sys.path.insert(0, sys.argv[2])
sys.modules["torch"] = None                       # (its own runtime would be loaded first)
hip = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
from paper_2505_01637_amd import binding as B
lib = B.lib()
NONE, P = (0, 0, 0, 0, 0), 1 << 20                # (addresses that nothing reads)
NAMES = ("mx_tile_kernelILi256ELi256E", "mx_tile_kernelILi256ELi128E", "mx_tile_kernelILi128ELi128ELi2ELi2E", "mx_tile_kernelILi128ELi128ELi2ELi4E", "mx_tile_kernelILi64E",
         "mx_rows_kernel", "mx_quantize_across", "mx_quantize_kernel", "mx_dequantize", "rest_kernel", "norm_grad_rows", "norm_columns", "norm_sums", "norm_grad_kernel", "norm_grad_few", "norm_few", "norm_rows",
         "norm_kernel")

def took():
    n = {k: hip.fake_launches_of(k.encode()) for k in NAMES}
    return {k: v for k, v in n.items() if v}

def linear(m, k, n, dtype=1, blocks=False, columns=False, b=1):
    lhs = NONE if blocks else (P, dtype, 1, m, m * k) if columns else (P, dtype, 0, k, m * k)
    d = B._MX_LINEAR.pack(b, m, k, n, *lhs, *((P, P) if blocks else (0, 0)), 0, 0, P, P, 1, 0, *NONE, *NONE, P, 1, 0, n, m * n, 0, 0)
    size = C.c_size_t()
    assert lib.mrl_mx_linear_bytes(d, C.addressof(size)) == 0, lib.mrl_last_error()
    if size.value:
        assert lib.mrl_mx_linear(d, P, size.value - 1, None) == B.E_NOMEM
    assert lib.mrl_mx_linear(d, P, size.value, None) == 0, lib.mrl_last_error()
    return took(), size.value

def norm(m, n, dtype=1, b=1):
    x = (P, dtype, 0, n, m * n)
    assert lib.mrl_layer_norm(B._NORM.pack(b, m, n, 1e-5, *x, *x, *NONE, *NONE, P), None) == 0, lib.mrl_last_error()
    return took()

def grad(m, n, dtype=1, x=True, sums=True):
    t = (P, dtype, 0, n, m * n)
    d = B._NORM_GRAD.pack(1, m, n, 0, *t, *t, *NONE, *NONE, *(t if x else NONE), *((P, 0, 0, 1, 0) if sums else NONE), *((P, 0, 0, 1, 0) if sums else NONE), P)
    size = C.c_size_t()
    assert lib.mrl_layer_norm_grad_bytes(d, C.addressof(size)) == 0, lib.mrl_last_error()
    if size.value:
        assert lib.mrl_layer_norm_grad(d, P, size.value - 1, None) == B.E_NOMEM
    assert lib.mrl_layer_norm_grad(d, P, size.value, None) == 0, lib.mrl_last_error()
    return took(), size.value

took()
for kernel, m, k, n, split in KERNELS_HERE:
    got, size = linear(m, k, n, blocks=True)
    assert got == ({kernel: 1, "rest_kernel": 1} if split else {kernel: 1}), (kernel, m, k, n, got)
    assert (size > 0) == split, (m, k, n, size)
    got, _ = linear(m, k, n, columns=True)
    assert got.get("mx_quantize_across") == 1, (m, k, n, got)
for i, (b, m, k, n) in enumerate(SEVERAL_HERE):
    got, size = linear(m, k, n, blocks=True, b=b)
    assert got == {"mx_tile_kernelILi256ELi256E" if i < 4 else "mx_tile_kernelILi128ELi128ELi2ELi2E": 1} and size == 0, (b, m, k, n, got)
# a token: one launch, no workspace, from either type
for dtype in (0, 1):
    assert linear(1, 2048, 16384, dtype) == ({"mx_rows_kernel": 1}, 0)
    assert linear(7, 2047, 1001, dtype) == ({"mx_rows_kernel": 1}, 0)
assert linear(1, 7, 64)[0] == {"mx_rows_kernel": 1, "mx_quantize_kernel": 1}, "lines of fewer than eight values are put into blocks by a launch of their own"
assert linear(16, 16384, 16384)[0].get("mx_quantize_kernel"), "as are those that shared memory does not hold"
# batches that share rhs are one product
assert linear(4, 256, 256, b=8)[0] == {"mx_rows_kernel": 1}
assert linear(0, 8, 8) == ({}, 0) and linear(8, 8, 0) == ({}, 0) and linear(8, 0, 8)[0], "a sum over nothing still has an epilogue"
q = lambda lib_call, x: lib_call(B._MX.pack(1, 100, 300, 0, *x, P, P, 0, 0), None)
assert q(lib.mrl_mx_quantize, (P, 1, 0, 300, 0)) == 0 and took() == {"mx_quantize_kernel": 1}
assert q(lib.mrl_mx_quantize, (P, 0, 1, 100, 0)) == 0 and took() == {"mx_quantize_across": 1}
assert q(lib.mrl_mx_dequantize, (P, 0, 0, 300, 0)) == 0 and took() == {"mx_dequantize": 1}
# rows in registers from 8 to 16384 elements
for m, n in ((1, 8), (5, 128), (8192, 2048), (3, 16384)):
    assert norm(m, n) == {"norm_rows": 1}, (m, n)
for m, n in ((1, 1), (100, 7)):
    assert norm(m, n) == {"norm_few": 1}, (m, n)
assert norm(2, 16385) == {"norm_kernel": 1}
assert norm(0, 8) == {} and norm(8, 0) == {}
for m, n in ((1, 2048), (8, 1000), (64, 128), (4, 16384)):
    assert grad(m, n) == ({"norm_grad_rows": 1}, 0), "the sums of few rows need no second launch"
got, size = grad(8192, 2048)
assert got == {"norm_grad_rows": 1, "norm_sums": 1} and size == 256 * 2 * 2048 * 4
assert grad(8192, 2048, sums=False) == ({"norm_grad_rows": 1}, 0) and grad(8192, 2048, x=False)[0] == {"norm_grad_rows": 1, "norm_sums": 1}
assert grad(100, 20000) == ({"norm_grad_kernel": 1, "norm_columns": 1, "norm_sums": 1}, 2 * 2 * 20000 * 4)
assert grad(64, 5)[0] == {"norm_grad_few": 1, "norm_columns": 1}
assert grad(100, 64, x=False, sums=False) == ({}, 0) and grad(5, 0) == ({}, 0)
assert grad(0, 64) == ({"norm_grad_rows": 1}, 0), "the sums over no rows are zeros"
print("done")
"""


def test_what_is_launched(tmp_path):
    run_on_fake_hip(tmp_path, BODY.replace("KERNELS_HERE", repr(KERNELS)).replace("SEVERAL_HERE", repr(SEVERAL)))


def close(got, want, bound, dtype):
    """All on the GPU, in 64 bits: |got - want| <= bound, and a rounding of what is stored."""
    assert ((got.double() - want).abs() <= bound + UNIT[dtype] * (want.abs() + bound) + 1e-37).all()


# More tiles than run at once, of 256 x 256 and of 128 x 128; sums of two steps, of a step's part more, and of more.
SEVERAL = [(1, 8000, 512, 4090), (1, 8192, 520, 4096), (2, 4000, 1030, 4001), (1, 32700, 300, 1000), (1, 4224, 512, 4224), (1, 4190, 700, 4221), (3, 2400, 512, 2408)]


@gpu
@pytest.mark.parametrize("kernel,m,k,n,split", KERNELS, ids=["%s-%d-%d-%d" % (c[0][3:].split("E")[0] + c[0][-8:], *c[1:4]) for c in KERNELS])
def test_every_kernel(kernel, m, k, n, split):
    """bf16 with bias and residual from a matrix, f32 from blocks; the tolerance is that of k products in f32."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    x, w = torch.randn((m, k), generator=gen, device="cuda"), B.mx_quantize(torch.randn((k, n), generator=gen, device="cuda") * k ** -0.5, dim=-2)
    x = (x * torch.exp(torch.randn(k, generator=gen, device="cuda"))).bfloat16()
    bias, res = torch.randn(n, generator=gen, device="cuda"), torch.randn((m, n), generator=gen, device="cuda").bfloat16()
    q = B.mx_quantize(x)
    L, R = B.mx_dequantize(q).double(), B.mx_dequantize(w, dtype=torch.float32).double().contiguous()
    z, S = L @ R, L.abs() @ R.abs()
    close(B.mx_linear(q, w, dtype=torch.float32), z, (k + 2) * U * S, "f32")
    out = B.mx_linear(x, w, bias, res)
    close(out, z + bias.double() + res.double(), (k + 4) * U * (S + bias.abs().double()) + 2 * U * res.abs().double(), "bf16")
    out = B.mx_linear(x.t().contiguous().t(), w, bias, activation="relu", dtype=torch.float32)
    close(out, (z + bias.double()).clamp(min=0), (k + 4) * U * (S + bias.abs().double()), "f32")


@gpu
@pytest.mark.parametrize("b,m,k,n", SEVERAL)
def test_several_tiles_a_workgroup(b, m, k, n):
    """More tiles than run at once: the lines' and blocks' scales differ widely, so that a tile with another's operands or scales is seen."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(m + k)

    def spread(*shape):
        return torch.randn(shape, generator=gen, device="cuda") * torch.exp2(torch.randint(-9, 10, (*shape[:-1], 1), generator=gen, device="cuda").float())

    x = (spread(b, m, k) * torch.exp2(torch.randint(-3, 4, (b, m, (k + 31) // 32), generator=gen, device="cuda").float()).repeat_interleave(32, -1)[..., :k]).bfloat16()
    q, w = B.mx_quantize(x), B.mx_quantize(spread(b, n, k).transpose(1, 2) * k ** -0.5, dim=-2)
    bias, res = torch.randn(n, generator=gen, device="cuda"), torch.randn((b, m, n), generator=gen, device="cuda")
    many = torch.full((b, m + 1, n), 7.0, device="cuda", dtype=torch.bfloat16)
    out, full = B.mx_linear(q, w, bias, res, out=many[:, :m]), B.mx_linear(x, w, dtype=torch.float32)
    assert (many[:, m] == 7.0).all()
    same = res.clone()
    assert B.mx_linear(q, w, bias, same, out=same) is same and torch.equal(same, B.mx_linear(q, w, bias, res, dtype=torch.float32))
    L, R = B.mx_dequantize(q, dtype=torch.float32).double(), B.mx_dequantize(w, dtype=torch.float32).double()
    for i in range(b):
        z, S = L[i] @ R[i].contiguous(), L[i].abs() @ R[i].abs().contiguous()
        close(full[i], z, (k + 2) * U * S, "f32")
        close(out[i], z + bias.double() + res[i].double(), (k + 4) * U * (S + bias.abs().double()) + 2 * U * res[i].abs().double(), "bf16")


@gpu
@pytest.mark.parametrize("m,k,n", [(8000, 640, 4090), (4000, 640, 4090), (2000, 900, 2040), (600, 128, 600), (300, 1000, 300), (9, 385, 70)])
def test_a_line_depends_on_no_other(m, k, n):
    """An odd number of half steps: what follows a line in memory is the next line, here with values that would be seen."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(k)
    x, w = torch.randn((m, k), generator=gen, device="cuda"), torch.randn((n, k), generator=gen, device="cuda")
    x[::7] *= 1e-22                                # (products down to the smallest that there are)
    w[::5] *= 1e-22
    want = B.mx_linear(B.mx_quantize(x), B.mx_quantize(w.t(), dim=-2), dtype=torch.float32)
    x2, w2 = x.clone(), w.clone()
    x2[1::2] = torch.randn((m // 2, k), generator=gen, device="cuda") * 1e30
    x2[3::4, 0] = float("nan")
    w2[1::2] = torch.randn((n // 2, k), generator=gen, device="cuda") * 1e30
    w2[3::4, 0] = float("inf")
    got = B.mx_linear(B.mx_quantize(x2), B.mx_quantize(w2.t(), dim=-2), dtype=torch.float32)
    assert torch.equal(got[::2, ::2], want[::2, ::2]) and torch.isnan(got[3::4]).all() and torch.isnan(got[:, 3::4]).all()


@gpu
@pytest.mark.parametrize("m,n,gap", [(4096, 4096, 0), (4096, 4096, 3), (8000, 2056, 5), (4000, 4099, 0), (130000, 120, 1), (2000, 8200, 0), (1000, 16001, 2)])
def test_results_past_the_caches(m, n, gap):
    """bf16 results of up to 32 MB, rows at any alignment: nothing beside them is written."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(n)

    def room(dtype):
        return torch.full((m, n + gap), 7.0, device="cuda", dtype=dtype)[:, :n]

    def beside(t):
        assert gap == 0 or (t.as_strided((m, gap), (n + gap, 1), n)[:-1] == 7.0).all()

    x = torch.randn((m, n), generator=gen, device="cuda").bfloat16()
    w, b = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda")
    out = room(torch.bfloat16)
    _, stats = B.layer_norm(x, w, b, out=out, stats=True)
    beside(out)
    X = x.double()
    mean, var = X.mean(-1, keepdim=True), X.var(-1, unbiased=False, keepdim=True)
    r = (var + 1e-5).rsqrt()
    h = (X - mean) * r
    c = n / 64 + 32                                # (tolerances of test_norm.py)
    off = ((c / 2 + 10) * h.abs() + (c + 4) * r * (X - mean).abs().mean(-1, keepdim=True)) * U
    want = h * w.double() + b.double()
    close(out, want, off * w.abs().double() + 3 * U * (want.abs() + h.abs() * w.abs().double()), "bf16")
    grad, res = torch.randn((m, n), generator=gen, device="cuda").bfloat16(), torch.randn((m, n), generator=gen, device="cuda").bfloat16()
    dx, dw, db = B.layer_norm_grad(grad, x, stats, w, b, res)
    h = (X - stats[:, :1].double()) * stats[:, 1:].double()
    g = grad.double() * w.double()
    r = stats[:, 1:].double()
    a, q = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    k = n / 64 + 38
    bound = r * (5 * U * (g.abs() + a.abs() + (h * q).abs()) + k * U * (g.abs().mean(-1, keepdim=True) + h.abs() * (g * h).abs().mean(-1, keepdim=True)))
    close(dx, r * (g - a - h * q) + res.double(), bound + 2 * U * res.abs().double() + U * bound, "bf16")
    close(dw, (grad.double() * h).sum(0), (m + 8) * U * (grad.double() * h).abs().sum(0), "f32")
    close(db, grad.double().sum(0), (m + 8) * U * grad.double().abs().sum(0), "f32")
    del X, h, g, want, off, bound
    # a product
    L = torch.randn((m, 100), generator=gen, device="cuda").bfloat16()
    v = B.mx_quantize(torch.randn((100, n), generator=gen, device="cuda"), dim=-2)
    out = room(torch.bfloat16)
    B.mx_linear(L, v, b, out=out, activation="relu")
    beside(out)
    l, R = B.mx_dequantize(B.mx_quantize(L)).double(), B.mx_dequantize(v, dtype=torch.float32).double().contiguous()
    close(out, (l @ R + b.double()).clamp(min=0), 104 * U * (l.abs() @ R.abs() + b.abs().double()), "bf16")


@gpu
def test_results_beyond_every_cache():
    """256 MB and more: values read back, lines at any alignment, a normalisation and a product; against the same of pieces."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    m, k = 4100, 32771
    x = torch.randn((m, k), generator=gen, device="cuda").bfloat16()
    pieces = [slice(at, at + 100) for at in range(0, m, 1000)] + [slice(m - 3, m)]
    back = B.mx_dequantize(B.mx_quantize(x))
    wide = B.mx_dequantize(B.mx_quantize(x[:2050]), dtype=torch.float32)
    for at in pieces:
        assert torch.equal(back[at], B.mx_dequantize(B.mx_quantize(x[at])))
    assert torch.equal(wide, back[:2050].float())
    y = x.as_strided((16400, 8190), (8191, 1))
    out, stats = B.layer_norm(y, stats=True)
    dx, _, _ = B.layer_norm_grad(y, y, stats)
    w = B.mx_quantize(torch.randn((200, 8190), generator=gen, device="cuda"), dim=-2)
    v = torch.randn((16400, 200), generator=gen, device="cuda").bfloat16()
    product = B.mx_linear(v, w)
    for at in [slice(at, at + 40) for at in range(0, 16400, 1500)] + [slice(16397, 16400)]:
        piece, s = B.layer_norm(y[at], stats=True)
        assert torch.equal(out[at], piece) and torch.equal(stats[at], s) and torch.equal(dx[at], B.layer_norm_grad(y[at], y[at], s)[0])
        # (sums of 200 products, whole within a step: the same bits by every kernel)
        assert torch.equal(product[at], B.mx_linear(v[at], w))
