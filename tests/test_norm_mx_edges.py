"""Layer normalisation and 4-bit operands at the ends of what the calls take: the widest results, the most rows, the largest values, sizes of zero;
and sums whose order is the same however lhs is given."""
import numpy as np
import pytest

from paper_2505_01637_amd import binding as B
from test_host_part import run_on_fake_hip
from test_norm import norm_of
from test_operators import U, _torch, check, f64

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("n", [(1 << 30) + 5])
def test_rows_of_four_gigabytes(n):
    """f32 results, a row of more than 2^32 bytes (77 GB with its weights): every element is stored, those too behind which 2^30 and a few are left."""
    import torch
    k = 40
    gen = torch.Generator(device="cuda").manual_seed(2)
    # columns 0 to 4095 again and again: whole groups of 64, so that scales repeat with the codes
    w = B.mx_quantize(torch.randn((k, 4096), generator=gen, device="cuda"), dim=-2)
    times = -(-n // 4096)
    codes = w.codes.repeat(times, 1)[:n]
    scales = w.scales.repeat(times, 1, 1, 1, 1)[:-(-n // 64)]
    x = torch.randn((1, k), generator=gen, device="cuda")
    out = torch.full((1, n), float("nan"), device="cuda")
    print("a product of 1 x %d x %d" % (k, n), flush=True)
    B.mx_linear(x, B.MX(codes, scales, k, dim=-2, dtype=torch.float32), out=out)
    want = B.mx_linear(x, w)
    bound = (k + 2) * U * (B.mx_dequantize(B.mx_quantize(x)).abs() @ B.mx_dequantize(w, dtype=torch.float32).abs())
    near = (out[0, :n // 4096 * 4096].view(-1, 4096) - want).abs_() <= 2 * bound          # (either product is within one of them of the exact one)
    assert near.all(), (~near).nonzero()[:8].tolist()
    tail = out[:, n // 4096 * 4096:]
    assert ((tail - want[:, :tail.shape[1]]).abs() <= 2 * bound[:, :tail.shape[1]]).all()
    del out, codes, scales, near, tail
    torch.cuda.empty_cache()


# (m, k, n) at which a lhs in blocks and one that the call puts into them would be split differently if what the latter costs counted
APART = [(2, 6152, 1876), (8, 4709, 395), (7, 5403, 192), (5, 14490, 2167), (3, 5690, 3186), (2, 5078, 39), (6, 4800, 669), (6, 10624, 1081), (2, 16129, 4087), (17, 5413, 16)]

HEAD = r"""
import ctypes as C, math, random, sys
sys.path.insert(0, sys.argv[2])
sys.modules["torch"] = None                       # (its own runtime would be loaded first)
hip = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
hip.fake_blocks_of.restype = C.c_uint64
from paper_2505_01637_amd import binding as B
lib = B.lib()
NONE, P = (0, 0, 0, 0, 0), 1 << 20                # (addresses that nothing reads)
"""

ORDER = HEAD + r"""
def plan(how, b, m, k, n, shared):
    # the products' kernel, its workgroups, and the bytes of partial sums
    lhs = {"blocks": NONE, "columns": (P, 1, 1, m, m * k), "bf16": (P, 1, 0, k, m * k), "f32 and a gap": (P, 0, 0, k + 1, m * (k + 1))}[how]
    d = B._MX_LINEAR.pack(b, m, k, n, *lhs, *((P, P) if how == "blocks" else (0, 0)), 0, 0, P, P, shared, 0, *NONE, *NONE, P, 1, 0, n, m * n, 0, 0)
    size = C.c_size_t()
    assert lib.mrl_mx_linear_bytes(d, C.addressof(size)) == 0, lib.mrl_last_error()
    hip.fake_blocks_of(b"mx_")
    hip.fake_launches_of(b"mx_quantize")
    assert lib.mrl_mx_linear(d, P, size.value, None) == 0, lib.mrl_last_error()
    up = lambda x: (x + 255) // 256 * 256
    steps = -(-k // 128)
    mine = (up(b * m * steps * 64) + up((-(-b * m // 64) if shared else b * -(-m // 64)) * steps * 256)) if hip.fake_launches_of(b"mx_quantize") else 0
    names = [t for t in ("mx_tile_kernelILi256ELi256E", "mx_tile_kernelILi256ELi128E", "mx_tile_kernelILi128ELi128ELi2ELi2E", "mx_tile_kernelILi128ELi128ELi2ELi4E", "mx_tile_kernelILi64E", "mx_rows_kernel")
             if hip.fake_launches_of(t.encode())]
    return names, hip.fake_blocks_of(b"mx_tile") + hip.fake_blocks_of(b"mx_rows"), size.value - mine

r = random.Random(5)
size = lambda lo, hi: int(math.exp(r.uniform(math.log(lo), math.log(hi))))
cases = [(1, *c, 0) for c in APART] + [(2, *c, 0) for c in APART]
for i in range(3000):
    cases.append((1, size(1, 64 if i % 2 else 8192), size(1, 20000), size(1, 20000), 0))
for i in range(300):                              # batches with a rhs each, and rows of whole groups of 64 that share one
    cases.append((r.randint(2, 9), size(1, 300), size(1, 20000), size(1, 5000), 0))
    cases.append((r.randint(2, 9), 64 * r.randint(1, 5), size(1, 20000), size(1, 5000), 1))
for case in cases:
    plans = [plan(how, *case) for how in (("blocks", "bf16", "f32 and a gap") if case[0] > 1 and case[4] else ("blocks", "bf16", "f32 and a gap", "columns"))]
    assert len(plans[0][0]) == 1 and all(p == plans[0] for p in plans), (case, plans)
print("done")
"""


def test_sums_have_one_order_however_lhs_is_given(tmp_path):
    """A lhs in blocks, of either type with its rows' elements adjacent, and with its columns': the same kernel, workgroups and splits."""
    run_on_fake_hip(tmp_path, ORDER.replace("APART", repr(APART)))


@gpu
@pytest.mark.parametrize("m,k,n", APART)
def test_the_same_bits_however_lhs_is_given(m, k, n):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    x = torch.randn((m, k), generator=gen, device="cuda").bfloat16()
    w = B.mx_quantize(torch.randn((k, n), generator=gen, device="cuda"), dim=-2)
    want = B.mx_linear(x, w, dtype=torch.float32)
    for lhs in (x.float(), x.t().contiguous().t(), B.mx_quantize(x)):
        assert torch.equal(B.mx_linear(lhs, w, dtype=torch.float32), want)


MANY = HEAD + r"""
x = lambda m, n: (P, 1, 0, n, m * n)
same = lambda n: (P, 1, 0, 0, 0)                  # every row the same memory
for m, n in (((1 << 22) - 1, 16385), (1 << 22, 16385), (5000000, 16385), ((1 << 23) + 3, 20000), (5000000, 64), (1 << 30, 3)):
    for t in (x(m, n), same(n)):
        hip.fake_blocks_of(b"norm_")
        assert lib.mrl_layer_norm(B._NORM.pack(1, m, n, 1e-5, *t, *x(m, n), *NONE, *NONE, P), None) == 0, (m, n, lib.mrl_last_error())
        assert n < 8192 or hip.fake_blocks_of(b"norm_") == m, "a workgroup for each long row"
        for sums in (0, 1):
            v = (P, 0, 0, 1, 0) if sums else NONE
            d = B._NORM_GRAD.pack(1, m, n, 0, *t, *t, *NONE, *NONE, *x(m, n), *v, *v, P)
            size = C.c_size_t()
            assert lib.mrl_layer_norm_grad_bytes(d, C.addressof(size)) == 0, lib.mrl_last_error()
            assert lib.mrl_layer_norm_grad(d, P, size.value, None) == 0, (m, n, sums, lib.mrl_last_error())
print("done")
"""


def test_more_rows_than_a_launch_takes(tmp_path):
    """A launch has fewer than 2^32 threads (the runtime here holds callers to that): millions of long rows, a workgroup of 1024 each, go in several."""
    run_on_fake_hip(tmp_path, MANY)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 5, 7, 40, 130, 2048, 3000, 16001, 40000])
def test_rows_of_large_magnitude(n, dtype):
    """Rows whose squares' sum leaves f32's range: the mean is right (test_norm.py's tolerance), r is 0 and the row its bias; d_x is then the residual.  Magnitudes of
    both signs and of one, up to 1e38 / n: sums of n of them, and of n differences of two, are below 2^128.  Rows whose own sum leaves it are NaN."""
    torch, types = _torch()
    rng = np.random.default_rng(n)
    magnitude = np.array([1e15, 1e22, 1e27, 1e33, 0.5e38 / n] * 2).clip(max=0.5e38 / n)
    x = (1 + rng.random((10, n))) * magnitude[:, None]
    x[5:] *= np.where(rng.random((5, n)) < 0.5, -1, 1)
    x[:, 0] *= np.where(x[:, 0] < 0, 1, -1)               # (no row of equal elements)
    x = torch.from_numpy(x).to(types[dtype]).cuda()
    w, b = (torch.from_numpy(rng.standard_normal(n)).float().cuda() for _ in range(2))
    out, stats = B.layer_norm(x, w, b, stats=True, dtype=torch.float32)
    want, mean, r, bound = norm_of(f64(x), f64(w), f64(b))
    X, c = f64(x), n / 64 + 32
    check(stats[:, 0], mean, c * U * np.abs(X - mean[:, None]).mean(-1) + (c * U) ** 2 * np.abs(X).mean(-1), "f32", "mean")
    for i in (0, 5):
        check(out[i], want[i], bound[i], "f32", i)
    large = [1, 2, 3, 4, 6, 7, 8, 9]
    assert (stats[large, 1] == 0).all() and torch.equal(out[large], b.expand(8, n))
    grad, res = (torch.from_numpy(rng.standard_normal((10, n))).float().cuda() for _ in range(2))
    dx, dw, _ = B.layer_norm_grad(grad[large], x[large], stats[large], w, b, res[large])
    assert torch.equal(dx, res[large].to(types[dtype])) and (dw == 0).all()
    assert torch.equal(B.layer_norm(x, stats=True)[1], stats)
    if n >= 40:
        out, stats = B.layer_norm(torch.full((2, n), 1.5e38, device="cuda").to(types[dtype]), w, b, stats=True)
        assert out.isnan().all() and stats[:, 1].isnan().all()


@gpu
@pytest.mark.parametrize("shape", [(4, 0), (2, 3, 0), (0, 0)], ids=str)
def test_statistics_of_rows_without_elements(shape):
    """There is no mean of nothing: NaN, as 0 / 0 is, and not what the memory held."""
    torch, _ = _torch()
    filled = torch.full((8, 2), 7.0, device="cuda")
    del filled                                    # (what torch gives out next)
    out, stats = B.layer_norm(torch.empty(shape, device="cuda"), stats=True)
    assert out.shape == shape and stats.shape == shape[:-1] + (2,) and stats.isnan().all()


def test_workspace_of_a_gradient_without_a_gpu():
    """Gradients of many rows ask for their blocks' sums (f32, two for each column) and refuse less, none and what is not aligned; of few rows they ask for nothing.
    Host code: nothing is launched (the addresses are of nothing)."""
    import ctypes as C
    P, lib = 1 << 20, B.lib()
    vector = (P, 0, 0, 1, 0)

    def grad(m, n, dw=vector, db=vector):
        x, size = (P, 0, 0, n, m * n), C.c_size_t()
        d = B._NORM_GRAD.pack(1, m, n, 0, *x, *x, *B._ABSENT, *B._ABSENT, *x, *dw, *db, P)
        assert lib.mrl_layer_norm_grad_bytes(d, C.addressof(size)) == 0
        return size.value, lambda work, have: lib.mrl_layer_norm_grad(d, work, have, None)

    for m, n, blocks in ((1 << 16, 16, 256), (8192, 2048, 256), (100, 20000, 2), (1 << 16, 5, 1024)):
        for dw, db in ((vector, vector), (vector, B._ABSENT), (B._ABSENT, vector)):
            need, run = grad(m, n, dw, db)
            assert need == blocks * 2 * n * 4
            assert run(None, 0) == B.E_NOMEM and run(P, need - 1) == B.E_NOMEM and run(P + 2, need) == B.E_INVAL and run(None, need) == B.E_INVAL
        assert grad(m, n, B._ABSENT, B._ABSENT)[0] == 0
    for m, n in ((1, 16), (256, 16), (8, 2048), (0, 16), (64, 20000)):
        assert grad(m, n)[0] == 0
