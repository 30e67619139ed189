"""Edges of the operators on data: what the library's host part launches there (on the CPU, on a runtime
that launches nothing but counts: fake_hip.c), and values against 64 bits on a GPU."""
import numpy as np
import pytest

from test_host_part import run_on_fake_hip
from test_operators import U, UNIT, check, f64, plain_grad, scale_of, strided

gpu = pytest.mark.gpu

# what the programs below begin with: descriptors by what a matrix is, and the (mangled) names of what they launched
HOST = r"""
import ctypes as C, sys
sys.path.insert(0, sys.argv[2])
sys.modules["torch"] = None                       # (its own runtime would be loaded first)
hip = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
from paper_2505_01637_amd import binding as B
lib = B.lib()
NONE, P = (0, 0, 0, 0, 0), 1 << 20                # (addresses that nothing reads)

def mat(rows, columns, dtype, layout=0, at=0, ld=0, shared=False):
    ld = ld or (rows if layout else columns)
    return P + at, dtype, layout, ld, 0 if shared else ld * (columns if layout else rows)

def grad(m, k, n, dtype=1, b=1, act=0, drop=0, lhs=0, rhs=0, d_rhs=None, shared=True, at=0, need_lhs=True, need_rhs=True, d_bias=False):
    mats = (mat(m, n, dtype, at=at), mat(m, k, dtype, lhs), mat(k, n, dtype, rhs, shared=shared), mat(m, n, dtype) if act else NONE,
            mat(m, k, dtype) if need_lhs else NONE, mat(k, n, dtype, rhs if d_rhs is None else d_rhs, shared=shared) if need_rhs else NONE,
            mat(1, n, 0) if d_bias else NONE)
    return B._LINEAR_GRAD.pack(b, m, k, n, *(v for x in mats for v in x), act, drop, 0, 0)

def linear(m, k, n, dtype=1, b=1, lhs=0, rhs=0, shared=True, at_lhs=0, at_rhs=0, out=None):
    mats = (mat(m, k, dtype, lhs, at_lhs), mat(k, n, dtype, rhs, at_rhs, shared=shared), NONE, NONE, mat(m, n, dtype if out is None else out), NONE)
    return B._LINEAR.pack(b, m, k, n, *(v for x in mats for v in x), 0, 0, 0, 0)

def took(*names):
    # how often each was launched (counting takes what it counts: a part of a longer name comes after it)
    n = {k: hip.fake_launches_of(k.encode()) for k in names}
    return {k: v for k, v in n.items() if v}

def run(name, desc):
    size = C.c_size_t()
    assert getattr(lib, name + "_bytes")(desc, C.addressof(size)) == 0, lib.mrl_last_error()
    assert getattr(lib, name)(desc, P, size.value, None) == 0, lib.mrl_last_error()
    return size.value
"""

NARROW = HOST + r"""
# lines of dz are padded, but a line that holds less than 16 bytes of elements must not be read as 16 bytes of them
def wide():
    n = took("rows_wide_kernel")
    # (the last template argument of product_kernel: loads of 16 bytes)
    for t in ("DF16b", "f"):
        for a in "01":
            for b in "01":
                for tile in ("Li128ELi128ELi2ELi2E", "Li64ELi64ELi2ELi2E"):
                    n.update(took("product_kernelI%sLb%sELb%sE%sLb1E" % (t, a, b, tile)))
    return n
seen = 0
for dtype, narrow in ((1, range(1, 8)), (0, range(1, 4))):
    for n in narrow:
        for m, k in ((100, 33), (3, 7), (1, 1001), (2000, 511), (9, 40)):
            for act, drop in ((1, 0), (0, 6554), (2, 100)):
                for lhs in (0, 1):
                    for rhs in (0, 1):
                        for d_rhs in (0, 1):
                            for need_lhs, need_rhs in ((True, False), (False, True), (True, True)):
                                wide()
                                run("mrl_linear_grad", grad(m, k, n, dtype, 1, act, drop, lhs, rhs, d_rhs, need_lhs=need_lhs, need_rhs=need_rhs))
                                assert not wide(), (dtype, m, k, n, act, lhs, rhs, d_rhs, need_lhs, need_rhs)
                                seen += bool(took("product_kernel"))
assert seen
# of eight (four) and more they are
run("mrl_linear_grad", grad(100, 33, 9, 1, act=1, need_lhs=False))
assert wide()
print("done")
"""


def test_narrow_gradients_take_no_loads_of_16_bytes(tmp_path):
    run_on_fake_hip(tmp_path, NARROW)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6, 7])
@pytest.mark.parametrize("lhs_columns,rhs_columns", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("m,k", [(100, 33), (65, 72), (1, 129)])
def test_gradients_of_narrow_outputs(dtype, n, lhs_columns, rhs_columns, m, k):
    """Few columns of out, dz made by a pass.  The bounds are those of the formula's other shapes: dz before it is rounded within two products
    of f32 (ReLU, D), rounded to the operands' type, then a sum over n or m."""
    from paper_2505_01637_amd import binding as B
    rng = np.random.default_rng(n)
    lhs, rhs = strided(rng.standard_normal((m, k)), dtype, lhs_columns), strided(rng.standard_normal((k, n)), dtype, rhs_columns)
    bias = strided(rng.standard_normal((1, n)), "f32")[0]
    grad, z = strided(rng.standard_normal((m, n)), dtype), strided(rng.standard_normal((m, n)), dtype)
    print("linear_grad", m, k, n, dtype, lhs_columns, rhs_columns, flush=True)
    d_lhs, d_rhs, d_bias = B.linear_grad(grad, lhs, rhs, bias, z, activation="relu", dropout=0.25, seed=9, offset=2)
    G, L, R, Z = f64(grad), f64(lhs), f64(rhs), f64(z)
    dz, want_l, want_r = plain_grad(G, L, R, Z, "relu", scale_of(G.shape, 0.25, 9, 2))
    db = 2 * U * np.abs(dz)
    rounded = db + UNIT[dtype] * (np.abs(dz) + db)
    check(d_lhs, want_l, rounded @ np.abs(R).T + (n + 2) * U * (np.abs(dz) @ np.abs(R).T), dtype, "d_lhs")
    check(d_rhs, want_r, np.abs(L).T @ rounded + (m + 2) * U * (np.abs(L).T @ np.abs(dz)), dtype, "d_rhs")
    check(d_bias, dz.sum(0), db.sum(0) + (m + 2) * U * np.abs(dz).sum(0), "f32", "d_bias")


NO_BATCHES = HOST + r"""
# d_rhs of batches that share rhs, of which there are none: zeros, and lhs, of which there is nothing, is not copied
took("copy_kernel")
seen = []
for dtype in (0, 1):
    for m, k, n in ((3, 8192, 8192), (5, 4000, 9000), (100, 33, 70), (1001, 511, 777), (8, 64, 64), (1, 1, 1)):
        for lhs in (0, 1):
            for d_rhs in (0, 1):
                for act in (0, 1):
                    took("_kernel")
                    run("mrl_linear_grad", grad(m, k, n, dtype, 0, act, 0, lhs, 0, d_rhs, need_lhs=False))
                    n_copies = took("copy_kernel")
                    if n_copies: seen.append((dtype, m, k, n, lhs, d_rhs, act))
                    assert took("_kernel"), "zeros are stored"
assert not seen, seen
print("done")
"""


def test_no_copies_of_batches_that_are_not_there(tmp_path):
    run_on_fake_hip(tmp_path, NO_BATCHES)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(3, 8192, 8192), (100, 33, 70), (8, 64, 64)])
@pytest.mark.parametrize("activation", ["none", "silu"])
def test_gradient_of_no_batches_is_zero(dtype, m, k, n, activation):
    """rhs shared by the batches, of which there are none; lhs column-major."""
    import torch
    from paper_2505_01637_amd import binding as B
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    lhs = torch.empty((0, k, m), device="cuda", dtype=t).transpose(-1, -2)
    rhs = torch.ones((k, n), device="cuda", dtype=t)
    grad = torch.empty((0, m, n), device="cuda", dtype=t)
    print("linear_grad of no batches", m, k, n, dtype, activation, flush=True)
    for _ in range(2):
        torch.full((k, n), float("nan"), device="cuda", dtype=t)        # (what the result's memory held)
        d_lhs, d_rhs, d_bias = B.linear_grad(grad, lhs, rhs, torch.ones(n, device="cuda"), grad, activation=activation)
        assert d_lhs.shape == lhs.shape and d_rhs.shape == rhs.shape and not d_rhs.any() and not d_bias.any()


TENSORS = HOST + r"""
class Device:
    index = 0

class Tensor:
    # what the binding asks of a tensor
    def __init__(self, shape, strides, dtype, at):
        self.shape, self.strides, self.dtype, self.at, self.device = tuple(shape), tuple(strides), dtype, at, Device
    def data_ptr(self): return self.at
    def stride(self, i=None): return self.strides if i is None else self.strides[i]
    def get_device(self): return 0
    def is_contiguous(self): return True
    def dim(self): return len(self.shape)
    def numel(self):
        n = 1
        for s in self.shape: n *= s
        return n
    def element_size(self): return {"f32": 4, "bf16": 2, "u8": 1}[self.dtype]
    def new_empty(self, shape, dtype=None):
        return row_major(shape if isinstance(shape, tuple) else (shape,), dtype or self.dtype)
    def transpose(self, a, b):
        return Tensor(self.shape[:-2] + self.shape[:-3:-1], self.strides[:-2] + self.strides[:-3:-1], self.dtype, self.at)

def row_major(shape, dtype, at=P):
    strides = [1]
    for s in shape[:0:-1]: strides.insert(0, strides[0] * s)
    return Tensor(shape, strides, dtype, at)

B._codes, B._uint8, B._raw_stream, B._current_device = {"f32": 0, "bf16": 1}, "u8", lambda i: None, lambda: 0
"""

FORMS = TENSORS + r"""
off = {"f32": (0, 4, 8), "bf16": (0, 2, 8)}
for dtype in ("bf16", "f32"):
    for m, k, n in ((4096, 4096, 1024), (8192, 1024, 1024), (4096, 2048, 8192), (1, 16384, 256), (300, 301, 302)):
        shifts = [(a, b, c) for a in off[dtype] for b in off[dtype] for c in off[dtype]]
        for order in (shifts, shifts[::-1]):
            B._forms.clear()
            for a, b, c in order:
                lhs, rhs, g = row_major((m, k), dtype, P + a), row_major((k, n), dtype, P + b), row_major((m, n), dtype, P + c)
                B.linear(lhs, rhs)                     # (a workspace that is too small is refused)
                B.linear_grad(g, lhs, rhs)
            assert len(B._forms) <= 4 + 8, "as many forms as there are plans, not one an address"
print("done")
"""


def test_operands_at_different_alignments_in_turn(tmp_path):
    """The same sizes and strides with now one operand and now another off a multiple of 16 bytes: each call has the workspace
    that it needs, whatever was called before."""
    run_on_fake_hip(tmp_path, FORMS)


@gpu
@pytest.mark.parametrize("shifts", [((0, 0), (0, 4), (4, 0), (4, 4)), ((4, 0), (0, 4), (0, 0), (4, 4))])
def test_values_at_different_alignments_in_turn(shifts):
    """And the results are the same: 8192 x 1024 x 1024 in bf16, where only an operand that is off is copied."""
    import torch
    from paper_2505_01637_amd import binding as B
    B._forms.clear()
    m, k, n = 8192, 1024, 1024
    gen = torch.Generator(device="cuda").manual_seed(3)
    flat = [torch.randn(r * c + 8, generator=gen, device="cuda").bfloat16() for r, c in ((m, k), (k, n), (m, n))]
    values = [f[:r * c].clone().view(r, c) for f, (r, c) in zip(flat, ((m, k), (k, n), (m, n)))]
    want = values[0].double() @ values[1].double()
    bound = (k + 2) * U * (values[0].double().abs() @ values[1].double().abs())
    grads = values[2].double() @ values[1].double().t(), values[0].double().t() @ values[2].double()
    bounds = (n + 2) * U * (values[2].double().abs() @ values[1].double().abs().t()), (m + 2) * U * (values[0].double().abs().t() @ values[2].double().abs())
    for a, b in shifts:
        lhs, rhs = (f[s:s + v.numel()].view(v.shape) for f, v, s in zip(flat, values, (a, b)))
        lhs.copy_(values[0])
        rhs.copy_(values[1])
        print("linear", m, k, n, a, b, flush=True)
        out = B.linear(lhs, rhs, dtype=torch.float32)
        assert ((out.double() - want).abs() <= bound + U * want.abs()).all()
        for got, w, e in zip(B.linear_grad(values[2], lhs, rhs), grads, bounds):
            assert ((got.double() - w).abs() <= e + UNIT["bf16"] * (w.abs() + e)).all()


PROBABILITY = TENSORS + r"""
import struct
class Scalar:
    # a number that a program changes in place, as a tensor of one element is
    def __init__(self, v): self.v = v
    def __mul__(self, x): return self.v * x
    def __float__(self): return float(self.v)
    def __ge__(self, x): return self.v >= x
    def __le__(self, x): return self.v <= x

drops = []
real = B._run
def keep(desc, run, need, given, like):
    drops.append((B._LINEAR if run is B._lib.mrl_linear else B._LINEAR_GRAD).unpack(desc)[-3])
    real(desc, run, need, given, like)
B._run = keep
lhs, rhs, g = row_major((8, 16), "f32"), row_major((16, 4), "f32"), row_major((8, 4), "f32")
p = Scalar(0.25)
for v in (0.25, 0.5, 0.0, 0.25):
    p.v = v
    B.linear(lhs, rhs, dropout=p)
    B.linear_grad(g, lhs, rhs, dropout=p)
assert drops == [16384, 16384, 32768, 32768, 0, 0, 16384, 16384], drops
for v in (1.5, float("nan")):
    for call in (lambda p: B.linear(lhs, rhs, dropout=p), lambda p: B.linear_grad(g, lhs, rhs, dropout=p)):
        p.v = v
        try:
            call(p)
        except B.MorelloError as e:
            assert e.code == B.E_INVAL
        else:
            assert 0, v
print("done")
"""


def test_a_probability_that_changes_in_place(tmp_path):
    """A call takes the value that the probability has then, also where it is an object that had another one before."""
    run_on_fake_hip(tmp_path, PROBABILITY)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("activation", ["relu", "gelu", "silu"])
def test_dropped_elements_of_a_gradient_are_zero_whatever_z_is(dtype, activation):
    """One row of m x n, so that d_bias is dz itself: where an element is dropped dz is 0, where it is not NaN, infinite and
    finite z count.  Two rows: a column's sum is that of the element that is kept."""
    import torch
    from paper_2505_01637_amd import binding as B
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    n = 256
    kw = {"activation": activation, "dropout": 0.5, "seed": 6, "offset": 3}
    bias, rhs = torch.zeros(n, device="cuda"), torch.zeros((8, n), device="cuda", dtype=t)
    for m in (1, 2):
        dropped = torch.from_numpy(scale_of((m, n), 0.5, 6, 3) == 0).cuda()
        lhs, grad = torch.zeros((m, 8), device="cuda", dtype=t), torch.ones((m, n), device="cuda", dtype=t)
        z = torch.full((m, n), float("nan"), device="cuda", dtype=t)
        _, _, dz = B.linear_grad(grad, lhs, rhs, bias, z, **kw)
        assert (dz[dropped.all(0)] == 0).all() and dz[~dropped.all(0)].isnan().all()
        # NaN only where it is dropped: as if it were not there
        clean = torch.full((m, n), 0.75, device="cuda", dtype=t)
        _, _, want = B.linear_grad(grad, lhs, rhs, bias, clean, **kw)
        d_lhs, d_rhs, dz = B.linear_grad(torch.where(dropped, float("inf"), grad), lhs + 1, rhs + 1, bias, torch.where(dropped, z, clean), **kw)
        assert torch.equal(dz, want) and d_lhs.isfinite().all() and d_rhs.isfinite().all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_relu_passes_nothing_on_where_z_is_not_positive(dtype, p):
    """One row, so that d_bias is dz: 0 where z <= 0 whatever the gradient is, the gradient times D where z > 0, NaN where z is NaN (as
    relu(z) is), 0 where it is dropped."""
    import torch
    from paper_2505_01637_amd import binding as B
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    inf, nan = float("inf"), float("nan")
    grads, zs = (1.5, -2.0, inf, -inf, nan), (1.0, inf, 2.0 ** -100, 0.0, -0.0, -3.0, -inf, -2.0 ** -100, nan)
    pairs = [(g, z) for g in grads for z in zs] * 3
    n = len(pairs)
    grad, z = (torch.tensor([[x[i] for x in pairs]], device="cuda", dtype=t) for i in (0, 1))
    lhs, rhs = torch.zeros((1, 8), device="cuda", dtype=t), torch.zeros((8, n), device="cuda", dtype=t)
    d = scale_of((1, n), p, 11, 1)[0]
    _, _, dz = B.linear_grad(grad, lhs, rhs, torch.zeros(n, device="cuda"), z, activation="relu", dropout=p, seed=11, offset=1)
    want = [0.0 if k == 0 else nan if z != z else g * k if z > 0 else 0.0 for (g, z), k in zip(pairs, d)]
    assert np.array_equal(f64(dz), np.array(want), equal_nan=True)
    # and what the products make of it: an infinite gradient at z <= 0 reaches neither
    grad, z = torch.ones((8, 16), device="cuda", dtype=t), torch.ones((8, 16), device="cuda", dtype=t)
    grad[2, 3], z[2, 3] = inf, -1.0
    d_lhs, d_rhs, d_bias = B.linear_grad(grad, torch.ones((8, 5), device="cuda", dtype=t), torch.ones((5, 16), device="cuda", dtype=t), torch.zeros(16, device="cuda"), z,
                                         activation="relu")
    rows, columns = torch.full((8,), 16.0, device="cuda"), torch.full((16,), 8.0, device="cuda")
    rows[2], columns[3] = 15.0, 7.0
    assert (d_lhs.float() == rows[:, None]).all() and (d_rhs.float() == columns).all() and torch.equal(d_bias, columns)


ONE_ROW = TENSORS + r"""
calls = []
class Library:                                     # what was asked of it, and the library's own answer
    def __getattr__(self, name): return getattr(lib, name)
    def mrl_dropout(self, desc, stream):
        calls.append(B._DROPOUT.unpack(desc))
        return lib.mrl_dropout(desc, stream)
B._lib = Library()

def swapped(a, b, c, ld=None):
    # a x 1 x c as a transposed 1 x a x c shows it: the only row of a batch has a stride that nothing uses
    return Tensor((a, 1, c), (ld or c, b, 1), "f32", P)

for x, ld in ((swapped(3, 24, 8), 8), (swapped(3, 1, 8), 8), (swapped(3, 99, 8, 16), 16), (Tensor((1, 3, 8), (5, 8, 1), "f32", P), 8), (row_major((3, 4, 8), "f32"), 8)):
    B.dropout(x, dropout=0.5, out=x)
    rows = x.shape[0] * x.shape[1]
    assert calls[-1][:2] == (rows, 8) and calls[-1][5] == calls[-1][15] == ld, calls[-1]
    B.dropout(x, x, dropout=0.5)
    B.dropout_grad(x, dropout=0.5)
# and of batches without rows there is nothing to do
for a, b in ((3, 0), (0, 3), (0, 0), (0, 1)):
    B.dropout(row_major((a, b, 8), "f32"), dropout=0.5)
    B.dropout(Tensor((a, b, 8), (8, 8, 1), "f32", P), dropout=0.5)
# batches that do not follow each other are still refused
for x in (Tensor((2, 3, 8), (32, 8, 1), "f32", P), Tensor((2, 2, 8), (8, 16, 1), "f32", P)):
    try:
        B.dropout(x, dropout=0.5)
    except B.MorelloError as e:
        assert e.code == B.E_INVAL
    else:
        assert 0
print("done")
"""


def test_dropout_of_batches_of_one_row(tmp_path):
    """The stride of a batch's only row says nothing: batches follow each other at their own stride."""
    run_on_fake_hip(tmp_path, ONE_ROW)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout_of_batches_of_one_row_on_data(dtype):
    import torch
    from paper_2505_01637_amd import binding as B
    x = strided(np.random.default_rng(1).standard_normal((1, 5, 33)), dtype).transpose(0, 1)
    assert x.is_contiguous() and x.shape == (5, 1, 33)
    got = B.dropout(x, x, dropout=0.4, seed=3, offset=1)
    assert torch.equal(got, B.dropout(x[:, 0], x[:, 0], dropout=0.4, seed=3, offset=1)[:, None])


FAR = HOST + r"""
# places beyond any address: two rows or batches that share one only when offsets are taken mod 2^64, and those that do not
def out(b, m, ld, batch, n=6):
    return B._LINEAR.pack(b, m, 8, n, P, 0, 0, 8, 0, P, 0, 0, n, 0, *NONE, *NONE, P, 0, 0, ld, batch, *NONE, 0, 0, 0, 0)
for desc in (out(2, (1 << 25) + 1, 1 << 39, 1 << 39), out(2, (1 << 25) + 1, 1 << 39, 6), out(2, (1 << 26) + 1, 1 << 38, 1 << 38), out(1, 1 << 30, (1 << 40) - 1, 0),
             out(1 << 30, 1, 6, (1 << 40) - 1)):
    assert lib.mrl_linear(desc, None, 0, None) == B.E_INVAL, lib.mrl_last_error()
    assert b"out" in lib.mrl_last_error(), lib.mrl_last_error()
lhs = B._LINEAR.pack(1, 1 << 30, 8, 6, P, 0, 0, (1 << 40) - 1, 0, P, 0, 0, 6, 0, *NONE, *NONE, P, 0, 0, 6, 0, *NONE, 0, 0, 0, 0)
assert lib.mrl_linear(lhs, None, 0, None) == B.E_INVAL and b"lhs" in lib.mrl_last_error(), lib.mrl_last_error()
# large, but possible
assert lib.mrl_linear(out(2, 1 << 12, 1 << 22, 1 << 35), None, 0, None) == 0, lib.mrl_last_error()
print("done")
"""


def test_offsets_that_no_address_has(tmp_path):
    run_on_fake_hip(tmp_path, FAR)


WORKSPACE = HOST + r"""
import itertools
size = C.c_size_t()
for name, desc in (("mrl_linear", linear(1, 1 << 16, 64)), ("mrl_linear", linear(4096, 4096, 1024, at_rhs=8)), ("mrl_linear_grad", grad(100, 64, 64, act=1)),
                   ("mrl_linear_grad", grad(4096, 1024, 1024, at=8)), ("mrl_linear_grad", grad(300, 64, 64, need_lhs=False, need_rhs=False, d_bias=True))):
    assert getattr(lib, name + "_bytes")(desc, C.addressof(size)) == 0
    assert size.value > 0, "a shape that needs a workspace"
    call = getattr(lib, name)
    took("_kernel")
    for at, have, code in ((P, size.value - 1, B.E_NOMEM), (P, 0, B.E_NOMEM), (None, size.value, B.E_INVAL), (P + 8, size.value, B.E_INVAL)):
        assert call(desc, at, have, None) == code, (name, at, have, lib.mrl_last_error())
    assert took("_kernel") == {}, "a refused call launches nothing"
    assert call(desc, P, size.value, None) == 0 and took("_kernel")
print("done")
"""


def test_workspaces_that_are_too_small_or_not_there(tmp_path):
    run_on_fake_hip(tmp_path, WORKSPACE)


@gpu
def test_operator_of_a_spec_takes_the_types_of_the_spec():
    """Table.apply refuses a bias of another type than the Spec's, as it does lhs and rhs, and an out of another type."""
    import torch
    from paper_2505_01637_amd import binding as B
    from paper_2505_01637_amd import workloads as W
    target, tabs = B.solve_config(W.config(5, max_size=16))
    gen = torch.Generator(device="cuda").manual_seed(1)
    lhs, rhs, bias = (torch.randn(s, generator=gen, device="cuda") for s in ((8, 16), (16, 4), (4,)))
    x = tabs["F"].coord_of_spec((1, 8, 16, 4), (3, 3, 3, 3, 3), layouts=(0, 0, 0, 0))
    out = tabs["F"].apply(x, lhs, rhs, bias)
    assert torch.equal(out, tabs["F"].apply(x, lhs[None], rhs, bias)[0])
    for bad in (lambda: tabs["F"].apply(x, lhs, rhs, bias.bfloat16()), lambda: tabs["F"].apply(x, lhs, rhs, bias, out=out.bfloat16()),
                lambda: tabs["F"].apply(x, lhs, rhs, bias.double()), lambda: tabs["F"].apply(x, lhs, rhs, bias[:3])):
        with pytest.raises(B.MorelloError) as e:
            bad()
        assert e.value.code == B.E_INVAL
