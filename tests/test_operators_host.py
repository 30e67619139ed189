"""What the library's host part launches for the operators, on the CPU (no GPU needed): it runs on a runtime that
launches nothing but counts (fake_hip.c)."""
from test_host_part import run_on_fake_hip

BODY = r"""
import ctypes as C, sys
sys.path.insert(0, sys.argv[2])
sys.modules["torch"] = None                       # (its own runtime would be loaded first)
hip = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
from paper_2505_01637_amd import binding as B
lib = B.lib()
NONE, P = (0, 0, 0, 0, 0), 1 << 20                # (addresses that nothing reads)
KERNELS = ("grad_rows_kernel", "rows_wide_kernel", "rows_kernel", "fast_kernel", "product_kernel", "copy_kernel", "rest_kernel", "drop_kernel")

def took():
    # (counting takes what it counts, and a part of a longer name counts there too: the longer ones first)
    n = {k: hip.fake_launches_of(k.encode()) for k in KERNELS}
    return {k: v for k, v in n.items() if v}

def linear(m, k, n, dtype=1, b=1, ld=0, at=0):
    lhs, rhs = (P + at, dtype, 0, k + ld, m * (k + ld)), (P, dtype, 0, n + ld, 0)
    d = B._LINEAR.pack(b, m, k, n, *lhs, *rhs, *NONE, *NONE, P, 0, 0, n, m * n, *NONE, 1, 0, 0, 0)
    size = C.c_size_t()
    assert lib.mrl_linear_bytes(d, C.addressof(size)) == 0, lib.mrl_last_error()
    if size.value:
        assert lib.mrl_linear(d, P, size.value - 1, None) == B.E_NOMEM
    assert lib.mrl_linear(d, P, size.value, None) == 0, lib.mrl_last_error()
    return took(), size.value

def grad(m, k, n, dtype=1, act=0, drop=0, bias=True, lhs=True, rhs=True):
    d = B._LINEAR_GRAD.pack(1, m, k, n, P, dtype, 0, n, 0, P, dtype, 0, k, 0, P, dtype, 0, n, 0, P, dtype, 0, n, 0, *((P, dtype, 0, k, 0) if lhs else NONE),
                            *((P, dtype, 0, n, 0) if rhs else NONE), *((P, 0, 0, 1, 0) if bias else NONE), act, drop, 0, 0)
    size = C.c_size_t()
    assert lib.mrl_linear_grad_bytes(d, C.addressof(size)) == 0, lib.mrl_last_error()
    assert lib.mrl_linear_grad(d, P, size.value, None) == 0, lib.mrl_last_error()
    return took(), size.value

took()
for m, k, n in ((0, 8, 8), (8, 8, 0)):
    assert linear(m, k, n) == ({}, 0), "nothing to compute"
assert linear(8, 0, 8)[0], "a sum over nothing still has an epilogue"
# one launch and no workspace where tiles fill the card or the sum is short
for shape in ((4096, 4096, 4096), (8192, 2048, 16384), (1, 2048, 16384), (1, 256, 256), (7, 500, 1001), (100, 72, 56)):
    for dtype in (0, 1):
        n, size = linear(*shape, dtype=dtype)
        assert sum(n.values()) == 1 and size == 0, (shape, dtype, n, size)
# few tiles over a long sum: split, one launch more and the partial sums
n, size = linear(1, 16384, 256)
assert n.get("rest_kernel") == 1 and size > 0, (n, size)
# operands that are not aligned: never a kernel that loads past the registers, unless a copy comes first
for m, k, n_, ld, at in ((300, 301, 302, 0, 0), (300, 304, 304, 1, 0), (300, 304, 304, 0, 2), (2, 3, 5, 0, 0), (3000, 3001, 3003, 0, 0), (1, 1, 1 << 22, 0, 0)):
    n, size = linear(m, k, n_, ld=ld, at=at)
    assert n.get("copy_kernel") or not (n.get("fast_kernel") or n.get("rows_kernel")), (m, k, n_, ld, at, n)
# a stride too long for offsets within a tile
n, size = linear(4, 4, 1 << 21, ld=8)
assert n.get("product_kernel") or n.get("rows_wide_kernel"), n
# a gradient: rows, two products, and one launch at most for all that is left
for shape in ((64, 64, 64), (1000, 511, 777), (4096, 2048, 2048)):
    for dtype in (0, 1):
        for act, drop, bias in ((0, 0, False), (2, 0, True), (1, 100, False), (0, 100, True)):
            n, size = grad(*shape, dtype=dtype, act=act, drop=drop, bias=bias)
            copies = n.pop("copy_kernel", 0)
            assert n.get("grad_rows_kernel", 0) == (1 if act or drop or bias else 0), (shape, n)
            assert n.get("rest_kernel", 0) <= 1 and copies <= 2
assert grad(64, 64, 64, act=2, bias=True)[0].get("rest_kernel") is None, "dbias of one block of rows needs no second launch"
assert grad(64, 64, 64, bias=False, lhs=False, rhs=False) == ({}, 0)
d = B._DROPOUT.pack(100, 72, P, 0, 0, 72, 0, *NONE, P, 0, 0, 72, 0, 6554, 1, 2)
assert lib.mrl_dropout(d, None) == 0 and took() == {"drop_kernel": 1}
d = B._DROPOUT.pack(100, 0, P, 0, 0, 72, 0, *NONE, P, 0, 0, 72, 0, 6554, 1, 2)
assert lib.mrl_dropout(d, None) == 0 and took() == {}
print("done")
"""


def test_what_is_launched(tmp_path):
    run_on_fake_hip(tmp_path, BODY)
