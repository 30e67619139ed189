"""Layer normalisation and 4-bit operands at the ends of what the calls take: the widest results, the most rows, the largest values, sizes of zero;
and sums whose order is the same however lhs is given."""
import pytest

from paper_2505_01637_amd import binding as B
from test_operators import U

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
