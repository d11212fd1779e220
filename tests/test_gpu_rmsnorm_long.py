"""The norm of one row of 2^30 elements and more, where 32-bit byte counts have wrapped.

What it writes is compared with its own y, and y with the 64-bit formula.  A thread adds at most n / 1024 squares one after
the other and the CTA ten sums: the mean square is off by at most (n / 1024 + 10) 2^-24 of itself, its root by half of that."""
import pytest
import torch

import paper_2310_10537_b200 as mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,dtype", [(1 << 30, torch.float32), (954437184 + 40, torch.bfloat16), ((1 << 30) + 33, torch.float32)])
def test_a_row_of_2_to_30(dim, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, dim, generator=g, device="cuda", dtype=dtype)
    w = torch.ones(dim, device="cuda", dtype=dtype)
    y = torch.empty_like(x)
    elems, scales, h = mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, 1e-6, y_out=y)
    assert h is None
    total = sum(float(c.double().square().sum()) for c in x[0].split(1 << 26))
    s = (total / dim + 1e-6) ** -0.5
    off = 0.5 * (dim / 1024 + 10) * 2.0 ** -24 + 2.0 ** -21 + (0 if dtype == torch.float32 else 2.0 ** -8)
    for c0 in range(0, dim, 1 << 26):
        want = x[0, c0:c0 + (1 << 26)].double() * s
        assert bool(((y[0, c0:c0 + (1 << 26)].double() - want).abs() <= off * want.abs()).all())
    if dtype == torch.float32:  # y is what was quantized
        e, sc = mx.mx_quantize(y, 1, mx.MX_E4M3)
        assert torch.equal(e, elems) and torch.equal(sc, scales)
