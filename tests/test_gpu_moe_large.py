"""Norm, gather, combine and grouped products on tensors of more than 2^32 elements (or bytes).

What lies beyond the 32-bit offsets must be what the same call gives for that part of the tensor alone, bit for
bit: rows, tokens and groups are computed independently of each other.  The one sum over all rows (the
weights' gradient) is fed zeros except in the last rows, and then held to the sum of those."""
import pytest
import torch

import paper_2310_10537_b200 as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _bytes(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 64, (n,), dtype=torch.uint8, device="cuda", generator=g)  # finite codes of every format


@pytest.mark.parametrize("dim", [4096, 4001])
def test_norm_and_its_gradient(dim):
    rows, last = (1 << 32) // dim // 128 * 128 + 256, 200
    x = torch.randn(rows, dim, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(dim, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 32
    r0 = rows - 256  # on a 128-row scale chunk
    e, s, h = mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, residual=x)
    e1, s1, h1 = mx.mx_rmsnorm_quantize(x[r0:], w, mx.MX_E4M3, residual=x[r0:])
    assert torch.equal(h[r0:], h1) and torch.equal(e[-e1.numel():], e1) and torch.equal(s[-s1.numel():], s1)
    del e, s
    dy = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    dy[rows - last:] = torch.randn(last, dim, device="cuda")
    dx, dw = mx.mx_rmsnorm_backward(dy, h, w)
    dx1, dw1 = mx.mx_rmsnorm_backward(dy[rows - last:], h[rows - last:], w)
    assert torch.equal(dx[rows - last:], dx1) and not bool(dx[: rows - last].any())
    h64 = h[rows - last:].double()
    terms = (dy[rows - last:].double() * h64 * torch.rsqrt((h64 * h64).mean(1, keepdim=True) + 1e-5)).abs().sum(0)
    # each is within (terms + 24 steps of each term's norm) half-ulps of the same 64-bit sum
    assert bool(((dw - dw1).abs().double() <= 2 * (last + dim / 64 + 48) * 2.0 ** -24 * terms).all())


def test_gather_and_combine():
    dim = 16384
    T = (1 << 32) // dim + 128
    ids = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    ids[1::2] = 1
    plan = mx.mx_moe_plan(ids, 3, 64)
    row = plan.row_of[:, 0].long()
    e, s = _bytes(T * dim, 1), _bytes(T * dim // 32, 2)
    ge, gs = mx.mx_moe_gather(e, s, dim, mx.MX_E4M3, plan, mx.MX_SCALES_LINEAR)
    assert ge.numel() > 1 << 32
    for part in (slice(0, 300), slice(T - 300, T)):
        assert torch.equal(ge.view(plan.rows, dim)[row[part]], e.view(T, dim)[part])
        assert torch.equal(gs.view(plan.rows, dim // 32)[row[part]], s.view(T, dim // 32)[part])
    del e, s, ge, gs
    y = torch.randn(plan.rows, dim, dtype=torch.bfloat16, device="cuda")
    out = mx.mx_moe_combine(y, None, plan)
    for part in (slice(0, 300), slice(T - 300, T)):
        assert torch.equal(out[part], y[row[part]])
    dy, dw = mx.mx_moe_combine_backward(out, y, None, plan)
    for part in (slice(0, 300), slice(T - 300, T)):
        assert torch.equal(dy[row[part]], out[part])
        sq = out[part].double().square().sum(1, keepdim=True)
        assert bool(((dw[part].double() - sq).abs() <= (dim / 32 + 20) * 2.0 ** -24 * sq).all())


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_grouped_product_with_a_large_result(out_dtype):
    N, K, last = 16384, 128, 448
    rows = (1 << 32) // N + last
    off = torch.tensor([0, 64, 64, rows - last, rows], dtype=torch.int32, device="cuda")
    x, w = torch.randn(rows, K, device="cuda"), torch.randn(4, N, K, device="cuda")
    eb, sb = mx.mx_quantize(w, 2, mx.MX_E4M3)
    e1, s1 = mx.mx_quantize(w[3].contiguous(), 1, mx.MX_E4M3)
    c = mx.mx_gemm_grouped(*mx.mx_quantize(x, 1, mx.MX_E4M3), eb, sb, off, rows, N, K, mx.MX_E4M3, mx.MX_E4M3, out_dtype=out_dtype, check_status=True)
    want = mx.mx_gemm_grouped(*mx.mx_quantize(x[rows - last:].contiguous(), 1, mx.MX_E4M3), e1, s1, torch.tensor([0, last], dtype=torch.int32, device="cuda"),
                              last, N, K, mx.MX_E4M3, mx.MX_E4M3, out_dtype=out_dtype, check_status=True)
    assert c.numel() > 1 << 32 and torch.equal(c[rows - last:], want)


def test_grouped_product_with_large_weights():
    G, N, K = 68, 16384, 4096
    eb, sb = _bytes(G * N * K, 3), _bytes(G * N * K // 32, 4) + 96
    assert eb.numel() > 1 << 32
    x = torch.randn(G * 64, K, device="cuda")
    off = torch.arange(0, G * 64 + 1, 64, dtype=torch.int32, device="cuda")
    c = mx.mx_gemm_grouped(*mx.mx_quantize(x, 1, mx.MX_E4M3), eb, sb, off, G * 64, N, K, mx.MX_E4M3, mx.MX_E4M3, check_status=True)
    want = mx.mx_gemm_grouped(*mx.mx_quantize(x[-64:].contiguous(), 1, mx.MX_E4M3), eb[-N * K:], sb[-N * K // 32:], off[:2], 64, N, K,
                              mx.MX_E4M3, mx.MX_E4M3, check_status=True)
    assert bool(want.isfinite().all()) and bool(want.any()) and torch.equal(c[-64:], want)


def test_grouped_product_along_k_with_a_large_result():
    G, M, N = 64, 8192, 8200
    a, b = torch.randn(M, G * 128, device="cuda"), torch.randn(N, G * 128, device="cuda")
    off = torch.arange(0, G * 128 + 1, 128, dtype=torch.int32, device="cuda")
    c = mx.mx_gemm_grouped_k(*mx.mx_quantize(a, 1, mx.MX_E5M2), *mx.mx_quantize(b, 1, mx.MX_E4M3), off, M, N, G * 128, mx.MX_E5M2, mx.MX_E4M3, check_status=True)
    want = mx.mx_gemm_grouped_k(*mx.mx_quantize(a[:, -128:].contiguous(), 1, mx.MX_E5M2), *mx.mx_quantize(b[:, -128:].contiguous(), 1, mx.MX_E4M3),
                                off[:2], M, N, 128, mx.MX_E5M2, mx.MX_E4M3, check_status=True)
    assert c.numel() > 1 << 32 and torch.equal(c[-1], want[0])
