"""Norm and its gradient for rows that start anywhere, at the sizes where the number of rows or their length changes
the way they go.  The checks and their bounds are those of the other norm tests."""
import pytest
import torch

import paper_2310_10537_b200 as mx
import test_gpu_rmsnorm as norm
from gpu_util import GUARD

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim", [(1023, 257), (1024, 257), (1025, 1), (1100, 31), (2500, 7), (1030, 511), (1031, 513), (1024, 1001),
                                      (1040, 1023), (1033, 1025), (2500, 255)])
def test_gradient_of_many_short_rows(rows, dim, dtype):
    norm.test_backward_against_the_formula(rows, dim, dtype)


@pytest.mark.parametrize("rows,dim", [(149, 767), (200, 769), (149, 1500), (160, 2047), (150, 2049), (1, 767), (148, 2047), (333, 9),
                                      (155, 8191), (3, 12345)])
def test_output_of_rows_of_odd_length(rows, dim):
    norm.test_mx_output_is_the_quantized_norm(rows, dim, mx.MX_E4M3, mx.MX_SCALES_SWIZZLED)
    norm.test_bf16_tensors_give_the_bytes_of_fp32_ones(rows, dim)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim", [(3, 5), (151, 257), (9, 1001), (150, 2047), (201, 4001)])
def test_nothing_outside_is_written_and_h_may_replace_an_input(rows, dim, dtype):
    x, r, w = norm._inputs(rows, dim, 8, dtype)
    y = torch.empty_like(x)
    e, s, h = mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, norm.EPS, residual=r, y_out=y)
    n = rows * dim
    raws = []

    def guarded(t):
        raw = torch.full((t.numel() * t.element_size() + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        raws.append((raw, t.numel() * t.element_size()))
        return raw[GUARD:GUARD + t.numel() * t.element_size()].view(t.dtype).view(t.shape)

    for alias in (None, "x", "residual"):
        raws.clear()
        out, y2 = (guarded(e), guarded(s)), guarded(x)
        x2, r2 = guarded(x).copy_(x), guarded(x).copy_(r)
        h2 = guarded(x) if alias is None else x2 if alias == "x" else r2
        e2, s2, h3 = mx.mx_rmsnorm_quantize(x2, w, mx.MX_E4M3, norm.EPS, residual=r2, h_out=h2, y_out=y2, out=out)
        assert torch.equal(h3, h) and torch.equal(e2, e) and torch.equal(s2, s) and torch.equal(y2, y)
        assert h3.data_ptr() == h2.data_ptr() and h3.numel() == n
        for raw, size in raws:
            assert bool((raw[:GUARD] == 0xA5).all()) and bool((raw[GUARD + size:] == 0xA5).all())
