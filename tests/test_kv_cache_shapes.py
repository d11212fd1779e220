"""mx_kv_cache: what it makes, and what it refuses, with and without pages (on the CPU: only memory is allocated)."""
import pytest
import torch

import paper_2310_10537_b200 as mx


@pytest.mark.parametrize("pages", [0, 2])
def test_shapes(pages):
    for fmt, dim, code, scale in ((mx.MX_E4M3, 160, 160, 8), (mx.MX_E2M1, 96, 48, 4), (mx.MX_INT8, 32, 32, 4)):
        c = mx.mx_kv_cache(pages, 5, 3, dim, fmt, device="cpu")
        assert c.k_elems.shape == c.v_elems.shape == (pages, 3, 5, code) and c.k_scales.shape == c.v_scales.shape == (pages, 3, 5, scale)
        assert all(t.dtype == torch.uint8 and not t.any() for t in c[:4]) and (c.dim, c.fmt) == (dim, fmt)


@pytest.mark.parametrize("pages", [0, 2, -1])
def test_refusals(pages):
    for bad in ((0, 2, 64, mx.MX_E4M3), (-1, 2, 64, mx.MX_E4M3), (16, 0, 64, mx.MX_E4M3), (16, 2, 48, mx.MX_E4M3), (16, 2, 0, mx.MX_E4M3), (16, 2, 64, mx.MX_E3M2), (16, 2, 64, mx.MX_E2M3),
                (16, 2, 64, 9), (16, 2, 64, -1)):
        with pytest.raises(ValueError):
            mx.mx_kv_cache(pages, *bad, device="cpu")
    if pages < 0:
        with pytest.raises(ValueError):
            mx.mx_kv_cache(pages, 16, 2, 64, mx.MX_E4M3, device="cpu")
