"""The gradient of the routing weights does not depend on the groups: with any value in those fields the C call
writes what it writes without groups."""
import ctypes

import pytest
import torch

import paper_2310_10537_b200 as mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,experts", [(5, 16), (4096, 16), (7, 160)])
@pytest.mark.parametrize("groups,topk_groups,group_score", [(32, 1, 0), (0, 0, 0), (-1, -1, -1), (7, 9, 5)])
def test_backward_ignores_the_groups(tokens, experts, groups, topk_groups, group_score):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn(tokens, experts, generator=g, device="cuda")
    dw = torch.randn(tokens, 2, generator=g, device="cuda")
    ids, _ = mx.mx_route(x, 2)
    want = mx.mx_route_backward(dw, x, ids)
    got = torch.full_like(x, 77.0)
    r = mx.binding.mx_route_t(2, mx.MX_SCORE_SOFTMAX, groups, topk_groups, group_score, 1, 1.0)
    o = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, torch.cuda.current_stream().cuda_stream, 1)
    assert mx.lib().mx_route_backward(dw.data_ptr(), x.data_ptr(), ids.data_ptr(), tokens, experts, ctypes.byref(r), got.data_ptr(),
                                      ctypes.byref(o)) == mx.MX_OK
    assert torch.equal(got, want)
