"""The sigmoid of the routing scores over the whole range of floats, read off as the weights of a route that takes all
experts and divides by nothing.

With t = exp(-|x|), off by 2 units in the last place (the bound CUDA states for expf), s = 1 / (1 + t) or t / (1 + t): the error of
t counts once at most (2^-22), 1 + t, the reciprocal's last Newton-Raphson step and the product round once each (2^-24), and the
square of the approximate reciprocal's error (2^-46) is left of it: less than 2^-21 in all.  Below the normal range
the units of t and of the product are absolute: 3 * 2^-149."""
import pytest
import torch

import paper_2310_10537_b200 as mx

pytestmark = pytest.mark.gpu
REL, ABS = 2.0 ** -21, 2.0 ** -147


def _values(dtype):
    if dtype == torch.bfloat16:
        v = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
        return v[~v.isnan()]
    near = torch.linspace(-110, 110, 1 << 19, dtype=torch.float64).float()
    tiny = torch.logspace(-45, 2.1, 1 << 16, dtype=torch.float64).float()
    edge = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), 3.4e38, -3.4e38, 87.336, -87.336, 88.73, -88.73, 103.9, -103.9, -104.0, 16.6, 17.4])
    return torch.cat([near, tiny, -tiny, edge])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts,tokens", [(8, None), (8, 64), (16, 64), (256, 64)])  # a few lanes per token; a warp
def test_scores_over_the_whole_range(experts, tokens, dtype):
    topk = 8
    v = _values(dtype).cuda()
    v = v[torch.randperm(v.numel(), generator=torch.Generator().manual_seed(0)).cuda()]
    if experts == topk:
        x = torch.nn.functional.pad(v, (0, -v.numel() % experts)).view(-1, experts)
    else:  # the rest is never chosen (or ties with what is, at 0)
        x = torch.full((-(-v.numel() // topk), experts), -float("inf"), device="cuda", dtype=dtype)
        x[:, :topk] = torch.nn.functional.pad(v, (0, -v.numel() % topk)).view(-1, topk)
    for part in ([x] if tokens is None else x[:tokens * 64].split(tokens)):
        part = part.contiguous()
        ids, w = mx.mx_route(part, topk, mx.MX_SCORE_SIGMOID, renormalize=False)
        want = torch.sigmoid(part.double()).gather(1, ids.long())
        assert bool(((w.double() - want).abs() <= REL * want + ABS).all())
        assert bool((w[:, 1:] <= w[:, :-1]).all())
