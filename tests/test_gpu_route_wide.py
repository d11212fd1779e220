"""Routing of many tokens to 129 .. 256 experts, which is done with sixteen lanes per token as from 2048 tokens on: the tests of
many tokens at those widths and lengths."""
import pytest
import torch

import paper_2310_10537_b200 as mx
import test_gpu_route_many as many
from test_gpu_route import SIG, SOFT, _logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(2048, 256, 8, 16, 8), (2049, 256, 5, 4, 1), (2051, 132, 8, 1, 1), (2050, 192, 8, 12, 6), (2053, 160, 1, 1, 1)])
def test_ids_are_exact_and_weights_within_fp32(T, E, k, groups, kg, score, dtype):
    many.test_ids_are_exact_and_weights_within_fp32(T, E, k, groups, kg, score, dtype)


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(2050, 256, 8, 8, 4), (2060, 160, 4, 10, 3)])
def test_bias_and_sum_of_two_group_scores(T, E, k, groups, kg, score):
    many.test_bias_and_sum_of_two_group_scores_as_with_few_tokens(T, E, k, groups, kg, score)


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(2049, 160, 6, 8, 3), (2048, 200, 8, 20, 4), (2100, 256, 8, 32, 9)])
def test_groups_of_any_size(T, E, k, groups, kg, score):
    many.test_groups_of_any_size(T, E, k, groups, kg, score)


@pytest.mark.parametrize("E", [132, 160, 256])
def test_few_tokens_are_routed_like_many(E):
    x = _logits(2100, E, E, torch.float32)
    ids, w = mx.mx_route(x, 8, SIG, groups=4, topk_groups=2)
    for t0, n in ((0, 1), (1000, 700), (2093, 7)):
        i1, w1 = mx.mx_route(x[t0:t0 + n].contiguous(), 8, SIG, groups=4, topk_groups=2)
        assert torch.equal(ids[t0:t0 + n], i1) and bool(((w[t0:t0 + n] - w1).abs() <= 128 * 2.0 ** -24 * w1).all())


def test_equal_rows_masked_experts_and_nan():
    E, inf = 256, float("inf")
    x = torch.randn(2048, E, device="cuda")
    x[0], x[1], x[2] = 0, -inf, 100.0
    x[3, 4] = float("nan")
    x[4] = torch.finfo(torch.float32).min
    ids, w = mx.mx_route(x, 3, SOFT)
    for r in (0, 1, 2, 4):
        assert ids[r].tolist() == [0, 1, 2]
    assert w[1].tolist() == [0, 0, 0] and ids[3, 0] == 4 and bool(torch.isnan(w[3]).all())
    assert torch.equal(ids[5:].long(), torch.topk(x[5:], 3).indices)
