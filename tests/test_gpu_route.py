"""Routing and its gradient against the definition in 64 bits.

Where the choice compares logits, or scores that are far apart for different logits (BF16 logits of at most
8: neighbours differ by 2^-8 relative, their sigmoids by more than 2e-6), the ids are compared exactly,
ties included.  With a bias, c = s + bias is off by at most 2^-22 in FP32 (s and c are below 4): the ids have to be a
right choice up to that."""
import pytest
import torch

import paper_2310_10537_b200 as mx

pytestmark = pytest.mark.gpu
SOFT, SIG = mx.MX_SCORE_SOFTMAX, mx.MX_SCORE_SIGMOID


def _logits(T, E, seed, dtype, ties=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = 2 * torch.randn(T, E, generator=g, device="cuda")
    if ties:
        x = torch.round(x * 4) / 4  # few distinct values: many ties
    return x.clamp(-8, 8).bfloat16().to(dtype)


def _scores64(x, score):
    x = x.double()
    return torch.softmax(x, 1) if score == SOFT else torch.sigmoid(x)


def _choice64(c, groups, topk_groups, group_score, s):
    """c with the experts of groups that are not kept at -inf (lowest group first among equals)."""
    if groups == 1:
        return c
    T, E = c.shape
    v = c.view(T, groups, -1)
    if group_score == mx.MX_GROUP_TOP2:
        gs = torch.sort(v, dim=2, descending=True).values[:, :, :2].sum(2)
    else:
        gs = v.max(2).values
    drop = torch.sort(gs, dim=1, descending=True, stable=True).indices[:, topk_groups:]
    return v.clone().scatter_(1, drop.unsqueeze(2).expand(-1, -1, v.shape[2]), -float("inf")).view(T, E)


def _weights64(s, ids, renorm, scale):
    w = s.gather(1, ids.long())
    return scale * (w / w.sum(1, keepdim=True) if renorm else w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(1, 1, 1, 1, 1), (1, 8, 2, 1, 1), (5, 33, 7, 1, 1), (64, 64, 2, 1, 1), (130, 256, 8, 8, 4),
                                             (67, 160, 6, 8, 3), (9, 40, 5, 4, 2), (31, 1000, 32, 1, 1), (6, 1024, 8, 32, 2), (40, 384, 8, 8, 8),
                                             (33, 96, 4, 32, 5), (3, 512, 1, 2, 1), (7, 24, 24, 1, 1)])
def test_ids_are_exact_and_weights_within_fp32(T, E, k, groups, kg, score, dtype):
    x = _logits(T, E, E + k, dtype)
    for renorm in (True, False):
        ids, w = mx.mx_route(x, k, score, groups=groups, topk_groups=kg, renormalize=renorm, scale=1.5)
        c = _choice64(x.double(), groups, kg, mx.MX_GROUP_MAX, None)  # both scores keep the logits' order
        want = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids.long(), want)
        ref = _weights64(_scores64(x, score), ids, renorm, 1.5)
        # exp, the sum of at most 1024 terms (a chain of 32 + 5), two divisions
        assert bool(((w.double() - ref).abs() <= 64 * 2.0 ** -24 * ref).all())


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(130, 256, 8, 8, 4), (67, 160, 6, 8, 3), (20, 64, 4, 16, 4), (11, 48, 3, 16, 4), (50, 32, 4, 32, 9),
                                             (40, 128, 8, 1, 1)])
def test_bias_and_sum_of_two_group_scores(T, E, k, groups, kg, score):
    x = _logits(T, E, 3 * E + k, torch.float32, ties=False)
    bias = torch.randn(E, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 0.2
    for b in (bias, None):
        ids, w = mx.mx_route(x, k, score, bias=b, groups=groups, topk_groups=kg, group_score=mx.MX_GROUP_TOP2, scale=2.5)
        s = _scores64(x, score)
        c = s if b is None else s + b.double()
        assert all(len(set(r)) == k for r in ids.tolist())
        # no group left out is better than one that was chosen from, no candidate better than a chosen one
        v = c.view(T, groups, -1)
        gs = torch.sort(v, dim=2, descending=True).values[:, :, :2].sum(2)
        kth = torch.sort(gs, dim=1, descending=True).values[:, kg - 1:kg]
        mine = gs.gather(1, ids.long() // (E // groups))
        tol = 2.0 ** -21
        assert bool((mine >= kth - tol).all())
        got = c.gather(1, ids.long())
        assert bool((got[:, :-1] >= got[:, 1:] - tol).all()) if k > 1 else True
        sure = (gs > kth + tol).repeat_interleave(E // groups, 1) if groups > 1 else torch.ones_like(c, dtype=torch.bool)
        rest = torch.where(sure, c, torch.full_like(c, -1e9)).scatter(1, ids.long(), -1e9)
        assert bool((rest.max(1).values <= got[:, -1] + tol).all())
        ref = _weights64(s, ids, True, 2.5)
        assert bool(((w.double() - ref).abs() <= 64 * 2.0 ** -24 * ref).all())


def test_equal_rows_masked_experts_nan_and_saturated_scores():
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(8, 16, device="cuda")
    x[1] = -inf
    x[2] = -inf
    x[2, 5] = 1.0
    x[3, 4] = nan
    x[4] = 100.0                 # sigmoid is 1 for all
    x[5] = torch.finfo(torch.float32).min
    x[6, 3] = -0.0
    x[7, 15] = inf
    ids, w = mx.mx_route(x, 3, SOFT)
    assert ids[0].tolist() == [0, 1, 2] and torch.allclose(w[0], torch.full((3,), 1 / 3, device="cuda"))
    assert ids[1].tolist() == [0, 1, 2] and w[1].tolist() == [0, 0, 0]
    assert ids[2].tolist() == [5, 0, 1] and w[2].tolist() == [1, 0, 0]
    assert ids[3, 0] == 4 and bool(torch.isnan(w[3]).all())
    assert ids[4].tolist() == [0, 1, 2] and ids[5].tolist() == [0, 1, 2] and torch.allclose(w[5], w[0])
    assert ids[6].tolist() == [0, 1, 2]
    assert ids[7, 0] == 15 and bool(torch.isnan(w[7]).any())
    ids, w = mx.mx_route(x, 3, SIG, renormalize=False)
    assert ids[1].tolist() == [0, 1, 2] and w[1].tolist() == [0, 0, 0]
    assert ids[4].tolist() == [0, 1, 2] and w[4].tolist() == [1, 1, 1]
    assert ids[3, 0] == 4 and bool(torch.isnan(w[3, 0])) and bool((w[3, 1:] == 0.5).all())
    ids, w = mx.mx_route(x, 3, SIG)
    assert w[1].tolist() == [0, 0, 0]
    # a group whose experts are all masked is still a group
    y = torch.full((1, 8), -inf, device="cuda")
    y[0, 6] = 0.0
    ids, w = mx.mx_route(y, 3, SOFT, groups=4, topk_groups=2)
    assert ids[0].tolist() == [6, 0, 1] and w[0].tolist() == [1, 0, 0]
    e = mx.mx_route(x[:0], 3)
    assert e[0].shape == (0, 3) and e[1].shape == (0, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (5, 33, 7), (64, 64, 2), (130, 256, 8), (67, 160, 6), (31, 1000, 32), (9, 1024, 1)])
def test_gradient_against_the_formula(T, E, k, score, dtype):
    x = _logits(T, E, E, dtype, ties=False)
    for renorm in (True, False):
        ids, _ = mx.mx_route(x, k, score, renormalize=renorm, scale=2.0)
        dw = torch.randn(T, k, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
        got = mx.mx_route_backward(dw, x, ids, score, renorm, 2.0)
        with torch.enable_grad():
            x64 = x.double().requires_grad_(True)
            ref = torch.autograd.grad((_weights64(_scores64(x64, score), ids, renorm, 2.0) * dw.double()).sum(), x64)[0]
        s = _scores64(x, score)
        # terms that cancel: |ds| up to 2 * 2 |dw| / S each, times s
        big = 4 * dw.double().abs().amax(1, keepdim=True) * (1 / s.gather(1, ids.long()).sum(1, keepdim=True) if renorm else 1.0)
        half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
        assert bool(((got.double() - ref).abs() <= 128 * 2.0 ** -24 * big * s + half * ref.abs() + 1e-37).all())


def test_gradient_against_differences():
    x = _logits(4, 24, 11, torch.float32, ties=False)
    for score in (SOFT, SIG):
        ids, _ = mx.mx_route(x, 3, score)
        dw = torch.randn(4, 3, generator=torch.Generator(device="cuda").manual_seed(12), device="cuda")
        got = mx.mx_route_backward(dw, x, ids, score, True, 1.0)
        for t, e in ((0, int(ids[0, 0])), (1, int(ids[1, 2])), (2, 7), (3, 23)):
            d = torch.zeros(4, 24, dtype=torch.float64, device="cuda")
            d[t, e] = 1e-5
            f = lambda z: float((_weights64(_scores64(z, score), ids, True, 1.0) * dw.double()).sum())  # noqa: E731
            num = (f(x.double() + d) - f(x.double() - d)) / 2e-5
            assert abs(num - float(got[t, e])) <= 1e-5


def test_gradient_ignores_ids_outside_and_handles_dead_rows():
    x = _logits(3, 16, 5, torch.float32)
    x[2] = -float("inf")
    ids = torch.tensor([[0, -1], [99, 3], [0, 1]], dtype=torch.int32, device="cuda")
    dw = torch.ones(3, 2, device="cuda")
    got = mx.mx_route_backward(dw, x, ids, SOFT, False, 1.0)
    s = _scores64(x[:2], SOFT)
    for t, e in ((0, 0), (1, 3)):
        ref = -s[t] * s[t, e]
        ref[e] += s[t, e]
        assert torch.allclose(got[t].double(), ref, rtol=1e-5, atol=1e-7)
    assert bool((mx.mx_route_backward(dw, x, ids, SOFT, True, 1.0)[2] == 0).all())
    assert mx.mx_route_backward(dw[:0], x[:0], ids[:0]).shape == (0, 16)


def test_python_refuses_wrong_tensors():
    x = torch.zeros(4, 16, device="cuda")
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    dw = torch.zeros(4, 2, device="cuda")
    for f in (lambda: mx.mx_route(x.t(), 2), lambda: mx.mx_route(x[0], 2), lambda: mx.mx_route(x, 2, bias=torch.zeros(8, device="cuda")),
              lambda: mx.mx_route(x.cpu(), 2), lambda: mx.mx_route_backward(dw, x, ids.long()), lambda: mx.mx_route_backward(dw[:3], x, ids)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: mx.mx_route(x, 17), lambda: mx.mx_route(x, 0), lambda: mx.mx_route(x, 2, groups=3), lambda: mx.mx_route(x, 9, groups=2),
              lambda: mx.mx_route(x, 2, 5), lambda: mx.mx_route(torch.zeros(1, 2048, device="cuda"), 2)):
        with pytest.raises(mx.MxError):
            f()
    with pytest.raises(TypeError):
        mx.mx_route(x.half(), 2)
