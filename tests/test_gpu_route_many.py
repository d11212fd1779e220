"""Routing of many tokens (a few lanes per token) against the definition in 64 bits, and against calls with few.

Bounds as for few tokens: ids are exact where the choice compares logits, weights are within 64 * 2^-24."""
import ctypes

import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_route import SIG, SOFT, _choice64, _logits, _scores64, _weights64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(4099, 4, 2, 1, 1), (4096, 8, 8, 1, 1), (4111, 32, 4, 2, 1), (5000, 20, 3, 1, 1), (2050, 64, 6, 4, 2),
                                             (2048, 36, 8, 1, 1), (2111, 128, 8, 8, 4), (2049, 128, 1, 2, 1), (1, 256, 8, 16, 8), (77, 256, 5, 4, 1),
                                             (33, 132, 8, 1, 1), (19, 512, 8, 32, 3), (21, 512, 7, 8, 2), (40, 384, 8, 3, 2), (64, 192, 8, 12, 6)])
def test_ids_are_exact_and_weights_within_fp32(T, E, k, groups, kg, score, dtype):
    x = _logits(T, E, E + k, dtype)
    for renorm in (True, False):
        ids, w = mx.mx_route(x, k, score, groups=groups, topk_groups=kg, renormalize=renorm, scale=1.5)
        c = _choice64(x.double(), groups, kg, mx.MX_GROUP_MAX, None)
        assert torch.equal(ids.long(), torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k])
        ref = _weights64(_scores64(x, score), ids, renorm, 1.5)
        assert bool(((w.double() - ref).abs() <= 64 * 2.0 ** -24 * ref).all())


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(2100, 64, 4, 4, 2), (4100, 32, 4, 2, 1), (2065, 128, 8, 8, 4), (50, 256, 8, 8, 4), (30, 512, 8, 32, 9)])
def test_bias_and_sum_of_two_group_scores_as_with_few_tokens(T, E, k, groups, kg, score):
    """A bias off the 16-byte boundary goes the other way, of a warp per token."""
    x = _logits(T, E, E, torch.float32)
    held = torch.zeros(E + 4, device="cuda")
    bias = torch.randint(0, 3, (E,), device="cuda").float()   # whole numbers: sums are rounded alike
    held[1:E + 1] = bias
    args = dict(groups=groups, topk_groups=kg, group_score=mx.MX_GROUP_TOP2, scale=2.5)
    ids, w = mx.mx_route(x, k, score, bias=bias, **args)
    ids2, w2 = mx.mx_route(x, k, score, bias=held[1:E + 1], **args)
    s = _scores64(x, score) + bias.double()
    # candidates closer than FP32 can tell may change places: what is chosen is compared by its score
    got, got2 = s.gather(1, ids.long()), s.gather(1, ids2.long())
    assert bool(((got - got2).abs() <= 2.0 ** -20).all())
    same = (ids == ids2).all(1)
    ref = _weights64(_scores64(x, score), ids, True, 2.5)
    assert bool(((w.double() - ref).abs() <= 64 * 2.0 ** -24 * ref).all())
    assert bool(((w - w2)[same].abs() <= 128 * 2.0 ** -24 * w[same]).all())


def test_equal_rows_masked_experts_and_nan():
    inf, nan = float("inf"), float("nan")
    for T, E in ((4100, 16), (2100, 64), (2100, 128), (9, 256), (9, 512)):
        x = torch.randn(T, E, device="cuda")
        x[0] = 0
        x[1] = -inf
        x[2] = -inf
        x[2, 5] = 1.0
        x[3, 4] = nan
        x[4] = 100.0
        x[5] = torch.finfo(torch.float32).min
        x[6] = 0.0
        x[6, 3] = -0.0
        x[7, 15] = inf
        ids, w = mx.mx_route(x, 3, SOFT)
        third = torch.full((3,), 1 / 3, device="cuda")
        for r in (0, 1, 4, 5, 6):
            assert ids[r].tolist() == [0, 1, 2]
        assert torch.allclose(w[0], third) and torch.allclose(w[5], third) and w[1].tolist() == [0, 0, 0]
        assert ids[2].tolist() == [5, 0, 1] and w[2].tolist() == [1, 0, 0]
        assert ids[3, 0] == 4 and bool(torch.isnan(w[3]).all())
        assert ids[7, 0] == 15 and bool(torch.isnan(w[7]).any())
        assert torch.equal(ids[8:].long(), torch.topk(x[8:], 3).indices)
        ids, w = mx.mx_route(x, 3, SIG, renormalize=False)
        assert ids[1].tolist() == [0, 1, 2] and w[1].tolist() == [0, 0, 0] and w[4].tolist() == [1, 1, 1]
        assert ids[3, 0] == 4 and bool(torch.isnan(w[3, 0]))


def test_many_tokens_are_routed_like_each_alone():
    x = _logits(5000, 64, 5, torch.bfloat16)
    ids, w = mx.mx_route(x, 4, SIG, groups=2, topk_groups=1)
    for t0 in (0, 1000, 4990):
        i1, w1 = mx.mx_route(x[t0:t0 + 8], 4, SIG, groups=2, topk_groups=1)
        assert torch.equal(ids[t0:t0 + 8], i1) and bool(((w[t0:t0 + 8] - w1).abs() <= 128 * 2.0 ** -24 * w1).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k", [(2049, 4, 2), (2050, 28, 8), (2100, 64, 6), (33, 68, 1), (1, 128, 8), (70, 256, 5), (21, 512, 8)])
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
        big = 4 * dw.double().abs().amax(1, keepdim=True) * (1 / s.gather(1, ids.long()).sum(1, keepdim=True) if renorm else 1.0)
        half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
        assert bool(((got.double() - ref).abs() <= 128 * 2.0 ** -24 * big * s + half * ref.abs() + 1e-37).all())


@pytest.mark.parametrize("T,E", [(2050, 16), (3, 128)])
def test_gradient_ignores_ids_outside_and_handles_dead_rows(T, E):
    x = _logits(T, E, 5, torch.float32)
    x[2] = -float("inf")
    ids = torch.zeros(T, 2, dtype=torch.int32, device="cuda")
    ids[:3] = torch.tensor([[0, -1], [E + 83, 3], [0, 1]])
    ids[3:, 1] = E - 1
    dw = torch.ones(T, 2, device="cuda")
    for score in (SOFT, SIG):
        got = mx.mx_route_backward(dw, x, ids, score, False, 1.0)
        s = _scores64(x[:2], score)
        for t, e in ((0, 0), (1, 3)):
            ref = -s[t] * s[t, e] if score == SOFT else torch.zeros_like(s[t])
            ref[e] += s[t, e] if score == SOFT else s[t, e] * (1 - s[t, e])
            assert torch.allclose(got[t].double(), ref, rtol=1e-5, atol=1e-7)
        assert bool((mx.mx_route_backward(dw, x, ids, score, True, 1.0)[2] == 0).all())


def test_outputs_are_filled_and_nothing_else():
    T, E, k = 2051, 64, 6
    x = _logits(T, E, 9, torch.float32)
    ids, w = mx.mx_route(x, k)
    d = mx.mx_route_backward(w, x, ids)
    lib = mx.lib()
    raw_i = torch.full((T * k + 512,), -7, dtype=torch.int32, device="cuda")
    raw_w, raw_d = (torch.full((n + 512,), 77.0, device="cuda") for n in (T * k, T * E))
    route = mx.binding.mx_route_t(k, mx.MX_SCORE_SOFTMAX, 1, 1, mx.MX_GROUP_MAX, 1, 1.0)
    opts = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, torch.cuda.current_stream().cuda_stream, 0, 0)
    assert lib.mx_route(x.data_ptr(), None, T, E, ctypes.byref(route), raw_i[256:].data_ptr(), raw_w[256:].data_ptr(), ctypes.byref(opts)) == 0
    assert lib.mx_route_backward(w.data_ptr(), x.data_ptr(), ids.data_ptr(), T, E, ctypes.byref(route), raw_d[256:].data_ptr(), ctypes.byref(opts)) == 0
    for raw, want, n in ((raw_i, ids, T * k), (raw_w, w, T * k), (raw_d, d, T * E)):
        assert torch.equal(raw[256:256 + n], want.flatten())
        assert bool((raw[:256] == raw[0]).all()) and bool((raw[256 + n:] == raw[0]).all()) and float(raw[0]) in (-7, 77)


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("T,E,k,groups,kg", [(4100, 8, 2, 4, 2), (4097, 24, 8, 3, 2), (2050, 40, 4, 8, 3), (2048, 64, 6, 32, 7), (2049, 96, 8, 8, 4), (2111, 128, 8, 16, 5),
                                             (33, 160, 6, 8, 3), (50, 384, 8, 8, 2), (21, 480, 8, 20, 4), (19, 512, 8, 32, 32)])
def test_groups_of_any_size(T, E, k, groups, kg, score):
    x = _logits(T, E, E + groups, torch.float32)
    ids, w = mx.mx_route(x, k, score, groups=groups, topk_groups=kg)
    c = _choice64(x.double(), groups, kg, mx.MX_GROUP_MAX, None)
    assert torch.equal(ids.long(), torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k])
    ref = _weights64(_scores64(x, score), ids, True, 1.0)
    assert bool(((w.double() - ref).abs() <= 64 * 2.0 ** -24 * ref).all())
    # sums of two: the same as through the other way (a bias of zeros off the 16-byte boundary), which adds nothing
    if E // groups > 1:
        zeros = torch.zeros(E + 4, device="cuda")
        args = dict(groups=groups, topk_groups=kg, group_score=mx.MX_GROUP_TOP2)
        ids, w = mx.mx_route(x, k, SIG, bias=zeros[:E], **args)
        ids2, w2 = mx.mx_route(x, k, SIG, bias=zeros[1:E + 1], **args)
        assert torch.equal(ids, ids2) and bool(((w - w2).abs() <= 128 * 2.0 ** -24 * w).all())
