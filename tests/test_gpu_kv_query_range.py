"""Queries and keys of very different sizes: what counts is the score, not the size of its factors."""
import math

import pytest
import torch

import paper_2310_10537_b200 as mx
from kv_util import bounds, values
from test_gpu_kv_attention import _gen, _problem, _wide

pytestmark = pytest.mark.gpu
FMTS = [mx.MX_E4M3, mx.MX_E5M2, mx.MX_E2M1, mx.MX_INT8]
ONE = {mx.MX_E4M3: 0x38, mx.MX_E5M2: 0x3C, mx.MX_E2M1: 0x2, mx.MX_INT8: 64}  # code of 1.0


def _definition(q, cache, table, length, scale):
    """One sequence, one new token, FP64; scale enters as a number of 64 bits."""
    ps, (_, _, heads, dim) = cache.k_elems.shape[2], q.shape
    kv = cache.k_elems.shape[1]
    j = torch.arange(length, device="cuda")
    p, o = table[0, j // ps].long(), j % ps
    k = values(cache.k_elems[p, :, o], cache.k_scales[p, :, o], dim, cache.fmt)
    v = values(cache.v_elems[p, :, o], cache.v_scales[p, :, o], dim, cache.fmt)
    x = q[0, 0].double().view(kv, heads // kv, dim)
    s = torch.einsum("hgd,nhd->hgn", x, k) * scale
    w = torch.softmax(s, 2)
    out = torch.einsum("hgn,nhd->hgd", w, v)
    xv = torch.exp2(cache.v_scales[p, :, o].double() - 127)[..., :dim // 32]
    peak = (w.unsqueeze(3) * xv.permute(1, 0, 2).unsqueeze(1)).amax(2)
    least = peak.repeat_interleave(32, -1) * (v / xv.repeat_interleave(32, -1)).abs().sum(0).unsqueeze(1)
    absv = torch.einsum("hgn,nhd->hgd", w, v.abs())
    # A query enters in FP16 (FP32: in two terms, the second one scaled by 2^11), each block with its largest element in
    # [2^14, 2^15): off by at most 2^-25 / 2^14 = 2^-39 (2^-50) of the block's largest, beside the relative rounding.
    # In units of the score's bound (dim + 16) 2^-23 `size` of kv_util.bounds:
    part = 2.0 ** (-39 if q.dtype == torch.bfloat16 else -50) / ((dim + 16) * 2.0 ** -23)
    top = x.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
    size = (torch.einsum("hgd,nhd->hgn", x.abs() + part * top, k.abs()) * abs(scale)).amax(2)
    back = lambda t: t.reshape(1, 1, heads, *t.shape[2:])  # noqa: E731
    return back(out), back(torch.logsumexp(s, 2)), back(absv), back(size), back(least)


def _check(q, cache, table, lengths, scale):
    n = int(lengths[0])
    out, lse = mx.mx_kv_attention(q, cache, table, lengths, scale, return_lse=True)
    want, wlse, absv, size, least = _definition(q, cache, table, n, float(torch.tensor(scale)))
    tol, ltol = bounds(q.dtype, want, absv, size, least, q.shape[-1], n)
    assert bool(torch.isfinite(lse).all()) and bool(torch.isfinite(out).all())
    assert bool(((lse.double() - wlse).abs() <= ltol).all()), float(((lse.double() - wlse).abs() / ltol).max())
    assert bool(((out.double() - want).abs() <= tol).all()), float(((out.double() - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("power", [10, 24, 34, 60, 100])
def test_a_small_block_of_a_query_meets_a_large_block_of_a_key(power, fmt, dtype):
    """q = 1 in one block and 2^-power in another, a key 0 there and 2^power here: its score is the scale."""
    q, cache, table, lengths = _problem([70], 1, 1, 64, 16, fmt, dtype, 400)
    q.zero_()
    q[..., 3], q[..., 40] = 1.0, 2.0 ** -power
    cache.k_elems.zero_()
    cache.k_scales[..., :2] = 127
    for j in (5, 33, 69):
        page, off = int(table[0, j // 16]), j % 16
        cache.k_elems[page, 0, off, 40 if fmt != mx.MX_E2M1 else 20] = ONE[fmt]
        cache.k_scales[page, 0, off, 1] = 127 + power
    for scale in (1.0, -2.0, 5.0):
        _check(q, cache, table, lengths, scale)
        lse = float(mx.mx_kv_attention(q, cache, table, lengths, scale, return_lse=True)[1])
        assert abs(lse - math.log(67 + 3 * math.exp(scale))) < 1e-5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("power", [10, 20, 31])
def test_a_small_element_beside_a_large_one(power, dtype):
    """The same within a block."""
    q, cache, table, lengths = _problem([70], 1, 1, 64, 16, mx.MX_E4M3, dtype, 401)
    q.zero_()
    q[..., 3], q[..., 20] = 1.0, 1.375 * 2.0 ** -power
    cache.k_elems.zero_()
    cache.k_scales[..., :2] = 127
    for j in (5, 33, 69):
        page, off = int(table[0, j // 16]), j % 16
        cache.k_elems[page, 0, off, 20] = ONE[mx.MX_E4M3]
        cache.k_scales[page, 0, off, 0] = 127 + power
    # 1.375 2^-31 is a multiple of FP16's smallest step where the largest element is 2^14: nothing is rounded
    lse = float(mx.mx_kv_attention(q, cache, table, lengths, 1.0, return_lse=True)[1])
    assert abs(lse - math.log(67 + 3 * math.exp(1.375))) < 1e-5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_blocks_of_all_sizes(dim, fmt, dtype):
    """Blocks of the queries between 2^-90 and 2^30 of the others', the keys' the other way round: each counts alike."""
    for seed, (heads, group) in enumerate(((2, 3), (1, 9))):
        q, cache, table, lengths = _problem([333], heads, group, dim, 16, fmt, dtype, 410 + seed, spread=1)
        g = _gen(420 + seed)
        power = torch.randint(-90, 31, (heads, dim // 32), generator=g, device="cuda")
        by = torch.exp2(power.double()).repeat_interleave(32, -1).repeat_interleave(group, 0)
        q = (q.double() * by).to(dtype)
        s = cache.k_scales[..., :dim // 32].int() - power[None, :, None, :].int()
        assert int(s.min()) >= 0 and int(s.max()) < 255
        cache.k_scales[..., :dim // 32] = s.to(torch.uint8)
        _check(q, cache, table, lengths, dim ** -0.5)
        _check(*_wide((q, cache, table, lengths), 9000), dim ** -0.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
def test_large_keys_and_small_queries(fmt, dtype):
    """Keys up to FP32's largest numbers, queries as small as its smallest, and the other way round: ordinary scores."""
    top = {mx.MX_E4M3: 8, mx.MX_E5M2: 15, mx.MX_E2M1: 2, mx.MX_INT8: 0}[fmt]
    for power in (90, 110, 119, 126 - top, 124 - top):
        q, cache, table, lengths = _problem([333], 2, 4, 128, 16, fmt, dtype, 430, spread=1, middle=127 + power - top)
        # (keys up to 2^power times 2 to 2^top, scores of a few units)
        q = (q.double() * 2.0 ** -power).to(dtype)
        _check(q, cache, table, lengths, 2.0 ** -3.5)
    for power in (60, 100, 115):
        q, cache, table, lengths = _problem([333], 2, 4, 128, 16, fmt, dtype, 431, spread=1, middle=127 - power - top if power + top < 126 else 2)
        q = (q.double() * 2.0 ** min(power, 124 - top)).to(dtype)
        _check(q, cache, table, lengths, 2.0 ** -3.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scales_of_any_size(dtype):
    """The scale's size, too, is made up for by queries or keys."""
    for scale, qs, ks in ((1e30, -100, 0), (1e30, 0, -100), (3.3e38, -120, -8), (1e-30, 100, 0), (1e-30, 20, 80), (1e-38, 60, 66), (1e20, 60, -126), (1e-20, -50, 117),
                          (-1e30, -100, 0), (1e-42, 70, 69)):
        q, cache, table, lengths = _problem([333], 2, 4, 128, 16, mx.MX_E4M3, dtype, 440, spread=1)
        cache.k_scales[..., :4] = (cache.k_scales[..., :4].int() + ks).clamp(0, 254).to(torch.uint8)
        q = (q.double() * 2.0 ** qs).to(dtype)
        _check(q, cache, table, lengths, scale)
