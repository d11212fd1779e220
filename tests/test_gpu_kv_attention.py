"""Attention of the newest tokens over the paged cache against its definition in 64 bits (bounds: kv_util.bounds)."""
import math

import numpy as np
import pytest
import torch

import paper_2310_10537_b200 as mx
from kv_util import attention64, bounds, random_cache

pytestmark = pytest.mark.gpu
FMTS = [mx.MX_E4M3, mx.MX_E5M2, mx.MX_E2M1, mx.MX_INT8]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _problem(lengths, heads, group, dim, page_size, fmt, dtype, seed, new=1, spread=3, middle=None, spare=2):
    g = _gen(seed)
    need = [-(-max(n, 0) // page_size) for n in lengths]
    pages = sum(need) + spare
    cache = random_cache(pages, page_size, heads, dim, fmt, g, spread, middle)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), max(need + [1])), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    q = torch.randn(len(lengths), new, heads * group, dim, generator=g, device="cuda").to(dtype)
    return q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def _check(q, cache, table, lengths, scale=None, window=0, got=None, **kw):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    out, lse = mx.mx_kv_attention(q, cache, table, lengths, scale, window, return_lse=True, **kw) if got is None else got
    assert out.dtype == q.dtype and out.shape == q.shape and lse.shape == q.shape[:-1]
    want, wlse, absv, size, least = attention64(q, cache, table, lengths, scale, window)
    tol, ltol = bounds(q.dtype, want, absv, size, least, q.shape[-1], int(lengths.max()))
    empty = wlse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert not out[empty].any()
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), f"out off by {float((err / tol).max()):.3g} of its bound"
    lerr = torch.where(empty, 0.0, (lse.double() - wlse).abs())
    assert bool((lerr <= ltol).all()), f"lse off by {float((lerr / ltol).max()):.3g} of its bound"
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_formats_and_rows(dim, fmt, dtype):
    lengths = [1, 0, 15, 16, 17, 100, 333]
    for seed, (heads, group, ps) in enumerate(((2, 4, 16), (1, 1, 24), (3, 9, 64))):
        _check(*_problem(lengths, heads, group, dim, ps, fmt, dtype, seed))


def _wide(problem, tokens):
    """The same with a table that could hold `tokens` tokens of each sequence: long enough for them to be split."""
    q, cache, table, lengths = problem
    more = -(-tokens // cache.k_elems.shape[2]) - table.shape[1]
    return q, cache, torch.nn.functional.pad(table, (0, max(more, 0)), value=-1).contiguous(), lengths


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_split_sequences(dim, fmt, dtype):
    """Few sequences, of which several blocks work on one; many, of which one block works on several."""
    _check(*_wide(_problem([1, 0, 63, 64, 65, 700, 1500, 0], 2, 4, dim, 32, fmt, dtype, 11, new=3), 10000), window=0)
    _check(*_wide(_problem([1500, 3, 900], 1, 11, dim, 24, fmt, dtype, 12), 10000), window=611)
    _check(*_wide(_problem([(37 * i) % 300 for i in range(70)], 2, 2, dim, 16, fmt, dtype, 13), 10000))


def test_long_sequences_of_one_head():
    """More parts than a warp has lanes, for both results."""
    for dtype, dim in ((torch.bfloat16, 128), (torch.float32, 64)):
        _check(*_problem([70000], 1, 3, dim, 128, mx.MX_E4M3, dtype, 14))
        _check(*_wide(_problem([20000, 5], 1, 8, dim, 48, mx.MX_E2M1, dtype, 15, new=2), 90000), window=15000)


def test_tokens_that_lie_one_after_the_other():
    """Whole tiles in a row in memory, across pages too, and tiles with a gap or a hidden page among them."""
    for dim, fmt in ((64, mx.MX_E4M3), (128, mx.MX_E4M3), (256, mx.MX_INT8), (128, mx.MX_E2M1), (96, mx.MX_E5M2)):
        for heads in (1, 2):
            q, cache, table, lengths = _problem([400, 256, 130], heads, 4, dim, 16, fmt, torch.bfloat16, 16 + heads)
            n = int((table >= 0).sum())
            table[table >= 0] = torch.arange(n, dtype=torch.int32, device="cuda")
            _check(q, cache, table, lengths)
            table[0, 5] = -1
            table[1, 3], table[1, 4] = int(table[1, 4]), int(table[1, 3])
            _check(q, cache, table, lengths)


def test_two_calls_with_a_workspace_of_their_own():
    probs = [_wide(_problem([2000, 50], 2, 4, 64, 16, mx.MX_E4M3, torch.bfloat16, 30 + i), 30000) for i in range(2)]
    want = [mx.mx_kv_attention(*p) for p in probs]
    need = 1 << 25
    spaces = [torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") for _ in probs]
    graphs = []
    for p, ws in zip(probs, spaces):
        mx.mx_kv_attention(*p, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = mx.mx_kv_attention(*p, workspace=ws)
        graphs.append((g, out))
    streams = [torch.cuda.Stream() for _ in probs]
    for _ in range(4):
        for (g, out), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                out.fill_(7)
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, w) for (_, out), w in zip(graphs, want))
    # one workspace, one call after the other on a stream
    a = [mx.mx_kv_attention(*probs[i % 2], workspace=spaces[0]) for i in range(4)]
    assert all(torch.equal(o, want[i % 2]) for i, o in enumerate(a))


@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 9, 15, 16, 17, 32, 33, 71])
def test_groups(group):
    for dtype in (torch.bfloat16, torch.float32):
        _check(*_problem([200, 65, 3], 2, group, 64, 32, mx.MX_E4M3, dtype, group))


@pytest.mark.parametrize("page_size", [1, 2, 3, 7, 8, 16, 31, 48, 100, 128, 512])
def test_pages(page_size):
    _check(*_problem([1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 400], 2, 4, 128, page_size, mx.MX_E4M3, torch.bfloat16, page_size))
    _check(*_problem([5, 260], 1, 2, 96, page_size, mx.MX_E2M1, torch.float32, page_size))


@pytest.mark.parametrize("new", [1, 2, 3, 5, 8])
@pytest.mark.parametrize("window", [0, 1, 2, 16, 33, 100, 1 << 40])
def test_new_tokens_and_windows(new, window):
    lengths = [0, 1, 2, 4, 7, 40, 150, 257]
    _check(*_problem(lengths, 2, 3, 64, 16, mx.MX_E4M3, torch.bfloat16, new + window % 97, new), window=window)
    _check(*_problem(lengths, 1, 5, 128, 24, mx.MX_INT8, torch.float32, new + window % 97 + 1, new), window=window)


@pytest.mark.parametrize("lengths", [[40000], [5000, 1, 20000], [3000] * 40, [1] * 300, [0] * 5, [17] * 1000, list(range(0, 2000, 13))])
def test_lengths(lengths):
    for heads, group in ((1, 1), (2, 8)):
        _check(*_problem(lengths, heads, group, 64, 64, mx.MX_E4M3, torch.bfloat16, len(lengths)))


def test_lengths_beyond_the_table_and_below_zero():
    q, cache, table, lengths = _problem([50, 60, 70], 2, 2, 64, 16, mx.MX_E4M3, torch.bfloat16, 3)
    lengths[0] = 1 << 30
    lengths[1] = -5
    _check(q, cache, table, lengths)
    _check(q, cache, table[:, :0].contiguous(), lengths)
    # a cache without pages, tables short and long
    empty = mx.mx_kv_cache(0, 16, 2, 64, mx.MX_E4M3)
    for t in (table, torch.zeros((3, 4000), dtype=torch.int32, device="cuda")):
        out, lse = mx.mx_kv_attention(q, empty, t, lengths, return_lse=True)
        assert not out.any() and bool((lse == -math.inf).all())


def test_pages_outside_the_cache_are_not_seen():
    q, cache, table, lengths = _problem([200, 300, 50, 90], 2, 4, 128, 16, mx.MX_E4M3, torch.bfloat16, 4, new=2)
    table[0, 3] = -1
    table[0, 12] = cache.k_elems.shape[0]
    table[1, 0] = 1 << 30
    table[1, 18] = -(1 << 31)
    table[2] = -7
    _check(q, cache, table, lengths)
    _check(q, cache, table, lengths, window=40)


@pytest.mark.parametrize("fmt", FMTS)
def test_what_nobody_sees_has_no_influence(fmt):
    """NaN scales, codes of NaN and Inf in free pages, behind the last token and before a window."""
    for new, window in ((1, 0), (3, 20), (1, 33)):
        q, cache, table, lengths = _problem([37, 100, 5, 64], 2, 4, 128, 16, fmt, torch.bfloat16, 5, new)
        plain = mx.mx_kv_attention(q, cache, table, lengths, window=window, return_lse=True)
        seen = torch.zeros(cache.k_elems.shape[0], 16, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lengths.tolist()):
            for j in range(max(0, n - new + 1 - window) if window else 0, n):
                seen[table[b, j // 16].long(), j % 16] = True
        hide = ~seen[:, None, :, None]
        for t in (cache.k_elems, cache.v_elems):
            t.copy_(torch.where(hide, torch.tensor(0x7F, dtype=torch.uint8, device="cuda"), t))
        for t in (cache.k_scales, cache.v_scales):
            t.copy_(torch.where(hide, torch.tensor(0xFF, dtype=torch.uint8, device="cuda"), t))
        again = mx.mx_kv_attention(q, cache, table, lengths, window=window, return_lse=True)
        assert torch.equal(plain[0], again[0]) and torch.equal(plain[1], again[1])


def test_a_draft_does_not_see_a_later_ones_nan():
    """The newest token's value is NaN in one block, its key NaN in one head: earlier queries do not see it."""
    q, cache, table, lengths = _problem([40, 33], 2, 2, 128, 16, mx.MX_E4M3, torch.bfloat16, 6, new=2)
    plain = mx.mx_kv_attention(q, cache, table, lengths)
    p, o = int(table[0, 39 // 16]), 39 % 16
    cache.v_scales[p, 0, o, 2] = 255
    cache.k_scales[p, 1, o, 0] = 255
    out, lse = mx.mx_kv_attention(q, cache, table, lengths, return_lse=True)
    assert torch.equal(out[0, 0], plain[0, 0]) and torch.equal(out[1], plain[1])
    assert out[0, 1, :2, 64:96].isnan().all() and torch.equal(out[0, 1, :2, :64], plain[0, 1, :2, :64]) and torch.equal(out[0, 1, :2, 96:], plain[0, 1, :2, 96:])
    assert out[0, 1, 2:].isnan().all() and lse[0, 1, 2:].isnan().all() and not lse[0, 1, :2].isnan().any()


def test_nan_and_infinite_queries():
    q, cache, table, lengths = _problem([70, 70], 2, 2, 64, 16, mx.MX_E4M3, torch.float32, 8)
    plain = mx.mx_kv_attention(q, cache, table, lengths)
    q[0, 0, 1, 3] = math.nan
    q[1, 0, 2, 60] = math.inf
    out = mx.mx_kv_attention(q, cache, table, lengths)
    assert out[0, 0, 1].isnan().all() and out[1, 0, 2].isnan().all()
    keep = torch.ones(2, 1, 4, dtype=torch.bool, device="cuda")
    keep[0, 0, 1] = keep[1, 0, 2] = False
    assert torch.equal(out[keep], plain[keep])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sizes_of_numbers(dtype):
    """Queries, keys and values of very different sizes; sharp and flat softmaxes."""
    for seed, (qs, spread, middle) in enumerate(((1e-30, 3, None), (30.0, 3, None), (1e30, 1, 30), (0.0, 3, None), (1.0, 12, 118), (1e-3, 3, 225))):
        q, cache, table, lengths = _problem([500, 33, 1], 2, 4, 64, 16, mx.MX_E4M3, dtype, 20 + seed, spread=spread, middle=middle)
        if middle == 30:   # large queries, small keys, ordinary values
            cache.v_scales.copy_((cache.v_scales.int() + 90).clamp(max=254).to(torch.uint8))
        if middle == 225:  # large values, ordinary keys
            cache.k_scales.copy_((cache.k_scales.int() - 105).clamp(min=0).to(torch.uint8))
        _check((q.float() * qs).to(dtype), cache, table, lengths)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_of_seen_tokens_differ_by_many_powers_of_two(dtype):
    """A token of weight 2^-60 whose value is 2^100 times the others', and the other way round."""
    q, cache, table, lengths = _problem([100], 1, 1, 64, 16, mx.MX_E4M3, dtype, 30)
    q.zero_()
    q[..., 0] = 1.0
    cache.k_elems.zero_()
    cache.k_elems[..., 0] = 0x38  # 1.0
    cache.k_scales.fill_(127)
    cache.v_scales.fill_(100)
    for far, weight in ((200, 60.0), (200, 130.0), (20, -60.0), (60, -5.0)):
        p, o = int(table[0, 41 // 16]), 41 % 16
        cache.k_elems[p, 0, o, 0] = 0x00 if weight > 0 else 0x40
        cache.v_scales[p, 0, o, :2] = far
        _check(q, cache, table, lengths, scale=abs(weight) * math.log(2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("first", [True, False])
def test_a_large_value_that_a_larger_score_makes_small(first, dtype):
    """Tokens of 2^60 times the others' values whose weights are 2^-90 of theirs, in the tiles before or behind them."""
    q, cache, table, lengths = _problem([900], 1, 1, 128, 16, mx.MX_E4M3, dtype, 35)
    q.zero_()
    q[..., 0] = 1.0
    cache.k_elems.zero_()
    cache.k_scales.fill_(127)
    for j in range(900):
        large = (j < 450) == first
        cache.k_elems[int(table[0, j // 16]), 0, j % 16, 0] = 0x00 if large else 0x38  # 0 or 1.0
        cache.v_scales[int(table[0, j // 16]), 0, j % 16] = 160 if large else 100
    for scale in (90 * math.log(2), 20 * math.log(2), 60 * math.log(2)):
        _check(q, cache, table, lengths, scale=scale)
        _check(*_wide((q, cache, table, lengths), 9000), scale=scale)


def _scale_just_above(n, value):
    """A scale whose product with log2 e in FP32, times `value`, is above the integer n by less than half a step of FP32 (so that it
    rounds to n)."""
    log2e = np.float32(1.4426950408889634)
    s = np.float32(n / value / float(log2e))
    for _ in range(50):
        s = np.nextafter(s, np.float32(0))
    for _ in range(100):
        f = s * log2e
        if float(f) * value > n and np.float32(f * np.float32(value)) == n:
            return float(s)
        s = np.nextafter(s, np.float32(np.inf))
    return None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scores_that_round_to_the_reference(dtype):
    """The reference of the running maximum is an integer (in powers of two).  Scores that exceed it by less than half a step
    pass it or do not, but the kernel may not be of two minds about it."""
    found = 0
    for n in (8, 7, 9, 10):
        # the first tiles' scores lie in (n - 3, n - 2], which puts the reference at n
        for value, code, first in ((1.5, 0x3C, 0x38), (1.75, 0x3E, 0x3A), (1.25, 0x3A, 0x34), (1.375, 0x3B, 0x38)):
            scale = _scale_just_above(n, value)
            v0 = {0x38: 1.0, 0x3A: 1.25, 0x34: 0.75}[first]
            if scale is None or not n - 3 < n / value * v0 <= n - 2:
                continue
            found += 1
            q, cache, table, lengths = _problem([700], 1, 1, 64, 16, mx.MX_E4M3, dtype, 33)
            q.zero_()
            q[..., 0] = 1.0
            cache.k_elems.zero_()
            cache.k_scales.fill_(127)
            for j in range(700):
                cache.k_elems[int(table[0, j // 16]), 0, j % 16, 0] = first if j < 256 else code
            _check(q, cache, table, lengths, scale=scale)
            _check(*_wide((q, cache, table, lengths), 9000), scale=scale)
    assert found


def test_very_large_scores():
    """Scores of 2^30 and more, whose steps are larger than one."""
    for qs in (1e8, 1e12, 1e20):
        q, cache, table, lengths = _problem([300, 20], 2, 4, 64, 16, mx.MX_E4M3, torch.float32, 34)
        out, lse = mx.mx_kv_attention(q * qs, cache, table, lengths, return_lse=True)
        want, wlse, _, size, _ = attention64(q * qs, cache, table, lengths, 0.125, 0)
        assert bool(torch.isfinite(out).all()) and bool(((lse.double() - wlse).abs() <= (64 + 16) * 2.0 ** -23 * size + 2.0 ** -20).all())
        # the scores lie so far apart that the largest takes all: its value, with a weight of 1 within the divisions' 2^-20
        assert float((out.double() - want).abs().max()) <= 2.0 ** -20 * float(want.abs().max())


def test_one_large_score():
    for at in (0, 31, 32, 700, 998):
        q, cache, table, lengths = _problem([999], 1, 4, 128, 16, mx.MX_E4M3, torch.bfloat16, 40 + at)
        p, o = int(table[0, at // 16]), at % 16
        cache.k_scales[p, 0, o, :] = 127
        cache.v_scales[p, 0, o, :] = 133
        _check(q, cache, table, lengths)


def test_strides_scale_and_outputs():
    q, cache, table, lengths = _problem([90, 12, 300], 2, 4, 64, 16, mx.MX_E4M3, torch.bfloat16, 50, new=2)
    wide = torch.zeros(3, 2, 3, 8, 64, device="cuda", dtype=torch.bfloat16)
    wide[:, :, 1] = q
    base = mx.mx_kv_attention(q, cache, table, lengths, 0.3)
    assert torch.equal(mx.mx_kv_attention(wide[:, :, 1], cache, table, lengths, 0.3), base)
    out = torch.full_like(q, 7)
    assert mx.mx_kv_attention(q, cache, table, lengths, 0.3, out=out) is out and torch.equal(out, base)
    _check(q, cache, table, lengths, scale=-0.2)
    _check(q, cache, table, lengths, scale=0.0)
    # three dimensions: one new token
    one = mx.mx_kv_attention(q[:, 1].contiguous(), cache, table, lengths)
    assert one.shape == (3, 8, 64) and torch.equal(one, mx.mx_kv_attention(q[:, 1:2].contiguous(), cache, table, lengths)[:, 0])
    assert torch.equal(one, mx.mx_kv_attention(q[:, 1], cache, table, lengths))
    none = mx.mx_kv_attention(q[:0], cache, table[:0], lengths[:0])
    assert none.shape == (0, 2, 8, 64)


def test_same_call_same_bits():
    q, cache, table, lengths = _problem([9000, 100, 4000], 2, 8, 128, 64, mx.MX_E4M3, torch.bfloat16, 60)
    first = mx.mx_kv_attention(q, cache, table, lengths, return_lse=True)
    for _ in range(3):
        again = mx.mx_kv_attention(q, cache, table, lengths, return_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_streams_and_graphs():
    """Two streams at once; a captured decoding step, replayed as the sequences grow."""
    probs = [_problem([3000, 50], 2, 4, 128, 16, mx.MX_E4M3, torch.bfloat16, 70 + i) for i in range(2)]
    want = [mx.mx_kv_attention(*p) for p in probs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in probs]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(mx.mx_kv_attention(*probs[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])

    q, cache, table, lengths = _problem([400, 90], 2, 4, 128, 16, mx.MX_E4M3, torch.bfloat16, 80)
    cap = table.shape[1] * 16
    lengths.copy_(torch.tensor([20, 3], dtype=torch.int32))
    k, v = (torch.zeros(2, 2, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    row = torch.arange(2, device="cuda")

    def step():
        lengths.add_(1)
        at = lengths.long() - 1
        slots = (table[row, at // 16].long() * 16 + at % 16).to(torch.int32)
        mx.mx_kv_append(cache, k, v, slots)
        return mx.mx_kv_attention(q, cache, table, lengths)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    g = _gen(81)
    for _ in range(40):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert int(lengths.max()) < cap
        assert torch.equal(out, mx.mx_kv_attention(q, cache, table, lengths))
    _check(q, cache, table, lengths, got=mx.mx_kv_attention(q, cache, table, lengths, return_lse=True))


def test_a_sequence_is_written_read_and_attended_as_a_whole():
    """Prompt and new tokens through the cache: what is read back gives the same attention in PyTorch."""
    g = _gen(90)
    heads, group, dim, ps = 2, 4, 64, 16
    for fmt in FMTS:
        cache = mx.mx_kv_cache(12, ps, heads, dim, fmt)
        table = torch.randperm(12, generator=g, device="cuda").to(torch.int32).view(2, 6)
        slots = (table.long()[:, :, None] * ps + torch.arange(ps, device="cuda")).view(2, -1).to(torch.int32)
        lens = [0, 0]
        for n0, n1 in ((40, 17), (1, 1), (1, 1), (3, 30)):
            for b, n in enumerate((n0, n1)):
                k, v = (torch.randn(n, heads, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
                mx.mx_kv_append(cache, k, v, slots[b, lens[b]:lens[b] + n].contiguous())
                lens[b] += n
            q = torch.randn(2, heads * group, dim, generator=g, device="cuda")
            out = mx.mx_kv_attention(q, cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
            for b in range(2):
                k, v = mx.mx_kv_read(cache, slots[b, :lens[b]].contiguous())
                s = torch.einsum("hgd,nhd->hgn", q[b].double().view(heads, group, dim), k.double()) * dim ** -0.5
                want = torch.einsum("hgn,nhd->hgd", torch.softmax(s, 2), v.double()).view(heads * group, dim)
                # scores below 20 and sums of 64 products: weights within 2^-13, values below 8
                assert float((out[b].double() - want).abs().max()) < 8 * 2.0 ** -13


def test_python_refusals():
    q, cache, table, lengths = _problem([50, 20], 2, 4, 64, 16, mx.MX_E4M3, torch.bfloat16, 95)
    ok = dict(q=q, cache=cache, table=table, lengths=lengths)
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    for bad in (dict(q=q.double()), dict(q=q[..., :32]), dict(q=q[:, :, :3].contiguous()), dict(q=q[0, 0]), dict(q=q.cpu()), dict(table=table.long()), dict(table=table[:1]),
                dict(table=table[0]), dict(lengths=lengths.long()), dict(lengths=lengths[:1]), dict(out=q[:1]), dict(out=q.float()), dict(window=-1),
                dict(scale=math.inf), dict(scale=math.nan), dict(workspace=small), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), dict(q=q[:, :0])):
        with pytest.raises((ValueError, TypeError, mx.MxError)):
            mx.mx_kv_attention(**(ok | bad))
    wide = mx.mx_kv_cache(4, 16, 2, 32, mx.MX_E4M3)
    with pytest.raises(mx.MxError):
        mx.mx_kv_attention(q[..., :32].contiguous(), wide, table, lengths)
