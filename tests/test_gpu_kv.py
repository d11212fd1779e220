"""The paged key-value cache: rows quantized into their slots are those of the oracle, byte for byte, nothing else
changes; what is read back are the values of codes and scales."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2310_10537_b200 as mx
from gpu_util import to_oracle_input
from kv_util import random_cache, values

pytestmark = pytest.mark.gpu
FMTS = [mx.MX_E4M3, mx.MX_E5M2, mx.MX_E2M1, mx.MX_INT8]
SHAPES = [(1, 1, 32, 1), (7, 3, 64, 16), (64, 8, 128, 64), (33, 5, 96, 24), (100, 2, 256, 7), (257, 1, 192, 128), (40, 4, 160, 1), (3, 2, 1056, 5)]


def _slots(tokens, page_size, g, holes):
    pages = -(-tokens // page_size) + 2
    slots = torch.randperm(pages * page_size, generator=g, device="cuda")[:tokens].to(torch.int32)
    if holes and tokens > 2:
        slots[1] = -1
        slots[tokens // 2] = pages * page_size
        slots[tokens - 1] = -(1 << 31)
    return pages, slots


def _rows(shape, dtype, g, extremes):
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp(3 * torch.randn(shape[:2] + (1,), generator=g, device="cuda"))
    if extremes:
        f = x.view(-1)
        n = len(f)
        for i, v in enumerate((0.0, -0.0, float("nan"), float("inf"), -float("inf"), 1e-42, 2.0 ** -126, 3.3e38, -3.3e38, 2.0 ** -120)):
            f[(i * 37 + 5) % n] = v
        x[0, 0] = 0
    return x.to(dtype)


@pytest.mark.parametrize("rounding", [mx.MX_RNE, mx.MX_RHAZ])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", FMTS)
def test_append_writes_the_oracles_bytes(fmt, dtype, rounding):
    for at, (tokens, heads, dim, ps) in enumerate(SHAPES):
        g = torch.Generator(device="cuda").manual_seed(fmt * 100 + at)
        pages, slots = _slots(tokens, ps, g, at % 2 == 1)
        cache = random_cache(pages, ps, heads, dim, fmt, g)
        k, v = (_rows((tokens, heads, dim), dtype, g, at > 0) for _ in range(2))
        before = [t.cpu().clone() for t in cache[:4]]
        mx.mx_kv_append(cache, k, v, slots, rounding)
        ok = ((slots >= 0) & (slots < pages * ps)).cpu().numpy()
        page, off = slots.cpu().numpy()[ok] // ps, slots.cpu().numpy()[ok] % ps
        for x, codes, scales, c0, s0 in ((k, cache.k_elems, cache.k_scales, before[0], before[1]), (v, cache.v_elems, cache.v_scales, before[2], before[3])):
            e, s = O.quantize(to_oracle_input(x.reshape(tokens * heads, dim)), 1, fmt, rounding, O.LINEAR)
            want_c, want_s = c0.numpy().copy(), s0.numpy().copy()
            want_c[page, :, off] = e.reshape(tokens, heads, -1)[ok]
            rows = np.zeros((tokens, heads, want_s.shape[3]), np.uint8)
            rows[:, :, :dim // 32] = s.reshape(tokens, heads, -1)
            want_s[page, :, off] = rows[ok]
            assert np.array_equal(codes.cpu().numpy(), want_c), (tokens, heads, dim, ps)
            assert np.array_equal(scales.cpu().numpy(), want_s), (tokens, heads, dim, ps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", FMTS)
def test_read_gives_the_values(fmt, dtype):
    for at, (tokens, heads, dim, ps) in enumerate(SHAPES):
        g = torch.Generator(device="cuda").manual_seed(fmt * 100 + at + 7)
        pages, slots = _slots(tokens, ps, g, at % 2 == 1)
        cache = random_cache(pages, ps, heads, dim, fmt, g, spread=100, middle=120)
        cache.k_scales.view(-1)[5 % cache.k_scales.numel()] = 255
        cache.k_scales.view(-1)[0] = 0
        if fmt in (mx.MX_E4M3, mx.MX_E5M2):
            cache.v_elems.view(-1)[3] = 0x7F
            cache.v_elems.view(-1)[-1] = 0xFC
        if tokens > 2:
            slots[0] = slots[2]  # the same slot twice is fine here
        k, v = mx.mx_kv_read(cache, slots, dtype)
        # results that begin in the middle of a 32-byte sector
        odd = [torch.empty(k.numel() + 16 // k.element_size(), dtype=dtype, device="cuda")[16 // k.element_size():].view(k.shape) for _ in range(2)]
        assert mx.mx_kv_read(cache, slots, dtype, out=tuple(odd)) is not None
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(odd, (k, v)))
        assert k.shape == v.shape == (tokens, heads, dim) and k.dtype == v.dtype == dtype
        ok = (slots >= 0) & (slots < pages * ps)
        page, off = slots[ok].long() // ps, slots[ok].long() % ps
        for got, codes, scales in ((k, cache.k_elems, cache.k_scales), (v, cache.v_elems, cache.v_scales)):
            want = torch.zeros((tokens, heads, dim), dtype=torch.float64, device="cuda")
            want[ok] = values(codes[page, :, off], scales[page, :, off], dim, fmt)
            # exact in FP32 (overflow to Inf), BF16 one rounding
            assert torch.equal(torch.nan_to_num(got.double(), nan=1.5e300), torch.nan_to_num(want.float().to(dtype).double(), nan=1.5e300))


def test_a_projections_output_is_read_in_place():
    g = torch.Generator(device="cuda").manual_seed(1)
    for dtype in (torch.bfloat16, torch.float32):
        tokens, heads, dim, ps = 37, 4, 64, 16
        qkv = torch.randn(tokens, 6 * heads * dim, generator=g, device="cuda").to(dtype)
        k, v = qkv[:, 4 * heads * dim:5 * heads * dim].view(tokens, heads, dim), qkv[:, 5 * heads * dim:].view(tokens, heads, dim)
        pages, slots = _slots(tokens, ps, g, False)
        a, b = (mx.mx_kv_cache(pages, ps, heads, dim, mx.MX_E4M3) for _ in range(2))
        mx.mx_kv_append(a, k, v, slots)
        mx.mx_kv_append(b, k.contiguous(), v.contiguous(), slots)
        assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))
        # rows of another spacing for keys and values, a single token of any stride
        wide = torch.randn(tokens, heads * dim + 64, generator=g, device="cuda").to(dtype)[:, :heads * dim].view(tokens, heads, dim)
        mx.mx_kv_append(a, k, wide, slots)
        mx.mx_kv_append(b, k, wide.contiguous(), slots)
        assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))
        mx.mx_kv_append(a, k[3:4], v[3:4], slots[3:4])
        mx.mx_kv_append(b, k[3:4].contiguous(), v[3:4].contiguous(), slots[3:4])
        assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))


def test_no_tokens_and_no_pages():
    cache = mx.mx_kv_cache(2, 16, 2, 64, mx.MX_E4M3)
    none = torch.empty((0, 2, 64), device="cuda")
    slots = torch.empty(0, dtype=torch.int32, device="cuda")
    mx.mx_kv_append(cache, none, none, slots)
    k, v = mx.mx_kv_read(cache, slots)
    assert k.shape == (0, 2, 64)
    empty = mx.mx_kv_cache(0, 16, 2, 64, mx.MX_E4M3)
    x = torch.ones((3, 2, 64), device="cuda")
    mx.mx_kv_append(empty, x, x, torch.arange(3, dtype=torch.int32, device="cuda"))
    k, v = mx.mx_kv_read(empty, torch.arange(3, dtype=torch.int32, device="cuda"), torch.bfloat16)
    assert not k.any() and not v.any()


def test_python_refusals():
    cache = mx.mx_kv_cache(2, 16, 2, 64, mx.MX_E4M3)
    x, slots = torch.ones((3, 2, 64), device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        mx.mx_kv_cache(2, 16, 2, 64, mx.MX_E3M2)
    for bad in (dict(k=x[:, :1]), dict(k=x.double()), dict(v=x.bfloat16()), dict(v=x[:2]), dict(slots=slots.long()), dict(slots=slots[:2]), dict(k=x.cpu()),
                dict(k=x.transpose(0, 1).contiguous().transpose(0, 1)), dict(cache=cache._replace(dim=96)), dict(cache=cache._replace(k_scales=cache.k_elems)),
                dict(rounding=2), dict(cache=cache._replace(fmt=9)), dict(cache=cache._replace(k_elems=cache.k_elems[:, :, ::2])), dict(cache=tuple(cache[:5]))):
        args = dict(cache=cache, k=x, v=x, slots=slots) | bad
        with pytest.raises((ValueError, TypeError, mx.MxError)):
            mx.mx_kv_append(**args)
    for bad in (dict(dtype=torch.float16), dict(slots=slots.long()), dict(slots=slots.view(1, 3)), dict(out=(x, x[:2]))):
        with pytest.raises((ValueError, TypeError, mx.MxError)):
            mx.mx_kv_read(**(dict(cache=cache, slots=slots) | bad))


def test_offsets_beyond_32_bits():
    """A cache of 5 GB of keys and as many of values: its last pages written, read and attended over like those of a small one."""
    heads, dim, ps, pages, tokens = 8, 128, 64, 80000, 150
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(tokens, heads, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(1, 2 * heads, dim, generator=g, device="cuda").bfloat16()
    length = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    small, large = mx.mx_kv_cache(3, ps, heads, dim, mx.MX_E4M3), mx.mx_kv_cache(pages, ps, heads, dim, mx.MX_E4M3)
    assert large.k_elems.numel() > 1 << 32
    got = []
    for cache, table in ((small, [0, 1, 2]), (large, [pages - 1, pages // 2, pages - 3])):
        table = torch.tensor([table], dtype=torch.int32, device="cuda")
        slots = (table[0, :, None] * ps + torch.arange(ps, dtype=torch.int32, device="cuda")).view(-1)[:tokens].contiguous()
        mx.mx_kv_append(cache, k, v, slots)
        got.append((*mx.mx_kv_read(cache, slots), mx.mx_kv_attention(q, cache, table, length)))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert not large.k_elems[:pages // 2].any() and not large.v_scales[pages // 2 + 1:pages - 3].any()
