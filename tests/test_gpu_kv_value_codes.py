"""NaN and Inf among the element codes of a cached value: they reach the queries that see the token, and no other."""
import math

import pytest
import torch

import paper_2310_10537_b200 as mx
from kv_util import attention64
from test_gpu_kv_attention import _problem, _wide

pytestmark = pytest.mark.gpu
CODES = [(mx.MX_E4M3, (0x7F, 0xFF)), (mx.MX_E5M2, (0x7C, 0x7C)), (mx.MX_E5M2, (0xFC, 0x7D)), (mx.MX_E5M2, (0x7C, 0xFC))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt,codes", CODES)
@pytest.mark.parametrize("dim,window", [(64, 0), (64, 70), (96, 33), (128, 0), (128, 40), (192, 17), (256, 130)])
def test_codes_of_a_token_that_some_drafts_see(dim, window, fmt, codes, dtype):
    """The newest token, which the last draft sees alone, and the oldest one of the first draft's window, which no later draft
    sees.  What does not see them keeps its bits; what does is NaN or Inf where the definition is."""
    lengths, heads, group, ps, new = [1, 2, 3, 4, 40, 150, 257, 600], 2, 3, 16, 4
    for wide in (False, True):
        q, cache, table, lens = _problem(lengths, heads, group, dim, ps, fmt, dtype, 200 + dim + window, new)
        if wide:
            q, cache, table, lens = _wide((q, cache, table, lens), 10000)
        plain, plain_lse = mx.mx_kv_attention(q, cache, table, lens, window=window, return_lse=True)
        for b, n in enumerate(lengths):
            tokens = [(n - 1, codes[0]), (n - 2, codes[1])]
            if window:
                oldest = n - (new - 1) - window
                tokens += [(oldest, codes[1]), (oldest + 1, codes[0])]
            for at, (j, code) in enumerate(tokens):
                if j < 0:
                    continue
                page, off = int(table[b, j // ps]), j % ps
                for e in (0, 5, 13 * (at + 1), dim - 1 - at):
                    cache.v_elems[page, at % heads, off, e] = code
        out, lse = mx.mx_kv_attention(q, cache, table, lens, window=window, return_lse=True)
        want = attention64(q, cache, table, lens, dim ** -0.5, window)[0]
        assert torch.equal(lse, plain_lse)
        odd = ~torch.isfinite(want)
        assert bool(odd.any()) and not bool(odd[:, 0].all())
        assert torch.equal(out[~odd], torch.where(odd, torch.zeros_like(plain), plain)[~odd])
        assert torch.equal(torch.nan_to_num(out[odd].double(), nan=7.0), torch.nan_to_num(want[odd], nan=7.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_query_without_tokens_beside_a_nan_code(dtype):
    """A sequence shorter than its drafts: the first ones see nothing and give zeros, whatever the tokens hold."""
    q, cache, table, lens = _problem([2, 1], 1, 2, 128, 16, mx.MX_E4M3, dtype, 210, 4)
    cache.v_elems[table[0, 0], :, :2] = 0x7F
    cache.v_elems[table[1, 0], :, 0] = 0xFF
    out, lse = mx.mx_kv_attention(q, cache, table, lens, return_lse=True)
    assert not out[0, :2].any() and not out[1, :3].any() and bool((lse[0, :2] == -math.inf).all()) and bool((lse[1, :3] == -math.inf).all())
    assert out[0, 2:].isnan().all() and out[1, 3].isnan().all() and torch.isfinite(lse[0, 2:]).all()
