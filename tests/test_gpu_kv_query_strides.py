"""Queries of one new token that lie inside a wider tensor: evenly spaced, whatever the second stride says."""
import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_kv_attention import _problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_new_token_inside_a_wider_tensor(dtype):
    heads, group, dim = 2, 4, 64
    q, cache, table, lengths = _problem([90, 12, 300], heads, group, dim, 16, mx.MX_E4M3, dtype, 50, new=3)
    width = heads * group * dim
    for i in range(3):  # one of several drafts
        part = q[:, i:i + 1]
        assert torch.equal(mx.mx_kv_attention(part, cache, table, lengths), mx.mx_kv_attention(part.contiguous(), cache, table, lengths))
    # a fused projection's output [batch, (query heads + 2 heads) * dim]
    qkv = torch.randn(3, width + 2 * heads * dim, device="cuda").to(dtype)
    want = mx.mx_kv_attention(qkv[:, :width].reshape(3, 1, heads * group, dim).contiguous(), cache, table, lengths)
    for part in (qkv[:, :width].view(3, 1, heads * group, dim), qkv[:, :width].view(3, heads * group, dim).unsqueeze(1)):
        assert torch.equal(mx.mx_kv_attention(part, cache, table, lengths), want)
    one = qkv[1:2, :width].view(1, 1, heads * group, dim)  # a single sequence of a single token
    assert torch.equal(mx.mx_kv_attention(one, cache, table[1:2], lengths[1:2]), want[1:2])


def test_uneven_spacing_is_refused():
    q, cache, table, lengths = _problem([90, 12, 300], 2, 4, 64, 16, mx.MX_E4M3, torch.bfloat16, 50, new=3)
    for bad in (q[:, :2], q[:, ::2], q[:, :1].expand(3, 2, 8, 64), q.transpose(0, 1)):
        with pytest.raises((ValueError, mx.MxError)):
            mx.mx_kv_attention(bad, cache, table[:bad.shape[0]], lengths[:bad.shape[0]])


def test_results_in_place_of_the_queries_are_refused():
    """Blocks read queries while others write results: `out` may not share memory with `q`."""
    q, cache, table, lengths = _problem([90, 12], 2, 4, 64, 16, mx.MX_E4M3, torch.bfloat16, 51)
    flat = torch.zeros(2 * q.numel(), dtype=q.dtype, device="cuda")
    first, second, across = (flat[i:i + q.numel()].view(q.shape) for i in (0, q.numel(), q.numel() // 2))
    first.copy_(q)
    for out in (first, across):
        with pytest.raises(ValueError):
            mx.mx_kv_attention(first, cache, table, lengths, out=out)
    assert torch.equal(mx.mx_kv_attention(first, cache, table, lengths, out=second), mx.mx_kv_attention(q, cache, table, lengths))
    # a result that lies between two tokens' queries, and one that is in the way
    wide = torch.zeros(1, 1536, dtype=q.dtype, device="cuda")
    one = wide[:, 512:1024].view(1, 1, 8, 64)
    one.copy_(q[:1])
    want = mx.mx_kv_attention(q[:1], cache, table[:1], lengths[:1])
    for at in (0, 1024):
        assert torch.equal(mx.mx_kv_attention(one, cache, table[:1], lengths[:1], out=wide[:, at:at + 512].view(1, 1, 8, 64)), want)
    with pytest.raises(ValueError):
        mx.mx_kv_attention(one, cache, table[:1], lengths[:1], out=wide[:, 520:1032].view(1, 1, 8, 64))
