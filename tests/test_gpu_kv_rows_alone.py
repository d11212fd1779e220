"""A query's result does not depend on which other queries share its pass over the cache: heads of its group, drafts."""
import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_kv_attention import _gen, _problem, _wide

pytestmark = pytest.mark.gpu


def _growing(cache, table, lengths, rate, g, dtype):
    """Value scales that grow by a power of two every `rate` tokens of a sequence, and wander by 2 around that: every row's scaling powers move all
    along, each at tokens of its own.  Every other token is small (2^-28, for FP32 results 2^-20 of the others): its weight, or that one's second term,
    lies among FP16's smallest numbers, whose rounding goes with the scaling power.  In the upper half of a block only the small ones
    are not zero, so that this rounding shows."""
    ps = cache.k_elems.shape[2]
    width = cache.v_elems.shape[3] * 32 // cache.dim  # bytes of a block
    for b, n in enumerate(lengths.tolist()):
        j = torch.arange(n, device="cuda")
        page, o, small = table[b, j // ps].long(), j % ps, j % 2 == 0
        s = 90 + (j // rate)[:, None, None] + torch.randint(-2, 3, (n, cache.k_elems.shape[1], cache.dim // 32), generator=g, device="cuda")
        s -= small[:, None, None] * (28 if dtype == torch.bfloat16 else 20)
        cache.v_scales[page, :, o, :cache.dim // 32] = s.to(torch.uint8)
        codes = cache.v_elems[page, :, o]
        upper = torch.arange(codes.shape[2], device="cuda") % width >= width // 2
        cache.v_elems[page, :, o] = torch.where(~small[:, None, None] & upper, torch.zeros_like(codes), codes)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", [mx.MX_E4M3, mx.MX_E2M1, mx.MX_INT8])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_the_other_heads_of_a_group(dim, fmt, dtype):
    """Neighbours of all sharpnesses, so that references and scaling powers move often: a head keeps its bits."""
    for seed in range(6):
        q, cache, table, lengths = _problem([1000, 333, 20], 2, 8, dim, 16, fmt, dtype, 300 + seed)
        g = _gen(310 + seed)
        _growing(cache, table, lengths, 60 + 50 * (seed // 2), g, dtype)
        if seed % 2:
            q, cache, table, lengths = _wide((q, cache, table, lengths), 9000)
        keep = 3
        want = None
        for i in range(5):
            other = torch.randn(q.shape, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 5, q.shape[:-1] + (1,), generator=g, device="cuda").float())
            if i:
                q = torch.where((torch.arange(q.shape[2], device="cuda") % 8 == keep)[:, None], q, other.to(dtype))
            out, lse = mx.mx_kv_attention(q, cache, table, lengths, return_lse=True)
            got = (out[:, :, keep::8].clone(), lse[:, :, keep::8].clone())
            if want is None:
                want = got
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (seed, i)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_head_alone(dtype):
    """The same head with and without others beside it."""
    for seed in range(4):
        q, cache, table, lengths = _problem([1000, 50], 1, 5, 128, 16, mx.MX_E4M3, dtype, 320 + seed)
        _growing(cache, table, lengths, 70, _gen(330 + seed), dtype)
        out = mx.mx_kv_attention(q, cache, table, lengths)
        for h in range(5):
            assert torch.equal(mx.mx_kv_attention(q[:, :, h:h + 1].contiguous(), cache, table, lengths), out[:, :, h:h + 1]), (seed, h)
