"""A query's result does not depend on which other queries share its pass over the cache: heads of its group, drafts."""
import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_kv_attention import _gen, _problem, _wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", [mx.MX_E4M3, mx.MX_E2M1, mx.MX_INT8])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_the_other_heads_of_a_group(dim, fmt, dtype):
    """Values whose scales wander by many powers of two along the sequence, and neighbours of all sharpnesses, so that references and
    scaling powers move often: a head keeps its bits."""
    for seed in range(6):
        problem = _problem([900, 333, 20], 2, 8, dim, 16, fmt, dtype, 300 + seed, spread=8)
        if seed % 2:
            problem = _wide(problem, 9000)
        q, cache, table, lengths = problem
        g = _gen(310 + seed)
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
