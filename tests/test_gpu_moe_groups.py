"""Weight gradients over many groups of unequal length, as many of them empty as not: the groups are worked on in
another order than they lie in.  Bound as for the other products."""
import numpy as np
import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_moe import _check_product, _offsets, _values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,M,N", [(5, 300, 520), (37, 64, 264), (128, 40, 128), (129, 40, 128), (400, 33, 8)])
def test_groups_of_unequal_length(G, M, N):
    rng = np.random.default_rng(G)
    lens = rng.integers(0, 5, G) * 128
    lens[rng.random(G) < 0.4] = 0
    lens[1] = 128
    off, rows = _offsets(lens), int(lens.sum())
    ea, sa = mx.mx_quantize(torch.randn(M, rows, device="cuda"), 1, mx.MX_E5M2)
    eb, sb = mx.mx_quantize(torch.randn(N, rows, device="cuda"), 1, mx.MX_E4M3)
    c = torch.full((G, M, N), 77.0, device="cuda")
    mx.mx_gemm_grouped_k(ea, sa, eb, sb, torch.from_numpy(off).cuda(), M, N, rows, mx.MX_E5M2, mx.MX_E4M3, out=c, check_status=True)
    a64, b64 = _values(ea, sa, M, rows, mx.MX_E5M2), _values(eb, sb, N, rows, mx.MX_E4M3)
    for g in range(G):
        if lens[g]:
            _check_product(c[g], a64[:, off[g]:off[g + 1]], b64[:, off[g]:off[g + 1]])
        else:
            assert not bool(c[g].any())
