"""Weight gradients whose rows end inside a chunk of 128: an offset of `rows` or more is the end of the tensor, every other
one is rounded down to a multiple of 128.  Bound as for the other products."""
import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_moe import _check_product, _values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,raw,used", [
    (160, [0, 128, 160], [0, 128, 160]),
    (160, [0, 128, 256], [0, 128, 160]),
    (160, [0, 160, 160], [0, 160, 160]),
    (160, [0, 159, 160], [0, 128, 160]),
    (160, [160, 1 << 30, 161], [160, 160, 160]),
    (32, [0, 32], [0, 32]),
    (96, [0, 95, 96, 96], [0, 0, 96, 96]),
    (1824, [0, 1024, 1792, 1824], [0, 1024, 1792, 1824]),
    (256, [0, 128, 256], [0, 128, 256]),
])
def test_groups_that_reach_the_end_of_the_rows(rows, raw, used, out_dtype):
    M, N, G = 200, 264, len(raw) - 1
    g = torch.Generator(device="cuda").manual_seed(rows)
    ea, sa = mx.mx_quantize(torch.randn(M, rows, generator=g, device="cuda"), 1, mx.MX_E5M2)
    eb, sb = mx.mx_quantize(torch.randn(N, rows, generator=g, device="cuda"), 1, mx.MX_E4M3)
    c = torch.full((G, M, N), 77.0, dtype=out_dtype, device="cuda")
    off = torch.tensor(raw, dtype=torch.int32, device="cuda")
    mx.mx_gemm_grouped_k(ea, sa, eb, sb, off, M, N, rows, mx.MX_E5M2, mx.MX_E4M3, out=c, check_status=True)
    a64, b64 = _values(ea, sa, M, rows, mx.MX_E5M2), _values(eb, sb, N, rows, mx.MX_E4M3)
    for i in range(G):
        _check_product(c[i], a64[:, used[i]:used[i + 1]], b64[:, used[i]:used[i + 1]])
