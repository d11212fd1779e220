"""Failure detection of the grouped products without a GPU fault: the operand copies leave out one fill of a stage
(nothing is copied for it, so nothing is in flight later) and every wait gets a budget of about a
millisecond.  The wait runs out, the kernel leaves through its common exit, the checked call returns
MX_ERR_TIMEOUT and the next product on the same context is right."""
import pytest
import torch

import paper_2310_10537_b200 as mx
from gpu_util import Guarded
from test_gpu_moe import _check_product, _offsets, _values

pytestmark = pytest.mark.gpu
BUDGET = 2_000_000


def _operands(rows, K, brows, fa, fb):
    g = torch.Generator(device="cuda").manual_seed(rows + K)
    ea, sa = mx.mx_quantize(torch.randn(rows, K, generator=g, device="cuda"), 1, fa)
    eb, sb = mx.mx_quantize(torch.randn(brows, K, generator=g, device="cuda"), 1, fb)
    return ea, sa, eb, sb


def _expect_timeout(run, first_wait):
    with pytest.raises(mx.MxError) as e:
        run()
    assert e.value.status == mx.MX_ERR_TIMEOUT
    # 2: the MMA issuer's wait for a stage; it is the only one with a single budget where all fills fit the stages
    assert "of a grouped product gave up" in str(e.value) and (not first_wait or "wait 2 " in str(e.value)), str(e.value)


@pytest.mark.parametrize("lens,N,K,fb,drop,all_fit", [
    ([64] * 4, 256, 512, mx.MX_E2M1, 1, True),      # tiles of 64 rows, two K chunks a stage
    ([128] * 2, 128, 1024, mx.MX_E4M3, 3, True),    # tiles of 128
    ([512, 256], 384, 512, mx.MX_E4M3, 0, True),    # tiles of 256, the first fill
    ([1024] * 8, 1024, 2048, mx.MX_E4M3, 5, False),  # several items per pair
])
def test_row_groups(lens, N, K, fb, drop, all_fit):
    G, rows, off = len(lens), sum(lens), _offsets(lens)
    ea, sa, eb, sb = _operands(rows, K, G * N, mx.MX_E4M3, fb)
    o = torch.from_numpy(off).cuda()
    args = (ea, sa, eb, sb, o, rows, N, K, mx.MX_E4M3, fb)
    buf = Guarded(rows * N * 4)
    c = buf.view.view(torch.float32).view(rows, N)
    _expect_timeout(lambda: mx.mx_gemm_grouped_ex(*args, out=c, check_status=True, wait_cycles=BUDGET, drop_fill=drop), all_fit)
    buf.check()
    mx.mx_gemm_grouped(*args, out=c, check_status=True)
    buf.check()
    a64, b64 = _values(ea, sa, rows, K, mx.MX_E4M3), _values(eb, sb, G * N, K, fb).view(G, N, K)
    for g in range(G):
        _check_product(c[off[g]:off[g + 1]], a64[off[g]:off[g + 1]], b64[g])
    assert torch.equal(mx.mx_gemm_grouped_ex(*args, check_status=True, wait_cycles=2_000_000_000), c)


@pytest.mark.parametrize("lens,M,N,drop", [([384, 256], 200, 264, 1), ([256, 0, 128], 64, 128, 0)])
def test_k_groups(lens, M, N, drop):
    G, rows, off = len(lens), sum(lens), _offsets(lens)
    ea, sa, eb, sb = _operands(M, rows, N, mx.MX_E5M2, mx.MX_E4M3)
    args = (ea, sa, eb, sb, torch.from_numpy(off).cuda(), M, N, rows, mx.MX_E5M2, mx.MX_E4M3)
    buf = Guarded(G * M * N * 4)
    c = buf.view.view(torch.float32).view(G, M, N)
    _expect_timeout(lambda: mx.mx_gemm_grouped_k_ex(*args, out=c, check_status=True, wait_cycles=BUDGET, drop_fill=drop), True)
    buf.check()
    mx.mx_gemm_grouped_k(*args, out=c, check_status=True)
    buf.check()
    a64, b64 = _values(ea, sa, M, rows, mx.MX_E5M2), _values(eb, sb, N, rows, mx.MX_E4M3)
    for g in range(G):
        _check_product(c[g], a64[:, off[g]:off[g + 1]], b64[:, off[g]:off[g + 1]])


def test_refusals():
    ea, sa, eb, sb = _operands(64, 128, 128, mx.MX_E4M3, mx.MX_E4M3)
    o = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    for kw in ({"wait_cycles": -1}, {"drop_fill": -2}, {"drop_fill": 1 << 40}):
        with pytest.raises(mx.MxError) as e:
            mx.mx_gemm_grouped_ex(ea, sa, eb, sb, o, 64, 128, 128, mx.MX_E4M3, mx.MX_E4M3, **kw)
        assert e.value.status == mx.MX_ERR_SHAPE
        with pytest.raises(mx.MxError) as e:
            mx.mx_gemm_grouped_k_ex(ea, sa, eb, sb, o, 64, 128, 128, mx.MX_E4M3, mx.MX_E4M3, **kw)
        assert e.value.status == mx.MX_ERR_SHAPE
