"""Which call learns of a grouped product's expired wait: the next checked one on the same stream, and no other."""
import ctypes

import pytest
import torch

import paper_2310_10537_b200 as mx
from test_gpu_moe import _offsets
from test_gpu_moe_drill import BUDGET, _operands

pytestmark = pytest.mark.gpu


def test_a_failure_is_reported_on_its_own_stream():
    lens, N, K = [64, 128], 256, 512
    rows = sum(lens)
    ops = _operands(rows, K, 2 * N, mx.MX_E4M3, mx.MX_E4M3)
    args = (*ops, torch.from_numpy(_offsets(lens)).cuda(), rows, N, K, mx.MX_E4M3, mx.MX_E4M3)
    want = mx.mx_gemm_grouped(*args, check_status=True)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        mx.mx_gemm_grouped_ex(*args, wait_cycles=BUDGET, drop_fill=1)  # not checked
    side.synchronize()
    with torch.cuda.stream(other):
        assert torch.equal(mx.mx_gemm_grouped(*args, check_status=True), want)
    assert torch.equal(mx.mx_gemm_grouped(*args, check_status=True), want)
    with torch.cuda.stream(side):
        with pytest.raises(mx.MxError) as e:
            mx.mx_gemm_grouped(*args, check_status=True)
        assert e.value.status == mx.MX_ERR_TIMEOUT
        assert torch.equal(mx.mx_gemm_grouped(*args, check_status=True), want)  # reported once


def test_more_streams_than_status_words_are_served():
    ops = _operands(64, 128, 128, mx.MX_E4M3, mx.MX_E4M3)
    args = (*ops, torch.from_numpy(_offsets([64])).cuda(), 64, 128, 128, mx.MX_E4M3, mx.MX_E4M3)
    want = mx.mx_gemm_grouped(*args, check_status=True)
    rt, handles = torch.cuda.cudart(), []
    torch.cuda.synchronize()
    try:
        for _ in range(300):
            h = ctypes.c_void_p()
            assert int(rt.cudaStreamCreate(ctypes.addressof(h))) == 0
            handles.append(h.value)
        for i, h in enumerate(handles):
            with torch.cuda.stream(torch.cuda.ExternalStream(h)):
                c = mx.mx_gemm_grouped(*args, out=torch.empty_like(want), check_status=i % 10 == 0)
            torch.cuda.synchronize()
            assert torch.equal(c, want)
    finally:
        for h in handles:
            rt.cudaStreamDestroy(h)
