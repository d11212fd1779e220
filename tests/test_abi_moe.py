"""Refusals of the norm, routing, row-moving and grouped-product entry points: the documented status for
each bad argument, without a GPU (nothing is launched before the checks)."""
import ctypes

import numpy as np

import paper_2310_10537_b200 as mx

lib = mx.lib()
_buf = np.zeros(1 << 16, np.uint8)
P = _buf.ctypes.data + (-_buf.ctypes.data) % 256
O = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, None, 0)
PAD = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, None, 0, 1)
BAD = mx.binding.mx_opts_t(9, mx.MX_SCALES_SWIZZLED, None, 0)
LIN = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_LINEAR, None, 0)
NAN, INF = float("nan"), float("inf")


def _calls(fn, base, table):
    assert len(base) == len(fn.argtypes)
    for changes, want in table:
        args = list(base)
        for i, v in changes.items():
            args[i] = ctypes.byref(v) if isinstance(v, ctypes.Structure) else v
        assert fn(*args) == want, (changes, want)


def test_rmsnorm_quantize():
    # x residual weight wdtype eps rows dim h y elems scales fmt rounding opts
    base = [P, None, P, 0, 1e-6, 4, 64, None, None, P, P, 0, 0, ctypes.byref(O)]
    _calls(lib.mx_rmsnorm_quantize, base, [
        ({0: None}, mx.MX_ERR_NULL), ({2: None}, mx.MX_ERR_NULL), ({9: None}, mx.MX_ERR_NULL), ({10: None}, mx.MX_ERR_NULL),
        ({3: 2}, mx.MX_ERR_FMT), ({11: 6}, mx.MX_ERR_FMT), ({12: 2}, mx.MX_ERR_FMT), ({13: BAD}, mx.MX_ERR_FMT),
        ({13: PAD}, mx.MX_ERR_UNSUPPORTED), ({4: -1.0}, mx.MX_ERR_SHAPE), ({4: NAN}, mx.MX_ERR_SHAPE), ({4: INF}, mx.MX_ERR_SHAPE),
        ({5: -1}, mx.MX_ERR_SHAPE), ({6: 0}, mx.MX_ERR_SHAPE), ({6: -32}, mx.MX_ERR_SHAPE), ({5: 1 << 40, 6: 1 << 40}, mx.MX_ERR_SHAPE),
        ({5: 1 << 31, 6: 1}, mx.MX_ERR_UNSUPPORTED), ({0: P + 4}, mx.MX_ERR_ALIGN), ({1: P + 4}, mx.MX_ERR_ALIGN), ({7: P + 8}, mx.MX_ERR_ALIGN),
        ({8: P + 8}, mx.MX_ERR_ALIGN), ({5: 0, 0: None}, mx.MX_OK)])


def test_rmsnorm_backward():
    need = lib.mx_rmsnorm_backward_workspace_bytes(4, 64)
    assert need >= 64 * 4 and lib.mx_rmsnorm_backward_workspace_bytes(-1, 64) == 0 and lib.mx_rmsnorm_backward_workspace_bytes(4, 0) == 0
    # dy h weight wdtype eps dres rows dim dh dweight opts workspace bytes
    base = [P, P, P, 0, 1e-6, None, 4, 64, P, P, ctypes.byref(O), P, need]
    _calls(lib.mx_rmsnorm_backward, base, [
        ({0: None}, mx.MX_ERR_NULL), ({8: None}, mx.MX_ERR_NULL), ({9: None}, mx.MX_ERR_NULL), ({11: None}, mx.MX_ERR_NULL),
        ({3: 7}, mx.MX_ERR_FMT), ({10: BAD}, mx.MX_ERR_FMT), ({10: PAD}, mx.MX_ERR_UNSUPPORTED), ({4: -1.0}, mx.MX_ERR_SHAPE),
        ({7: 0}, mx.MX_ERR_SHAPE), ({6: -1}, mx.MX_ERR_SHAPE), ({5: P + 2}, mx.MX_ERR_ALIGN), ({11: P + 16}, mx.MX_ERR_ALIGN),
        ({12: need - 1}, mx.MX_ERR_WORKSPACE)])


def test_route():
    def r(**kw):
        d = dict(topk=2, score=0, groups=1, topk_groups=1, group_score=0, renormalize=1, scale=1.0)
        d.update(kw)
        return mx.binding.mx_route_t(*[d[k] for k in ("topk", "score", "groups", "topk_groups", "group_score", "renormalize", "scale")])
    # logits bias tokens experts route ids weights opts
    base = [P, None, 4, 16, ctypes.byref(r()), P, P, ctypes.byref(O)]
    _calls(lib.mx_route, base, [
        ({0: None}, mx.MX_ERR_NULL), ({4: None}, mx.MX_ERR_NULL), ({5: None}, mx.MX_ERR_NULL), ({6: None}, mx.MX_ERR_NULL),
        ({4: r(score=2)}, mx.MX_ERR_FMT), ({4: r(group_score=2)}, mx.MX_ERR_FMT), ({7: BAD}, mx.MX_ERR_FMT), ({7: PAD}, mx.MX_ERR_UNSUPPORTED),
        ({4: r(topk=0)}, mx.MX_ERR_SHAPE), ({4: r(topk=17)}, mx.MX_ERR_SHAPE), ({4: r(groups=3)}, mx.MX_ERR_SHAPE), ({4: r(groups=0)}, mx.MX_ERR_SHAPE),
        ({4: r(groups=4, topk_groups=5)}, mx.MX_ERR_SHAPE), ({4: r(groups=8, topk=3)}, mx.MX_ERR_SHAPE), ({2: -1}, mx.MX_ERR_SHAPE), ({3: 0}, mx.MX_ERR_SHAPE),
        ({3: 1025}, mx.MX_ERR_UNSUPPORTED), ({3: 64, 4: r(topk=33)}, mx.MX_ERR_UNSUPPORTED), ({3: 64, 4: r(groups=64, topk_groups=64)}, mx.MX_ERR_UNSUPPORTED),
        ({2: 1 << 31}, mx.MX_ERR_UNSUPPORTED), ({0: P + 4}, mx.MX_ERR_ALIGN), ({1: P + 2}, mx.MX_ERR_ALIGN), ({5: P + 1}, mx.MX_ERR_ALIGN), ({2: 0, 0: None}, mx.MX_OK)])
    # dweights logits ids tokens experts route dlogits opts
    base = [P, P, P, 4, 16, ctypes.byref(r()), P, ctypes.byref(O)]
    _calls(lib.mx_route_backward, base, [
        ({0: None}, mx.MX_ERR_NULL), ({1: None}, mx.MX_ERR_NULL), ({2: None}, mx.MX_ERR_NULL), ({6: None}, mx.MX_ERR_NULL), ({5: None}, mx.MX_ERR_NULL),
        ({5: r(score=-1)}, mx.MX_ERR_FMT), ({5: r(topk=17)}, mx.MX_ERR_SHAPE), ({4: 2000}, mx.MX_ERR_UNSUPPORTED), ({6: P + 4}, mx.MX_ERR_ALIGN), ({3: 0}, mx.MX_OK)])


def test_moe_rows_and_plan():
    assert lib.mx_moe_rows(16, 8, 64, 64) == (128 + 64 * 63) // 64 * 64 and lib.mx_moe_rows(0, 8, 64, 64) == 0
    assert lib.mx_moe_rows(1, 1, 64, 64) == 64 and lib.mx_moe_rows(100, 1, 1, 1) == 100
    assert lib.mx_moe_rows(1, 0, 4, 64) == 0 and lib.mx_moe_rows(1 << 40, 1 << 40, 4, 64) == 0 and lib.mx_moe_rows(4, 2, 4, 2000) == 0
    need = lib.mx_moe_plan_workspace_bytes(4, 2, 8)
    assert need > 0 and lib.mx_moe_plan_workspace_bytes(4, 2, 1025) == 0
    # ids tokens topk experts align offsets counts row_of src_of opts workspace bytes
    base = [P, 4, 2, 8, 64, P, P, P, P, ctypes.byref(O), P, need]
    _calls(lib.mx_moe_plan, base, [
        ({0: None}, mx.MX_ERR_NULL), ({5: None}, mx.MX_ERR_NULL), ({6: None}, mx.MX_ERR_NULL), ({7: None}, mx.MX_ERR_NULL), ({8: None}, mx.MX_ERR_NULL), ({10: None}, mx.MX_ERR_NULL),
        ({1: -1}, mx.MX_ERR_SHAPE), ({2: 0}, mx.MX_ERR_SHAPE), ({3: 0}, mx.MX_ERR_SHAPE), ({4: 0}, mx.MX_ERR_SHAPE), ({4: 1025}, mx.MX_ERR_SHAPE),
        ({1: 1 << 31}, mx.MX_ERR_SHAPE), ({3: 1025}, mx.MX_ERR_UNSUPPORTED), ({9: BAD}, mx.MX_ERR_FMT), ({0: P + 2}, mx.MX_ERR_ALIGN), ({10: P + 8}, mx.MX_ERR_ALIGN),
        ({11: need - 1}, mx.MX_ERR_WORKSPACE)])


def test_moe_moves():
    # elems scales tokens topk dim fmt offsets counts row_of src_of experts rows elems_out scales_out opts
    base = [P, P, 4, 2, 64, 0, P, P, P, P, 8, 64, P, P, ctypes.byref(O)]
    _calls(lib.mx_moe_gather, base, [
        ({0: None}, mx.MX_ERR_NULL), ({6: None}, mx.MX_ERR_NULL), ({8: None}, mx.MX_ERR_NULL), ({9: None}, mx.MX_ERR_NULL), ({13: None}, mx.MX_ERR_NULL),
        ({5: 6}, mx.MX_ERR_FMT), ({4: 33}, mx.MX_ERR_SHAPE), ({3: 0}, mx.MX_ERR_SHAPE), ({11: -1}, mx.MX_ERR_SHAPE), ({10: 0}, mx.MX_ERR_SHAPE),
        ({10: 1025}, mx.MX_ERR_UNSUPPORTED), ({14: PAD}, mx.MX_ERR_UNSUPPORTED), ({11: 1 << 31}, mx.MX_ERR_UNSUPPORTED),
        ({4: 1 << 30, 11: 1 << 30}, mx.MX_ERR_UNSUPPORTED), ({12: P + 8}, mx.MX_ERR_ALIGN), ({11: 0}, mx.MX_OK)])
    # y weights row_of tokens topk dim rows out opts
    base = [P, None, P, 4, 2, 64, 64, P, ctypes.byref(O)]
    _calls(lib.mx_moe_combine, base, [
        ({0: None}, mx.MX_ERR_NULL), ({2: None}, mx.MX_ERR_NULL), ({7: None}, mx.MX_ERR_NULL), ({3: -1}, mx.MX_ERR_SHAPE), ({5: 0}, mx.MX_ERR_SHAPE),
        ({8: BAD}, mx.MX_ERR_FMT), ({1: P + 2}, mx.MX_ERR_ALIGN), ({7: P + 4}, mx.MX_ERR_ALIGN), ({3: 0}, mx.MX_OK)])
    # dout y weights offsets counts row_of tokens topk dim experts rows dy dweights opts
    base = [P, P, None, P, P, P, 4, 2, 64, 8, 64, P, P, ctypes.byref(O)]
    _calls(lib.mx_moe_combine_backward, base, [
        ({0: None}, mx.MX_ERR_NULL), ({1: None}, mx.MX_ERR_NULL), ({12: None}, mx.MX_ERR_NULL), ({3: None}, mx.MX_ERR_NULL), ({11: None}, mx.MX_ERR_NULL),
        ({9: 0}, mx.MX_ERR_SHAPE), ({9: 1025}, mx.MX_ERR_UNSUPPORTED), ({0: P + 4}, mx.MX_ERR_ALIGN), ({12: P + 2}, mx.MX_ERR_ALIGN)])


def test_grouped_products():
    # A sA B sB offsets C cdtype groups rows N K fmtA fmtB opts
    base = [P, P, P, P, P, P, 0, 4, 256, 128, 64, 0, 0, ctypes.byref(O)]
    _calls(lib.mx_gemm_grouped, base, [
        ({0: None}, mx.MX_ERR_NULL), ({4: None}, mx.MX_ERR_NULL), ({5: None}, mx.MX_ERR_NULL), ({6: 2}, mx.MX_ERR_FMT), ({11: 6}, mx.MX_ERR_FMT),
        ({12: 5}, mx.MX_ERR_UNSUPPORTED), ({13: PAD}, mx.MX_ERR_UNSUPPORTED), ({13: LIN}, mx.MX_ERR_UNSUPPORTED), ({7: 1025}, mx.MX_ERR_UNSUPPORTED),
        ({9: 64}, mx.MX_ERR_SHAPE), ({10: 48}, mx.MX_ERR_SHAPE), ({10: 96, 12: 4}, mx.MX_ERR_SHAPE), ({8: -1}, mx.MX_ERR_SHAPE), ({7: -1}, mx.MX_ERR_SHAPE),
        ({8: 1 << 31}, mx.MX_ERR_SHAPE), ({7: 1024, 9: 1 << 24}, mx.MX_ERR_SHAPE), ({0: P + 16}, mx.MX_ERR_ALIGN), ({4: P + 2}, mx.MX_ERR_ALIGN), ({5: P + 4}, mx.MX_ERR_ALIGN),
        ({7: 0}, mx.MX_OK), ({8: 0}, mx.MX_OK), ({9: 0}, mx.MX_OK)])
    # A sA B sB offsets C cdtype groups M N rows fmtA fmtB opts
    base = [P, P, P, P, P, P, 0, 4, 32, 64, 256, 0, 0, ctypes.byref(O)]
    _calls(lib.mx_gemm_grouped_k, base, [
        ({0: None}, mx.MX_ERR_NULL), ({4: None}, mx.MX_ERR_NULL), ({5: None}, mx.MX_ERR_NULL), ({6: 2}, mx.MX_ERR_FMT), ({11: 5}, mx.MX_ERR_UNSUPPORTED),
        ({13: LIN}, mx.MX_ERR_UNSUPPORTED), ({9: 12}, mx.MX_ERR_SHAPE), ({10: 48}, mx.MX_ERR_SHAPE), ({10: 96, 11: 2}, mx.MX_ERR_SHAPE), ({8: -1}, mx.MX_ERR_SHAPE),
        ({7: 1024, 8: 1 << 30, 9: 1 << 30}, mx.MX_ERR_SHAPE), ({7: 1025}, mx.MX_ERR_UNSUPPORTED), ({2: P + 16}, mx.MX_ERR_ALIGN), ({7: 0}, mx.MX_OK), ({8: 0}, mx.MX_OK)])
