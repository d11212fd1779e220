"""Refusals of the cache's entry points: the documented status for each bad argument, without a GPU (nothing is
launched before the checks)."""
import ctypes

import numpy as np

import paper_2310_10537_b200 as mx

lib = mx.lib()
_buf = np.zeros(1 << 16, np.uint8)
P = _buf.ctypes.data + (-_buf.ctypes.data) % 256
O = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, None, 0)
H = mx.binding.mx_opts_t(mx.MX_BF16, mx.MX_SCALES_SWIZZLED, None, 0)
PAD = mx.binding.mx_opts_t(mx.MX_F32, mx.MX_SCALES_SWIZZLED, None, 0, 1)
BAD = mx.binding.mx_opts_t(9, mx.MX_SCALES_SWIZZLED, None, 0)
NAN, INF = float("nan"), float("inf")


def _kv(**kw):
    d = dict(k_elems=P, k_scales=P, v_elems=P, v_scales=P, pages=3, page_size=16, heads=2, dim=64, fmt=mx.MX_E4M3) | kw
    return mx.binding.mx_kv_t(*[d[n] for n, _ in mx.binding.mx_kv_t._fields_])


def _at(**kw):
    d = dict(batch=2, new_tokens=1, q_heads=4, max_pages=3, q_stride=256, window=0, scale=0.1) | kw
    return mx.binding.mx_kv_attention_t(*[d[n] for n, _ in mx.binding.mx_kv_attention_t._fields_])


def _calls(fn, base, table):
    assert len(base) == len(fn.argtypes)
    for changes, want in table:
        args = list(base)
        for i, v in changes.items():
            args[i] = ctypes.byref(v) if isinstance(v, ctypes.Structure) else v
        assert fn(*args) == want, (changes, want)


CACHES = [(_kv(fmt=6), mx.MX_ERR_FMT), (_kv(fmt=-1), mx.MX_ERR_FMT), (_kv(fmt=mx.MX_E3M2), mx.MX_ERR_UNSUPPORTED), (_kv(fmt=mx.MX_E2M3), mx.MX_ERR_UNSUPPORTED),
          (_kv(pages=-1), mx.MX_ERR_SHAPE), (_kv(page_size=0), mx.MX_ERR_SHAPE), (_kv(heads=0), mx.MX_ERR_SHAPE), (_kv(dim=0), mx.MX_ERR_SHAPE),
          (_kv(dim=48), mx.MX_ERR_SHAPE), (_kv(pages=1 << 40, page_size=1 << 40), mx.MX_ERR_SHAPE), (_kv(pages=1 << 27), mx.MX_ERR_UNSUPPORTED),
          (_kv(pages=1 << 26, heads=4), mx.MX_ERR_UNSUPPORTED), (_kv(k_elems=None), mx.MX_ERR_NULL), (_kv(v_scales=None), mx.MX_ERR_NULL)]


def test_sizes():
    kv = _kv(k_elems=None, k_scales=None, v_elems=None, v_scales=None)
    size = lambda **k: (lib.mx_kv_elems_bytes(ctypes.byref(_kv(**k))), lib.mx_kv_scales_bytes(ctypes.byref(_kv(**k))))  # noqa: E731
    assert lib.mx_kv_elems_bytes(ctypes.byref(kv)) == 3 * 16 * 2 * 64 and lib.mx_kv_scales_bytes(ctypes.byref(kv)) == 3 * 16 * 2 * 4
    assert size(dim=160, fmt=mx.MX_E2M1) == (96 * 80, 96 * 8) and size(dim=256) == (96 * 256, 96 * 8) and size(pages=0) == (0, 0)
    assert lib.mx_kv_elems_bytes(None) == 0
    for bad, _ in CACHES[:-2]:
        assert lib.mx_kv_elems_bytes(ctypes.byref(bad)) == 0 and lib.mx_kv_scales_bytes(ctypes.byref(bad)) == 0
    assert size(pages=(1 << 31) // 16 - 1, heads=2)[0] == ((1 << 31) - 16) * 2 * 64


def test_append():
    # kv k v k_stride v_stride slots tokens rounding opts
    base = [ctypes.byref(_kv()), P, P, 128, 128, P, 5, 0, ctypes.byref(O)]
    _calls(lib.mx_kv_append, base, [({0: c}, rc) for c, rc in CACHES] + [
        ({0: None}, mx.MX_ERR_NULL), ({1: None}, mx.MX_ERR_NULL), ({2: None}, mx.MX_ERR_NULL), ({5: None}, mx.MX_ERR_NULL), ({7: 2}, mx.MX_ERR_FMT), ({8: BAD}, mx.MX_ERR_FMT),
        ({8: PAD}, mx.MX_ERR_UNSUPPORTED), ({3: 127}, mx.MX_ERR_SHAPE), ({4: 64}, mx.MX_ERR_SHAPE), ({6: -1}, mx.MX_ERR_SHAPE), ({3: 1 << 62}, mx.MX_ERR_SHAPE),
        ({6: 1 << 27}, mx.MX_ERR_UNSUPPORTED), ({6: 1 << 60}, mx.MX_ERR_SHAPE), ({1: P + 8}, mx.MX_ERR_ALIGN), ({2: P + 4}, mx.MX_ERR_ALIGN), ({3: 130}, mx.MX_ERR_ALIGN),
        ({4: 132, 8: H}, mx.MX_ERR_ALIGN), ({5: P + 2}, mx.MX_ERR_ALIGN), ({0: _kv(k_elems=P + 8)}, mx.MX_ERR_ALIGN), ({0: _kv(v_scales=P + 8)}, mx.MX_ERR_ALIGN),
        ({6: 0, 1: None}, mx.MX_OK), ({0: _kv(pages=0, k_elems=None)}, mx.MX_OK)])


def test_read():
    # kv slots tokens k_out v_out opts
    base = [ctypes.byref(_kv()), P, 5, P, P, ctypes.byref(O)]
    _calls(lib.mx_kv_read, base, [({0: c}, rc) for c, rc in CACHES] + [
        ({0: None}, mx.MX_ERR_NULL), ({1: None}, mx.MX_ERR_NULL), ({3: None}, mx.MX_ERR_NULL), ({4: None}, mx.MX_ERR_NULL), ({5: BAD}, mx.MX_ERR_FMT), ({5: PAD}, mx.MX_ERR_UNSUPPORTED),
        ({2: -1}, mx.MX_ERR_SHAPE), ({2: 1 << 27}, mx.MX_ERR_UNSUPPORTED), ({3: P + 8}, mx.MX_ERR_ALIGN), ({1: P + 2}, mx.MX_ERR_ALIGN), ({2: 0, 1: None}, mx.MX_OK)])


def test_attention():
    need = lib.mx_kv_attention_workspace_bytes(ctypes.byref(_kv()), ctypes.byref(_at()))
    assert need > 0 and lib.mx_kv_attention_workspace_bytes(ctypes.byref(_kv()), None) == 0
    assert lib.mx_kv_attention_workspace_bytes(ctypes.byref(_kv(dim=32)), ctypes.byref(_at())) == 0
    # kv attn q table lengths out lse opts workspace bytes
    base = [ctypes.byref(_kv()), ctypes.byref(_at()), P, P, P, P, P, ctypes.byref(O), P, need]
    _calls(lib.mx_kv_attention, base, [({0: c}, rc) for c, rc in CACHES] + [
        ({i: None}, mx.MX_ERR_NULL) for i in (0, 1, 2, 3, 4, 5, 8)] + [
        ({7: BAD}, mx.MX_ERR_FMT), ({7: PAD}, mx.MX_ERR_UNSUPPORTED), ({0: _kv(dim=32)}, mx.MX_ERR_UNSUPPORTED), ({0: _kv(dim=160), 1: _at(q_stride=640)}, mx.MX_ERR_UNSUPPORTED),
        ({1: _at(batch=-1)}, mx.MX_ERR_SHAPE), ({1: _at(new_tokens=0)}, mx.MX_ERR_SHAPE), ({1: _at(q_heads=3)}, mx.MX_ERR_SHAPE), ({1: _at(q_heads=0)}, mx.MX_ERR_SHAPE),
        ({1: _at(max_pages=-1)}, mx.MX_ERR_SHAPE), ({1: _at(window=-1)}, mx.MX_ERR_SHAPE), ({1: _at(scale=NAN)}, mx.MX_ERR_SHAPE), ({1: _at(scale=INF)}, mx.MX_ERR_SHAPE),
        ({1: _at(q_stride=255)}, mx.MX_ERR_SHAPE), ({1: _at(q_stride=1 << 50)}, mx.MX_ERR_SHAPE), ({1: _at(batch=1 << 40)}, mx.MX_ERR_SHAPE), ({1: _at(batch=1 << 30)}, mx.MX_ERR_UNSUPPORTED),
        ({1: _at(max_pages=1 << 28)}, mx.MX_ERR_UNSUPPORTED), ({1: _at(batch=1 << 14, max_pages=1 << 20)}, mx.MX_ERR_UNSUPPORTED), ({1: _at(batch=0, q_heads=1 << 40, q_stride=1 << 46)}, mx.MX_ERR_UNSUPPORTED),
        ({2: P + 8}, mx.MX_ERR_ALIGN), ({1: _at(q_stride=258)}, mx.MX_ERR_ALIGN), ({3: P + 2}, mx.MX_ERR_ALIGN), ({4: P + 1}, mx.MX_ERR_ALIGN), ({5: P + 4}, mx.MX_ERR_ALIGN),
        ({6: P + 2}, mx.MX_ERR_ALIGN), ({8: P + 16}, mx.MX_ERR_ALIGN), ({9: need - 1}, mx.MX_ERR_WORKSPACE), ({1: _at(batch=0), 2: None}, mx.MX_OK)])
