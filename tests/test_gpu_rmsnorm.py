"""RMS norm with MX output and its backward pass against the definition in 64 bits.

The MX output is checked in two exact steps and one bounded one: with FP32 tensors the call also hands
out the norm it quantized (y_out), whose codes and scales must be the oracle's bit for bit and whose
values must be those of the 64-bit definition; and the BF16 call must give exactly the bytes of the FP32
call on the same numbers (its arithmetic is the same, only the loads differ).

Bound of y: a sum of `dim` squares over at most 1024 threads is a chain of at most dim / 64 + 16 FP32
additions, each off by 2^-24 relative, halved by the square root; rsqrt, eps and two products add 6 more."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2310_10537_b200 as mx

pytestmark = pytest.mark.gpu
EPS = 1e-5
FMTS = [mx.MX_E4M3, mx.MX_E5M2, mx.MX_E3M2, mx.MX_E2M3, mx.MX_E2M1, mx.MX_INT8]


def _u(dim):
    return (dim / 64 + 24) * 2.0 ** -24


def _inputs(rows, dim, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gain = torch.exp(torch.randn(dim, generator=g, device="cuda"))
    x = (torch.randn(rows, dim, generator=g, device="cuda") * gain).bfloat16().to(dtype)
    r = (torch.randn(rows, dim, generator=g, device="cuda") * gain).bfloat16().to(dtype)
    w = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).bfloat16().to(dtype)
    return x, r, w


def _norm64(h, w):
    h = h.double()
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * w.double()


@pytest.mark.parametrize("layout", [mx.MX_SCALES_SWIZZLED, mx.MX_SCALES_LINEAR])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,dim", [(1, 32), (3, 64), (1, 1), (5, 31), (7, 1000), (130, 4096), (129, 160), (2, 8192), (200, 1001),
                                      (300, 16384), (3, 20000), (257, 8), (2, 60001), (310, 4001)])
def test_mx_output_is_the_quantized_norm(rows, dim, fmt, layout):
    x, r, w = _inputs(rows, dim, 1)
    for residual in (None, r):
        for rounding in (mx.MX_RNE, mx.MX_RHAZ):
            y = torch.empty_like(x)
            e, s, h = mx.mx_rmsnorm_quantize(x, w, fmt, EPS, residual=residual, rounding=rounding, layout=layout, y_out=y)
            want_h = x if residual is None else x + r
            assert (h is None) == (residual is None)
            if h is not None:
                assert torch.equal(h, want_h)
            ref = _norm64(x.double() if residual is None else x.double() + r.double(), w)
            err = (y.double() - ref).abs()
            assert bool((err <= _u(dim) * ref.abs()).all()), float((err / ref.abs().clamp(min=1e-300)).max())
            we, ws = O.quantize(y.cpu().numpy(), 1, fmt, rounding, layout)
            assert np.array_equal(e.cpu().numpy(), we), "codes"
            assert np.array_equal(s.cpu().numpy(), ws), "scales"


@pytest.mark.parametrize("rows,dim", [(1, 32), (5, 31), (200, 1001), (16, 4096), (301, 4096), (130, 8192), (150, 16384)])
def test_bf16_tensors_give_the_bytes_of_fp32_ones(rows, dim):
    x, r, w = _inputs(rows, dim, 2)
    xb, rb, wb = x.bfloat16(), r.bfloat16(), w.bfloat16()
    for fmt in (mx.MX_E4M3, mx.MX_E2M3, mx.MX_E2M1):
        y = torch.empty_like(x)
        yb = torch.empty_like(xb)
        e, s, h = mx.mx_rmsnorm_quantize(x, w, fmt, EPS, residual=r, y_out=y)
        eb, sb, hb = mx.mx_rmsnorm_quantize(xb, wb, fmt, EPS, residual=rb, y_out=yb)
        ew, sw, _ = mx.mx_rmsnorm_quantize(xb, w, fmt, EPS, residual=rb)  # FP32 weights of the same values
        assert torch.equal(e, eb) and torch.equal(s, sb) and torch.equal(e, ew) and torch.equal(s, sw)
        assert torch.equal(h.bfloat16(), hb) and torch.equal(y.bfloat16(), yb)


def test_residual_stream_may_be_updated_in_place_and_buffers_are_filled():
    x, r, w = _inputs(77, 1024, 3, torch.bfloat16)
    e, s, h = mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, EPS, residual=r)
    for alias in ("x", "residual"):
        x2, r2 = x.clone(), r.clone()
        out = (torch.full_like(e, 0xA5), torch.full_like(s, 0xA5))
        e2, s2, h2 = mx.mx_rmsnorm_quantize(x2, w, mx.MX_E4M3, EPS, residual=r2, h_out=x2 if alias == "x" else r2, out=out)
        assert h2.data_ptr() == (x2 if alias == "x" else r2).data_ptr()
        assert torch.equal(h2, h) and torch.equal(e2, e) and torch.equal(s2, s)


def test_zero_rows_infinities_and_tiny_values():
    x = torch.zeros(5, 256, device="cuda")
    x[1] = 1e-30
    x[2, 7] = float("inf")
    x[3, 9] = float("nan")
    x[4] = 1.5
    w = torch.ones(256, device="cuda")
    y = torch.empty_like(x)
    e, s, _ = mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, 1e-6, y_out=y, layout=mx.MX_SCALES_LINEAR)
    e, s = e.view(5, 256), s.view(5, 8)
    assert bool((e[0] == 0).all()) and bool((s[0] == 0).all())
    assert torch.allclose(y[1], torch.full_like(y[1], 1e-27), rtol=1e-5, atol=0)
    assert int(s[2, 0]) == 0xFF and bool((s[2, 1:] == 0).all()) and bool((e[2] == 0).all())   # Inf / Inf, finite / Inf
    assert bool((s[3] == 0xFF).all()) and bool((e[3] == 0).all())
    assert torch.allclose(y[4], torch.ones_like(y[4]), rtol=1e-6)
    assert mx.mx_rmsnorm_quantize(x[:0], w, mx.MX_E4M3)[0].numel() == 0


def _backward64(dy, h, w, dres):
    dy, h, w = dy.double(), h.double(), w.double()
    inv = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    n = h * inv
    g = dy * w
    dh = inv * (g - n * (g * n).mean(1, keepdim=True))
    return dh if dres is None else dh + dres.double(), (dy * n).sum(0), inv * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)), (dy * n).abs().sum(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,dim", [(1, 1), (1, 32), (4, 7), (300, 8), (1023, 1000), (130, 1001), (297, 4096), (64, 8192), (40, 8200), (700, 513), (600, 4001), (300, 8191), (5, 9000)])
def test_backward_against_the_formula(rows, dim, dtype):
    h, r, w = _inputs(rows, dim, 4, dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    dy = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    for dres in (None, r):
        dh, dw = mx.mx_rmsnorm_backward(dy, h, w, EPS, dres=dres)
        ref, refw, mag, magw = _backward64(dy, h, w, dres)
        # FP32 sums over a row (see above), 8 more roundings, and one to the output's type
        half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
        tol = 2 * _u(dim) * mag + half * (ref.abs() + (0 if dres is None else dres.double().abs() * 2.0 ** -23))
        assert bool(((dh.double() - ref).abs() <= tol + 2.0 ** -24 * (0 if dres is None else dres.double().abs())).all())
        # a column's sum is a chain of at most rows / 64 + 64 additions
        tolw = (rows / 64 + 64 + 2 * dim / 64 + 32) * 2.0 ** -24 * magw
        assert bool(((dw.double() - refw).abs() <= tolw).all())
        again = mx.mx_rmsnorm_backward(dy, h, w, EPS, dres=dres)
        assert torch.equal(again[0], dh) and torch.equal(again[1], dw), "not reproducible"
        for alias in (dy.clone(), None if dres is None else dres.clone()):  # in place of an input
            if alias is None:
                continue
            if torch.equal(alias, dy):
                got = mx.mx_rmsnorm_backward(alias, h, w, EPS, dres=dres, out=alias)
            else:
                got = mx.mx_rmsnorm_backward(dy, h, w, EPS, dres=alias, out=alias)
            assert torch.equal(got[0], dh) and torch.equal(got[1], dw)


def test_backward_against_differences():
    """Central differences of the 64-bit norm: loss = sum(dy * y(h, w)).  With step 1e-4 |h| the difference is
    exact to about 1e-8 of the terms' size; FP32 gives 1e-5 of it."""
    rows, dim = 3, 96
    h, _, w = _inputs(rows, dim, 6)
    dy = torch.randn(rows, dim, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    dh, dw = mx.mx_rmsnorm_backward(dy, h, w, EPS)

    def loss(h64, w64):
        return (dy.double() * (h64 / torch.sqrt((h64 * h64).mean(1, keepdim=True) + EPS) * w64)).sum()

    for i, j in ((0, 0), (1, 50), (2, 95)):
        step = 1e-4
        d = torch.zeros(rows, dim, dtype=torch.float64, device="cuda")
        d[i, j] = step
        num = (loss(h.double() + d, w.double()) - loss(h.double() - d, w.double())) / (2 * step)
        assert abs(float(num) - float(dh[i, j])) <= 1e-5 * float(dh[i].abs().max()) + 1e-7
        num = (loss(h.double(), w.double() + d[i]) - loss(h.double(), w.double() - d[i])) / (2 * step)
        assert abs(float(num) - float(dw[j])) <= 1e-5 * float(dw.abs().max()) + 1e-7


def test_backward_without_rows_and_on_another_stream():
    w = torch.ones(64, device="cuda")
    dh, dw = mx.mx_rmsnorm_backward(torch.empty(0, 64, device="cuda"), torch.empty(0, 64, device="cuda"), w)
    assert dh.shape == (0, 64) and bool((dw == 0).all())
    h, r, w = _inputs(500, 2048, 8, torch.bfloat16)
    want = mx.mx_rmsnorm_backward(r, h, w, EPS)
    fwd = mx.mx_rmsnorm_quantize(h, w, mx.MX_E4M3, EPS, residual=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mx.mx_rmsnorm_backward(r, h, w, EPS)
        gotf = mx.mx_rmsnorm_quantize(h, w, mx.MX_E4M3, EPS, residual=r)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + fwd, got + gotf))


def test_python_refuses_wrong_tensors():
    x, r, w = _inputs(4, 64, 9)
    for bad in (dict(residual=r.bfloat16()), dict(residual=r[:3]), dict(residual=r.t().contiguous().t()), dict(y_out=r[:, :32].contiguous()),
                dict(residual=r.cpu()), dict(out=(torch.empty(4, dtype=torch.uint8, device="cuda"),) * 2)):
        with pytest.raises(ValueError):
            mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, EPS, **bad)
    with pytest.raises(ValueError):
        mx.mx_rmsnorm_quantize(x, w[:32], mx.MX_E4M3)
    with pytest.raises(TypeError):
        mx.mx_rmsnorm_quantize(x.half(), w.half(), mx.MX_E4M3)
    with pytest.raises(mx.MxError):
        mx.mx_rmsnorm_quantize(x, w, mx.MX_E4M3, -1.0)
    with pytest.raises(mx.MxError):
        mx.mx_rmsnorm_backward(x, x, w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
