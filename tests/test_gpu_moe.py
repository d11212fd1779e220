"""Plan, gather and combine of a mixture of experts, and products over ragged groups.

Whole numbers and moved bytes are compared exactly.  A product is held to the bound of mx_gemm: within
1e-5 * sum |a||b| of the 64-bit dot product of the dequantized operands (BF16 outputs: and one rounding)."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2310_10537_b200 as mx
from gpu_util import GUARD

pytestmark = pytest.mark.gpu
ALL = [mx.MX_E4M3, mx.MX_E5M2, mx.MX_E3M2, mx.MX_E2M3, mx.MX_E2M1, mx.MX_INT8]


def _ids(T, k, E, seed, holes=False):
    rng = np.random.default_rng(seed)
    if T > 20000:  # (repeated experts of a token do not matter to a plan)
        ids = rng.integers(0, E, (T, k))
    else:
        ids = np.stack([rng.permutation(max(E, k))[:k] % E for _ in range(T)]) if T else np.zeros((0, k), int)
    if E > 4:
        ids[ids == 2] = 3          # an expert without rows, one with twice as many
    if holes and T:
        ids[rng.random(ids.shape) < 0.2] = -1
        ids[0, 0] = E + 5
    return ids.astype(np.int32)


def _plan_np(ids, E, align):
    counts = np.array([(ids == e).sum() for e in range(E)])
    off = np.concatenate([[0], np.cumsum((counts + align - 1) // align * align)])
    row, seen = np.full(ids.size, -1), np.zeros(E, int)
    for i, e in enumerate(ids.reshape(-1)):
        if 0 <= e < E:
            row[i] = off[e] + seen[e]
            seen[e] += 1
    return off, counts, row.reshape(ids.shape)


PLANS = [(1, 1, 1, 64), (0, 2, 4, 64), (16, 8, 64, 64), (300, 2, 5, 128), (33, 3, 7, 1), (1500, 4, 40, 64), (700, 6, 1024, 32), (4096, 8, 256, 64), (5, 40, 64, 64), (30000, 8, 200, 64), (70000, 4, 1000, 128)]


@pytest.mark.parametrize("T,k,E,align", PLANS)
def test_plan(T, k, E, align):
    for holes in (False, True):
        ids = _ids(T, k, E, T + E, holes)
        plan = mx.mx_moe_plan(torch.from_numpy(ids).cuda(), E, align)
        off, counts, row = _plan_np(ids, E, align)
        assert np.array_equal(plan.offsets.cpu().numpy(), off)
        assert np.array_equal(plan.counts.cpu().numpy(), counts)
        assert np.array_equal(plan.row_of.cpu().numpy(), row)
        assert plan.rows >= off[-1] and plan.rows % align == 0
        src = np.full(plan.rows, -1)
        src[row.reshape(-1)[row.reshape(-1) >= 0]] = np.flatnonzero(row.reshape(-1) >= 0)
        assert np.array_equal(plan.src_of.cpu().numpy(), src)


@pytest.mark.parametrize("layout", [mx.MX_SCALES_SWIZZLED, mx.MX_SCALES_LINEAR])
@pytest.mark.parametrize("fmt", ALL)
@pytest.mark.parametrize("T,k,E,align,dim", [(1, 1, 1, 64, 32), (16, 8, 64, 64, 256), (300, 2, 5, 128, 1056), (33, 3, 7, 1, 96), (70, 4, 40, 64, 4096),
                                             (0, 2, 4, 64, 64)])
def test_gather_moves_bytes(T, k, E, align, dim, fmt, layout):
    ids = _ids(T, k, E, 7, True)
    plan = mx.mx_moe_plan(torch.from_numpy(ids).cuda(), E, align)
    _, _, row = _plan_np(ids, E, align)
    R, kb, rb = plan.rows, dim // 32, dim * mx.mx_fmt_bits(fmt) // 8
    x = torch.randn(T, dim, device="cuda") * 3
    if T:
        e, s = mx.mx_quantize(x, 1, fmt, layout=layout)
    else:
        e = s = torch.empty(0, dtype=torch.uint8, device="cuda")
    ne, ns = mx.mx_elems_bytes((R, dim), 1, fmt), mx.mx_scales_bytes((R, dim), 1, layout)
    raw_e, raw_s = (torch.full((n + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda") for n in (ne, ns))
    ge, gs = mx.mx_moe_gather(e, s, dim, fmt, plan, layout, out=(raw_e[GUARD:GUARD + ne], raw_s[GUARD:GUARD + ns]))
    want_e, want_s = np.zeros((R, rb), np.uint8), np.zeros(ns, np.uint8)
    se, ss = e.cpu().numpy().reshape(T, rb), s.cpu().numpy()
    for t in range(T):
        src = [O.scale_offset(t, b, T, kb, layout) for b in range(kb)]
        for r in row[t]:
            if r >= 0:
                want_e[r] = se[t]
                want_s[[O.scale_offset(int(r), b, R, kb, layout) for b in range(kb)]] = ss[src]
    assert np.array_equal(ge.cpu().numpy().reshape(R, rb), want_e)
    assert np.array_equal(gs.cpu().numpy(), want_s)
    for raw, n in ((raw_e, ne), (raw_s, ns)):
        assert bool((raw[:GUARD] == 0xA5).all()) and bool((raw[GUARD + n:] == 0xA5).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,k,E,align,dim", [(1, 1, 1, 64, 1), (16, 8, 64, 64, 256), (300, 2, 5, 128, 1001), (33, 3, 7, 1, 96), (70, 4, 40, 64, 4096),
                                             (5, 40, 64, 64, 104), (9, 9, 16, 64, 8192), (0, 2, 4, 64, 64)])
def test_combine_and_its_gradients(T, k, E, align, dim, dtype):
    ids = _ids(T, k, E, 8, True)
    plan = mx.mx_moe_plan(torch.from_numpy(ids).cuda(), E, align)
    row, R = plan.row_of.long(), plan.rows
    g = torch.Generator(device="cuda").manual_seed(3)
    y = torch.randn(R, dim, generator=g, device="cuda").to(dtype)
    w = torch.randn(T, k, generator=g, device="cuda")
    dout = torch.randn(T, dim, generator=g, device="cuda").to(dtype)
    live = (row >= 0).unsqueeze(2)
    rows64 = torch.where(live, y.double()[row.clamp(min=0)], torch.zeros((), dtype=torch.float64, device="cuda"))
    half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    for weights in (w, None):
        w64 = (torch.ones(T, k, dtype=torch.float64, device="cuda") if weights is None else weights.double()).unsqueeze(2)
        out = mx.mx_moe_combine(y, weights, plan)
        ref, mag = (w64 * rows64).sum(1), (w64 * rows64).abs().sum(1)
        assert bool(((out.double() - ref).abs() <= (k + 1) * 2.0 ** -24 * mag + half * ref.abs()).all())
        dy, dw = mx.mx_moe_combine_backward(dout, y, weights, plan)
        want = torch.zeros(R, dim, dtype=torch.float64, device="cuda")
        for j in range(k):
            ok = row[:, j] >= 0
            want[row[ok, j]] = (w64[:, j] * dout.double())[ok]
        assert bool(((dy.double() - want).abs() <= half * want.abs()).all())
        terms = rows64 * dout.double().unsqueeze(1)
        # a dot product is a chain of at most dim / 32 + 16 additions
        assert bool(((dw.double() - terms.sum(2)).abs() <= (dim / 32 + 20) * 2.0 ** -24 * terms.abs().sum(2)).all())
        only, none = mx.mx_moe_combine_backward(dout, None, weights, plan)
        assert none is None and torch.equal(only, dy)


def test_combine_gradient_against_differences():
    plan = mx.mx_moe_plan(torch.tensor([[0, 2], [2, 1], [1, 0]], dtype=torch.int32, device="cuda"), 3, 64)
    g = torch.Generator(device="cuda").manual_seed(4)
    y, w, dout = (torch.randn(*s, generator=g, device="cuda") for s in ((plan.rows, 40), (3, 2), (3, 40)))
    dy, dw = mx.mx_moe_combine_backward(dout, y, w, plan)
    row = plan.row_of.long()
    f = lambda y64, w64: float(((w64.unsqueeze(2) * y64[row]).sum(1) * dout.double()).sum())  # noqa: E731
    for t, j, c in ((0, 0, 0), (1, 1, 17), (2, 0, 39)):
        d = torch.zeros_like(y, dtype=torch.float64)
        d[row[t, j], c] = 1e-4
        num = (f(y.double() + d, w.double()) - f(y.double() - d, w.double())) / 2e-4
        assert abs(num - float(dy[row[t, j], c])) <= 1e-6
        d = torch.zeros(3, 2, dtype=torch.float64, device="cuda")
        d[t, j] = 1e-4
        num = (f(y.double(), w.double() + d) - f(y.double(), w.double() - d)) / 2e-4
        assert abs(num - float(dw[t, j])) <= 1e-5


def _values(e, s, rows, K, fmt):
    return torch.from_numpy(O.dequantize(e.cpu().numpy(), s.cpu().numpy(), rows, K, fmt, O.F64)).cuda().view(rows, K)


def _check_product(c, a64, b64):
    ref, mag = a64 @ b64.T, a64.abs() @ b64.abs().T
    half = 0.0 if c.dtype == torch.float32 else 2.0 ** -8
    err = (c.double() - ref).abs()
    assert bool((err <= 1e-5 * mag + half * ref.abs()).all()), float((err / mag.clamp(min=1e-300)).max())


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,rows,N,K", [([64], 64, 128, 32), ([64, 0, 128], 192, 256, 128), ([0, 0], 64, 128, 96), ([192, 64, 256, 0, 320, 576], 1500, 384, 416),
                                           ([64] * 70, 70 * 64, 128, 256), ([0, 1024, 0, 64, 448], 1536, 640, 1024), ([128, 64], 64 * 3 + 13, 128, 160)])
def test_grouped_product(lens, rows, N, K, out_dtype):
    G = len(lens)
    off = _offsets(lens)
    a = torch.randn(rows, K, device="cuda")
    b = torch.randn(G, N, K, device="cuda") * 0.1
    for fa, fb in ((mx.MX_E4M3, mx.MX_E4M3), (mx.MX_E5M2, mx.MX_E4M3)):
        ea, sa = mx.mx_quantize(a, 1, fa)
        eb, sb = mx.mx_quantize(b, 2, fb)
        c = torch.full((rows, N), 77.0, dtype=out_dtype, device="cuda")
        mx.mx_gemm_grouped(ea, sa, eb, sb, torch.from_numpy(off).cuda(), rows, N, K, fa, fb, out=c, check_status=True)
        a64, b64 = _values(ea, sa, rows, K, fa), _values(eb, sb, G * N, K, fb).view(G, N, K)
        for g in range(G):
            _check_product(c[off[g]:off[g + 1]], a64[off[g]:off[g + 1]], b64[g])
        assert bool((c[off[-1]:] == 77.0).all())


@pytest.mark.parametrize("fa", [mx.MX_E4M3, mx.MX_E3M2, mx.MX_E2M1, mx.MX_E2M3])
@pytest.mark.parametrize("fb", [mx.MX_E5M2, mx.MX_E2M3, mx.MX_E2M1, mx.MX_E3M2])
def test_grouped_product_of_every_width(fa, fb):
    lens, N, K = [64, 192, 0, 128], 256, 384
    off, G, rows = _offsets(lens), 4, 384
    ea, sa = mx.mx_quantize(torch.randn(rows, K, device="cuda"), 1, fa)
    eb, sb = mx.mx_quantize(torch.randn(G, N, K, device="cuda"), 2, fb)
    o = torch.from_numpy(off).cuda()
    c = mx.mx_gemm_grouped(ea, sa, eb, sb, o, rows, N, K, fa, fb, check_status=True)
    a64, b64 = _values(ea, sa, rows, K, fa), _values(eb, sb, G * N, K, fb).view(G, N, K)
    for g in range(G):
        _check_product(c[off[g]:off[g + 1]], a64[off[g]:off[g + 1]], b64[g])
    # the same rows as a reduction axis: A [N2, rows], B [M2, rows]
    o128 = torch.tensor([0, 128, 128, 256, 384], dtype=torch.int32, device="cuda")
    ea, sa = mx.mx_quantize(torch.randn(96, rows, device="cuda"), 1, fa)
    eb, sb = mx.mx_quantize(torch.randn(200, rows, device="cuda"), 1, fb)
    c = mx.mx_gemm_grouped_k(ea, sa, eb, sb, o128, 96, 200, rows, fa, fb, check_status=True)
    a64, b64 = _values(ea, sa, 96, rows, fa), _values(eb, sb, 200, rows, fb)
    for g, (r0, r1) in enumerate(((0, 128), (128, 128), (128, 256), (256, 384))):
        _check_product(c[g], a64[:, r0:r1], b64[:, r0:r1])


@pytest.mark.parametrize("lens,rows", [([64, 128, 64], 256), ([64] * 40, 64 * 40), ([1024, 64], 1088)])
def test_grouped_product_is_that_of_mx_gemm_group_by_group(lens, rows):
    """Bit for bit: the same MMAs in the same order along K."""
    off, G, N, K = _offsets(lens), len(lens), 256, 768
    x, w = torch.randn(rows, K, device="cuda"), torch.randn(G, N, K, device="cuda")
    ea, sa = mx.mx_quantize(x, 1, mx.MX_E4M3)
    eb, sb = mx.mx_quantize(w, 2, mx.MX_E4M3)
    c = mx.mx_gemm_grouped(ea, sa, eb, sb, torch.from_numpy(off).cuda(), rows, N, K, mx.MX_E4M3, mx.MX_E4M3, check_status=True)
    for g in range(G):
        r0, r1 = int(off[g]), int(off[g + 1])
        e1, s1 = mx.mx_quantize(x[r0:r1].contiguous(), 1, mx.MX_E4M3)
        e2, s2 = mx.mx_quantize(w[g].contiguous(), 1, mx.MX_E4M3)
        assert torch.equal(c[r0:r1], mx.mx_gemm(e1, s1, e2, s2, r1 - r0, N, K, mx.MX_E4M3, mx.MX_E4M3))


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,rows,M,N", [([128], 128, 32, 8), ([0, 256, 0, 128], 512, 200, 264), ([384, 128, 0], 512, 1, 128), ([0, 0], 128, 64, 64),
                                           ([1024, 128, 640], 1824, 500, 1000)])
def test_grouped_product_along_k(lens, rows, M, N, out_dtype):
    off = _offsets(lens)
    ea, sa = mx.mx_quantize(torch.randn(M, rows, device="cuda"), 1, mx.MX_E5M2)
    eb, sb = mx.mx_quantize(torch.randn(N, rows, device="cuda"), 1, mx.MX_E4M3)
    c = torch.full((len(lens), M, N), 77.0, dtype=out_dtype, device="cuda")
    mx.mx_gemm_grouped_k(ea, sa, eb, sb, torch.from_numpy(off).cuda(), M, N, rows, mx.MX_E5M2, mx.MX_E4M3, out=c, check_status=True)
    a64, b64 = _values(ea, sa, M, rows, mx.MX_E5M2), _values(eb, sb, N, rows, mx.MX_E4M3)
    for g in range(len(lens)):
        _check_product(c[g], a64[:, off[g]:off[g + 1]], b64[:, off[g]:off[g + 1]])


def test_offsets_that_break_the_rule_touch_nothing_outside():
    rows, N, K = 256, 128, 64
    ea, sa = mx.mx_quantize(torch.randn(rows, K, device="cuda"), 1, mx.MX_E4M3)
    eb, sb = mx.mx_quantize(torch.randn(3, N, K, device="cuda"), 2, mx.MX_E4M3)
    a64, b64 = _values(ea, sa, rows, K, mx.MX_E4M3), _values(eb, sb, 3 * N, K, mx.MX_E4M3).view(3, N, K)
    big = torch.full((2 * GUARD + rows * N,), 77.0, device="cuda")
    c = big[GUARD:GUARD + rows * N].view(rows, N)
    for raw, used in (([-5, 100, 1 << 30, 1 << 30], [0, 64, 256, 256]), ([128, 64, 192, -1], [128, 64, 192, 0]), ([0, 256, 0, 999], [0, 256, 0, 256])):
        big.fill_(77.0)
        o = torch.tensor(raw, dtype=torch.int32, device="cuda")
        mx.mx_gemm_grouped(ea, sa, eb, sb, o, rows, N, K, mx.MX_E4M3, mx.MX_E4M3, out=c, check_status=True)
        assert bool((big[:GUARD] == 77.0).all()) and bool((big[GUARD + rows * N:] == 77.0).all())
        if raw[0] == -5:
            for g in range(3):
                _check_product(c[used[g]:used[g + 1]], a64[used[g]:used[g + 1]], b64[g])
    mx.mx_gemm_grouped_k(*mx.mx_quantize(torch.randn(64, rows, device="cuda"), 1, mx.MX_E4M3), *mx.mx_quantize(torch.randn(N, rows, device="cuda"), 1, mx.MX_E4M3),
                         torch.tensor([-9, 1 << 30, 5, 300], dtype=torch.int32, device="cuda"), 64, N, rows, mx.MX_E4M3, mx.MX_E4M3, check_status=True)


def test_grouped_products_on_two_streams_and_in_a_graph():
    lens, N, K = [64, 256, 128], 256, 512
    off, rows = torch.from_numpy(_offsets(lens)).cuda(), 448
    ea, sa = mx.mx_quantize(torch.randn(rows, K, device="cuda"), 1, mx.MX_E4M3)
    eb, sb = mx.mx_quantize(torch.randn(3, N, K, device="cuda"), 2, mx.MX_E2M1)
    run = lambda out: mx.mx_gemm_grouped(ea, sa, eb, sb, off, rows, N, K, mx.MX_E4M3, mx.MX_E2M1, out=out)  # noqa: E731
    want = run(torch.empty(rows, N, device="cuda")).clone()
    outs = [torch.zeros(rows, N, device="cuda") for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        run(outs[0])
        with torch.cuda.stream(side):
            run(outs[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(outs[2])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_python_refuses_wrong_tensors():
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    plan = mx.mx_moe_plan(ids, 4)
    x = torch.zeros(4, 64, device="cuda")
    e, s = mx.mx_quantize(x, 1, mx.MX_E4M3)
    off = plan.offsets
    for f in (lambda: mx.mx_moe_plan(ids.long(), 4), lambda: mx.mx_moe_plan(ids[0], 4), lambda: mx.mx_moe_plan(ids.cpu(), 4),
              lambda: mx.mx_moe_gather(e[:100], s, 64, mx.MX_E4M3, plan), lambda: mx.mx_moe_gather(e, s[:100], 64, mx.MX_E4M3, plan),
              lambda: mx.mx_moe_gather(e, s, 64, mx.MX_E4M3, plan._replace(offsets=off[:3])), lambda: mx.mx_moe_combine(x, None, plan),
              lambda: mx.mx_moe_combine_backward(x[:3], None, None, plan), lambda: mx.mx_moe_combine_backward(x, x, None, plan),
              lambda: mx.mx_gemm_grouped(e, s, e, s, off, 4, 128, 64, mx.MX_E4M3, mx.MX_E4M3), lambda: mx.mx_gemm_grouped(e, s, e, s, off.long(), 4, 128, 64, 0, 0),
              lambda: mx.mx_gemm_grouped_k(e, s, e, s, off, 4, 8, 96, 0, 0)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: mx.mx_moe_plan(ids, 0), lambda: mx.mx_moe_plan(ids, 2000), lambda: mx.mx_moe_plan(ids, 4, 5000),
              lambda: mx.mx_moe_gather(e, s, 40, mx.MX_E4M3, plan)):
        with pytest.raises(mx.MxError):
            f()
