"""Cases of the mixture-of-experts block on MX operands: RMS norm with MX output, routing, moving rows
to their experts and back, and the experts' products, each with its backward form.

`own` false: every operator in elementary torch operations in FP32.  `own` true: the calls a user makes
of the library.  Sizes are those of the library's own workloads (rows of 4096 and 8192, FFN widths of
4096 to 16384) and generic expert counts."""
import math

import torch

own = False

BLOCK = 32
EMAX = {"e4m3": 8, "e5m2": 15}
MAXN = {"e4m3": 448.0, "e5m2": 57344.0, "e2m1": 6.0}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BITS = {"e4m3": 8, "e5m2": 8, "e2m1": 4}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # one decoding step of 16 sequences: the norm in front of a product; a few microseconds
        {"name": "norm_decode", "op": "norm", "rows": 16, "dim": 4096, "dtype": "bf16", "residual": True, "fmt": "e4m3"},
        # a prefill or training batch of 8192 tokens
        {"name": "norm_prefill", "op": "norm", "rows": 8192, "dim": 8192, "dtype": "bf16", "residual": True, "fmt": "e4m3"},
        # the norm's backward pass in training, with the gradient that arrives along the residual
        {"name": "norm_grad", "op": "norm_grad", "rows": 8192, "dim": 4096, "dtype": "bf16", "residual": True},
        # odd row count, a dimension that is no whole number of blocks, FP32
        {"name": "norm_grad_ragged", "op": "norm_grad", "rows": 1023, "dim": 1000, "dtype": "f32", "residual": False},
        # routing one decoding step
        {"name": "route_decode", "op": "route", "tokens": 64, "experts": 64, "topk": 2, "score": "softmax", "bias": False,
         "groups": 1, "topk_groups": 1, "dtype": "bf16"},
        # routing a prefill batch with balanced sigmoid scores in groups
        {"name": "route_prefill", "op": "route", "tokens": 16384, "experts": 256, "topk": 8, "score": "sigmoid", "bias": True,
         "groups": 8, "topk_groups": 4, "dtype": "f32"},
        # the router's gradient in training
        {"name": "route_grad", "op": "route_grad", "tokens": 16384, "experts": 128, "topk": 8, "score": "softmax", "dtype": "f32"},
        # the tokens of a prefill batch to their experts: plan and MX rows
        {"name": "dispatch", "op": "dispatch", "tokens": 8192, "dim": 4096, "experts": 64, "topk": 8, "align": 64},
        # the experts' outputs back to the tokens, in training: gradients of outputs and routing weights
        {"name": "combine_grad", "op": "combine_grad", "tokens": 8192, "dim": 4096, "experts": 64, "topk": 4, "align": 128, "dtype": "bf16"},
        # one decoding step: a few rows for each of many experts, FP4 weights: bound by reading the weights
        {"name": "experts_decode", "op": "experts", "rows": 128, "experts": 64, "active": 56, "n": 2048, "k": 4096,
         "fmt_a": "e4m3", "fmt_b": "e2m1"},
        # a prefill batch: 8192 tokens to 8 of 32 experts
        {"name": "experts_prefill", "op": "experts", "rows": 65536, "experts": 32, "active": 32, "n": 4096, "k": 4096,
         "fmt_a": "e4m3", "fmt_b": "e4m3"},
        # the experts' weight gradients of a training batch
        {"name": "experts_wgrad", "op": "wgrad", "rows": 32768, "experts": 16, "active": 16, "m": 4096, "n": 2048,
         "fmt_a": "e5m2", "fmt_b": "e4m3"},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    n = max(lo, min(hi, int(round(v / step)) * step))
    return n + step if n == 24 * 128 else n  # a width of no workload here


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "route", "route", "route_grad", "dispatch", "combine_grad", "combine", "experts",
                     "experts", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "norm_grad"):
        rows = _log(rng, 16 if op == "norm" else 64, 16384)
        dim = _log(rng, 256, 8192, rng.choice([1, 8, 32, 128, 512]))
        c = {"op": op, "rows": rows, "dim": dim, "dtype": dtype, "residual": rng.random() < 0.7}
        if op == "norm":
            c["fmt"] = rng.choice(["e4m3", "e4m3", "e5m2"])
        return c
    if op in ("route", "route_grad"):
        experts = rng.choice([8, 16, 40, 64, 96, 128, 160, 256, 384])
        # a renormalised single choice has no gradient
        topk = rng.choice([k for k in (1, 2, 4, 6, 8) if k <= experts // 4 and (k > 1 or op == "route")])
        c = {"op": op, "tokens": _log(rng, 16, 32768), "experts": experts, "topk": topk,
             "score": rng.choice(["softmax", "sigmoid"]), "dtype": dtype}
        if op == "route":
            groups = rng.choice([1, 1, 4, 8])
            c["bias"] = c["score"] == "sigmoid" and rng.random() < 0.7
            c["groups"] = groups
            c["topk_groups"] = 1 if groups == 1 else max(groups // 2, -(-topk * groups // experts))
        return c
    if op in ("dispatch", "combine", "combine_grad"):
        experts = rng.choice([8, 16, 32, 64, 128, 256])
        c = {"op": op, "tokens": _log(rng, 8, 8192), "dim": _log(rng, 512, 8192, rng.choice([32, 128])), "experts": experts,
             "topk": rng.choice([1, 2, 4, 6, 8]), "align": rng.choice([64, 128])}
        if op != "dispatch":
            c["dtype"] = dtype
        return c
    experts = rng.choice([4, 8, 16, 32])
    if op == "experts":
        rows = _log(rng, 8, 32768)
        active = max(1, min(experts, rows // 2, rng.randint(experts // 2, experts)))
        return {"op": op, "rows": rows, "experts": experts, "active": active, "n": _log(rng, 512, 4096, 128),
                "k": _log(rng, 512, 4096, 128), "fmt_a": rng.choice(["e4m3", "e4m3", "e5m2"]), "fmt_b": rng.choice(["e4m3", "e2m1"])}
    rows = _log(rng, 512, 32768)
    return {"op": op, "rows": rows, "experts": experts, "active": max(1, rng.randint(experts // 2, experts)),
            "m": _log(rng, 512, 4096, 128), "n": _log(rng, 512, 2048, 128), "fmt_a": rng.choice(["e4m3", "e5m2"]), "fmt_b": "e4m3"}


# ---------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _swizzle(s, fill=0):
    """[rows, kblocks] scale bytes -> the 512-byte chunks of 128 rows x 4 blocks that the products read."""
    rows, kb = s.shape
    full = torch.nn.functional.pad(s, (0, -kb % 4, 0, -rows % 128), value=fill)
    v = full.view(full.shape[0] // 128, 4, 32, full.shape[1] // 4, 4)
    return v.permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _unswizzle(flat, rows, kb):
    r, k = (rows + 127) // 128, (kb + 3) // 4
    v = flat.view(r, k, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(r * 128, k * 4)
    return v[:rows, :kb]


def _block_scale(v, emax):
    """v [rows, blocks, 32] FP32 -> scale bytes (shared exponent + 127) and v / scale."""
    amax = v.abs().amax(-1)
    e = torch.frexp(amax)[1] - 1
    byte = torch.where(amax >= 2.0 ** -126, (e - emax + 127).clamp(0, 254), torch.zeros_like(e))
    return byte, torch.ldexp(v, (127 - byte).unsqueeze(-1))


def _make_mx(x, fmt):
    """An MX tensor of x [rows, K] FP32 as a user's program holds it: packed codes, swizzled scales."""
    rows, K = x.shape
    byte, p = _block_scale(x.view(rows, K // BLOCK, BLOCK), 2 if fmt == "e2m1" else EMAX[fmt])
    p = p.view(rows, K).clamp(-MAXN[fmt], MAXN[fmt])
    if fmt == "e2m1":
        grid = torch.tensor(E2M1, device=x.device)
        code = torch.bucketize(p.abs(), (grid[1:] + grid[:-1]) / 2).to(torch.uint8) | ((p < 0).to(torch.uint8) << 3)
        codes = code[:, 0::2] | (code[:, 1::2] << 4)
    else:
        codes = p.to(F8[fmt]).view(torch.uint8)
    return codes.contiguous().view(-1), _swizzle(byte.to(torch.uint8))


def _split(g, total, experts, active):
    """Rows per expert: `active` experts share `total` rows unevenly, as trained routers do."""
    load = torch.exp(0.5 * torch.randn(active, generator=g, device="cuda", dtype=torch.float64))
    n = torch.floor((total - active) * load / load.sum()).long() + 1
    n[0] += total - int(n.sum())
    who = torch.randperm(experts, generator=g, device="cuda")[:active]
    counts = torch.zeros(experts, dtype=torch.long, device="cuda")
    counts[who] = n
    return counts


def _offsets(counts, align):
    padded = (counts + align - 1) // align * align
    return torch.cat([padded.new_zeros(1), padded.cumsum(0)])


def _choices(g, tokens, experts, topk):
    """Distinct experts per token, some experts preferred."""
    taste = 0.5 * torch.randn(experts, generator=g, device="cuda")
    noise = -torch.log(-torch.log(torch.rand((tokens, experts), generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    return torch.topk(taste + noise, min(topk, experts), dim=1).indices.to(torch.int32)


def _rows_bound(tokens, topk, experts, align):
    return (tokens * topk + min(experts, tokens * topk) * (align - 1)) // align * align


def _plan_of(ids, experts, align):
    """Group offsets and the row of every choice, choices of an expert in token order."""
    flat = ids.view(-1).long()
    counts = (flat.unsqueeze(1) == torch.arange(experts, device=flat.device)).sum(0) if flat.numel() * experts < 1 << 24 \
        else torch.zeros(experts, dtype=torch.long, device=flat.device).index_add_(0, flat, torch.ones_like(flat))
    offsets = _offsets(counts, align)
    order = torch.sort(flat, stable=True).indices
    first = counts.cumsum(0) - counts
    row = torch.empty_like(flat)
    row[order] = torch.arange(flat.numel(), device=flat.device) - first[flat[order]] + offsets[flat[order]]
    return offsets.to(torch.int32), counts.to(torch.int32), row.to(torch.int32).view(ids.shape)


def prepare(case, seed):
    g = _rng(seed)
    dev = "cuda"
    op = case["op"]
    randn = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    s = dict(case)
    if op in ("norm", "norm_grad"):
        dt, rows, dim = DT[case["dtype"]], case["rows"], case["dim"]
        # a residual stream has a few large channels
        gain = torch.exp(0.5 * randn(dim))
        s["x"] = (randn(rows, dim) * gain).to(dt)
        s["w"] = (1.0 + 0.1 * randn(dim)).to(dt)
        s["res"] = (2.0 * randn(rows, dim) * gain).to(dt) if case["residual"] and op == "norm" else None
        if op == "norm_grad":
            s["dy"] = (1e-3 * randn(rows, dim)).to(dt)
            s["res"] = (1e-3 * randn(rows, dim)).to(dt) if case["residual"] else None
        return s
    if op in ("route", "route_grad"):
        dt, T, E, k = DT[case["dtype"]], case["tokens"], case["experts"], case["topk"]
        s["logits"] = (1.5 * randn(T, E) + 0.5 * randn(E)).to(dt)
        s["bias"] = 0.05 * randn(E) if case.get("bias") else None
        if op == "route_grad":
            s["dweights"] = 1e-2 * randn(T, k)
            s["ids"] = torch.topk(s["logits"].float(), k, dim=1).indices.to(torch.int32)
        return s
    if op in ("dispatch", "combine", "combine_grad"):
        T, D, E, k = case["tokens"], case["dim"], case["experts"], case["topk"]
        s["topk"] = k = min(k, E)
        s["ids"] = _choices(g, T, E, k)
        s["rows"] = _rows_bound(T, k, E, case["align"])
        if op == "dispatch":
            s["elems"], s["scales"] = _make_mx(randn(T, D), "e4m3")
            return s
        dt = DT[case["dtype"]]
        s["offsets"], s["counts"], s["row_of"] = _plan_of(s["ids"], E, case["align"])
        s["y"] = randn(s["rows"], D).to(dt)
        s["weights"] = torch.softmax(randn(T, k), 1)
        if op == "combine_grad":
            s["dout"] = (1e-3 * randn(T, D)).to(dt)
        return s
    E = case["experts"]
    counts = _split(g, case["rows"], E, case["active"])
    align = 64 if op == "experts" else 128
    offsets = _offsets(counts, align)
    # rows that a program allocates before it knows how the groups fall
    R = _rows_bound(case["rows"], 1, E, align)
    s["offsets"], s["rows_padded"], s["largest"] = offsets.to(torch.int32), R, int((offsets[1:] - offsets[:-1]).max())
    pos = torch.arange(R, device=dev)
    group = torch.searchsorted(offsets[1:], pos, right=True).clamp(max=E - 1)
    live = pos - offsets[group] < counts[group]
    if op == "experts":
        N, K = case["n"], case["k"]
        s["a"], s["sa"] = _make_mx(randn(R, K) * live.unsqueeze(1), case["fmt_a"])
        s["b"], s["sb"] = _make_mx(0.02 * randn(E * N, K), case["fmt_b"])
        s["out"] = torch.zeros((R, N), dtype=torch.bfloat16, device=dev)  # rows behind the last group stay as they are
    else:
        s["a"], s["sa"] = _make_mx(1e-3 * randn(case["m"], R) * live, case["fmt_a"])
        s["b"], s["sb"] = _make_mx(randn(case["n"], R) * live, case["fmt_b"])
    return s


# ---------------------------------------------------------------------------------------------------
# The operators
# ---------------------------------------------------------------------------------------------------

_mx = None


def _lib():
    global _mx
    if _mx is None:
        import paper_2310_10537_b200
        _mx = paper_2310_10537_b200
    return _mx


def run(s):
    return (_run_own if own else _run_plain)(s)


EPS = 1e-6
ROUTED_SCALE = 2.5


def _run_own(s):
    mx = _lib()
    op = s["op"]
    if op == "norm":
        elems, scales, h = mx.mx_rmsnorm_quantize(s["x"], s["w"], mx.FORMATS[s["fmt"]], EPS, residual=s["res"])
        out = {"codes": elems.view(F8[s["fmt"]]), "scales": scales.view(torch.float8_e8m0fnu)}
        if h is not None:
            out["h"] = h
        return out
    if op == "norm_grad":
        dh, dw = mx.mx_rmsnorm_backward(s["dy"], s["x"], s["w"], EPS, dres=s["res"])
        return {"dh": dh, "dw": dw}
    if op == "route":
        ids, w = mx.mx_route(s["logits"], s["topk"], mx.SCORES[s["score"]], bias=s["bias"], groups=s["groups"],
                             topk_groups=s["topk_groups"], group_score=mx.MX_GROUP_TOP2 if s["score"] == "sigmoid" else mx.MX_GROUP_MAX,
                             renormalize=True, scale=ROUTED_SCALE)
        return {"ids": ids, "weights": w}
    if op == "route_grad":
        return {"dlogits": mx.mx_route_backward(s["dweights"], s["logits"], s["ids"], mx.SCORES[s["score"]], renormalize=True,
                                                scale=ROUTED_SCALE)}
    if op == "dispatch":
        plan = mx.mx_moe_plan(s["ids"], s["experts"], s["align"])
        elems, scales = mx.mx_moe_gather(s["elems"], s["scales"], s["dim"], mx.MX_E4M3, plan)
        return {"offsets": plan.offsets, "row_of": plan.row_of, "codes": elems.view(torch.float8_e4m3fn),
                "scales": scales.view(torch.float8_e8m0fnu)}
    if op in ("combine", "combine_grad"):
        plan = mx.MoePlan(s["offsets"], s["counts"], s["row_of"], s["rows"])
        if op == "combine":
            return {"out": mx.mx_moe_combine(s["y"], s["weights"], plan)}
        dy, dw = mx.mx_moe_combine_backward(s["dout"], s["y"], s["weights"], plan)
        return {"dy": dy, "dw": dw}
    fa, fb, R = mx.FORMATS[s["fmt_a"]], mx.FORMATS[s["fmt_b"]], s["rows_padded"]
    if op == "experts":
        return {"c": mx.mx_gemm_grouped(s["a"], s["sa"], s["b"], s["sb"], s["offsets"], R, s["n"], s["k"], fa, fb,
                                        out=s["out"])}
    return {"c": mx.mx_gemm_grouped_k(s["a"], s["sa"], s["b"], s["sb"], s["offsets"], s["m"], s["n"], R, fa, fb,
                                      out_dtype=torch.bfloat16)}


def _quantized(y, fmt):
    """Algorithm 1 along the last axis, rows zero-padded to whole blocks: element and scale values."""
    rows, L = y.shape
    y = torch.nn.functional.pad(y, (0, -L % BLOCK))
    byte, p = _block_scale(y.view(rows, -1, BLOCK), EMAX[fmt])
    codes = p.clamp(-MAXN[fmt], MAXN[fmt]).to(F8[fmt])
    return codes.view(-1), _swizzle(byte.to(torch.uint8)).view(torch.float8_e8m0fnu)


def _values(codes, scales, rows, K, fmt):
    """The FP32 values of an MX tensor [rows, K] with swizzled scales."""
    if fmt == "e2m1":
        grid = torch.tensor(E2M1 + [-v for v in E2M1], device=codes.device)
        b = codes.view(rows, K // 2)
        p = torch.stack([grid[(b & 15).long()], grid[(b >> 4).long()]], -1).view(rows, K)
    else:
        p = codes.view(F8[fmt]).view(rows, K).float()
    x = torch.exp2(_unswizzle(scales, rows, K // BLOCK).float() - 127.0)
    return (p.view(rows, -1, BLOCK) * x.unsqueeze(-1)).view(rows, K)


def _scores(logits, score):
    x = logits.float()
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    e = torch.exp(x - x.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _in_groups(rows, offsets, largest):
    """Index [groups, largest] of each group's rows, and which of them exist."""
    at = offsets[:-1].long().unsqueeze(1) + torch.arange(largest, device=offsets.device)
    return at.clamp(max=max(rows - 1, 0)), at < offsets[1:].long().unsqueeze(1)


def _run_plain(s):
    op = s["op"]
    if op == "norm":
        h = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["w"].float()
        codes, scales = _quantized(y, s["fmt"])
        out = {"codes": codes, "scales": scales}
        if s["res"] is not None:
            out["h"] = h.to(s["x"].dtype)
        return out
    if op == "norm_grad":
        h, dy = s["x"].float(), s["dy"].float()
        r = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        xh, gr = h * r, dy * s["w"].float()
        dh = r * (gr - xh * (gr * xh).mean(1, keepdim=True))
        if s["res"] is not None:
            dh = dh + s["res"].float()
        return {"dh": dh.to(s["x"].dtype), "dw": (dy * xh).sum(0)}
    if op == "route":
        T, E = s["logits"].shape
        sc = _scores(s["logits"], s["score"])
        # softmax keeps the order of the logits, and equal logits are ties
        c = sc + s["bias"] if s["bias"] is not None else (s["logits"].float() if s["score"] == "softmax" else sc)
        if s["groups"] > 1:
            grp = c.view(T, s["groups"], -1)
            gs = torch.sort(grp, dim=2, descending=True).values[:, :, :2].sum(2) if s["score"] == "sigmoid" else grp.amax(2)
            best = torch.sort(gs, dim=1, descending=True, stable=True).indices[:, :s["topk_groups"]]
            keep = torch.zeros_like(gs).scatter_(1, best, 1.0) > 0
            c = torch.where(keep.unsqueeze(2), grp, torch.full_like(grp, -math.inf)).view(T, E)
        ids = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :s["topk"]]
        w = sc.gather(1, ids)
        return {"ids": ids.to(torch.int32), "weights": w / w.sum(1, keepdim=True) * ROUTED_SCALE}
    if op == "route_grad":
        ids, dw = s["ids"].long(), s["dweights"]
        sc = _scores(s["logits"], s["score"])
        sel = sc.gather(1, ids)
        tot = sel.sum(1, keepdim=True)
        ds = ROUTED_SCALE * (dw - (dw * sel).sum(1, keepdim=True) / tot) / tot
        full = torch.zeros_like(sc).scatter_(1, ids, ds)
        d = full * sc * (1.0 - sc) if s["score"] == "sigmoid" else sc * (full - (full * sc).sum(1, keepdim=True))
        return {"dlogits": d.to(s["logits"].dtype)}
    if op == "dispatch":
        T, D, k, R = s["tokens"], s["dim"], s["topk"], s["rows"]
        offsets, counts, row_of = _plan_of(s["ids"], s["experts"], s["align"])
        token = torch.arange(T * k, device="cuda") // k
        codes = torch.zeros((R, D), dtype=torch.uint8, device="cuda")
        codes[row_of.view(-1).long()] = s["elems"].view(T, D)[token]
        kb = D // BLOCK
        sc = torch.zeros((R, kb), dtype=torch.uint8, device="cuda")
        sc[row_of.view(-1).long()] = _unswizzle(s["scales"], T, kb)[token]
        return {"offsets": offsets, "row_of": row_of, "codes": codes.view(-1).view(torch.float8_e4m3fn),
                "scales": _swizzle(sc).view(torch.float8_e8m0fnu)}
    if op in ("combine", "combine_grad"):
        at = s["row_of"].long()
        rows = s["y"][at.view(-1)].float().view(*at.shape, -1)
        if op == "combine":
            return {"out": (rows * s["weights"].unsqueeze(2)).sum(1).to(s["y"].dtype)}
        dout = s["dout"].float()
        dy = torch.zeros(s["y"].shape, device="cuda")
        dy[at.view(-1)] = (s["weights"].unsqueeze(2) * dout.unsqueeze(1)).view(-1, dout.shape[1])
        return {"dy": dy.to(s["y"].dtype), "dw": (rows * dout.unsqueeze(1)).sum(2)}
    R, off = s["rows_padded"], s["offsets"]
    at, live = _in_groups(R, off, s["largest"])
    if op == "experts":
        E, N, K = s["experts"], s["n"], s["k"]
        a = _values(s["a"], s["sa"], R, K, s["fmt_a"])
        b = _values(s["b"], s["sb"], E * N, K, s["fmt_b"]).view(E, N, K)
        c = torch.matmul(a[at.view(-1)].view(E, -1, K), b.transpose(1, 2))
        out = torch.zeros((R, N), device="cuda")
        out[at[live]] = c[live]
        return {"c": out.to(torch.bfloat16)}
    a = _values(s["a"], s["sa"], s["m"], R, s["fmt_a"])
    b = _values(s["b"], s["sb"], s["n"], R, s["fmt_b"])
    pick = lambda v: v[:, at.view(-1)].view(v.shape[0], *at.shape).permute(1, 0, 2) * live.unsqueeze(1)  # noqa: E731
    return {"c": torch.matmul(pick(a), pick(b).transpose(1, 2)).to(torch.bfloat16)}


# ---------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    esz = {"bf16": 2, "f32": 4}.get(case.get("dtype"), 2)
    if op in ("norm", "norm_grad"):
        n, dim = case["rows"] * case["dim"], case["dim"]
        if op == "norm":
            per = esz * (3 if case["residual"] else 1) + 1 + 1 / 32
            return {"bytes": n * per + dim * esz, "flops": 8 * n}
        return {"bytes": n * esz * (4 if case["residual"] else 3) + dim * (esz + 4), "flops": 12 * n}
    if op in ("route", "route_grad"):
        n, t = case["tokens"] * case["experts"], case["tokens"] * min(case["topk"], case["experts"])
        if op == "route":
            return {"bytes": n * esz + 8 * t, "flops": 6 * n}
        return {"bytes": 2 * n * esz + 8 * t, "flops": 8 * n}
    if op in ("dispatch", "combine", "combine_grad"):
        T, D, k, E = case["tokens"], case["dim"], min(case["topk"], case["experts"]), case["experts"]
        R = _rows_bound(T, k, E, case["align"])
        if op == "dispatch":
            return {"bytes": (T + R) * D * (1 + 1 / 32) + 8 * T * k + 8 * E, "flops": 0}
        if op == "combine":
            return {"bytes": (T * k + T) * D * esz + 8 * T * k, "flops": 2 * T * k * D}
        return {"bytes": (T + T * k + R) * D * esz + 12 * T * k, "flops": 3 * T * k * D}
    wa, wb = (BITS[case["fmt_a"]] / 8 + 1 / 32), (BITS[case["fmt_b"]] / 8 + 1 / 32)
    if op == "experts":
        r, N, K = case["rows"], case["n"], case["k"]
        return {"bytes": r * K * wa + case["active"] * N * K * wb + 2 * r * N, "flops": 2 * r * N * K}
    r, M, N = case["rows"], case["m"], case["n"]
    return {"bytes": r * (M * wa + N * wb) + 2 * case["experts"] * M * N, "flops": 2 * r * M * N}


# ---------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------

def _round_to_grid(p, mbits, emin, top):
    """p on the element grid (ties to even, saturating), FP64."""
    e = torch.floor(torch.log2(p.abs().clamp(min=2.0 ** (emin - 60)))).clamp(min=emin)
    step = torch.exp2(e - mbits)
    return (torch.round(p / step) * step).clamp(-top, top)


def _decode64(codes, scales, rows, K, fmt):
    """FP64 values of an MX tensor, from the bit fields of its codes."""
    ebits, mbits = {"e4m3": (4, 3), "e5m2": (5, 2), "e2m1": (2, 1)}[fmt]
    c = torch.arange(1 << (1 + ebits + mbits), device=codes.device)
    man, ex = (c & ((1 << mbits) - 1)).double(), (c >> mbits) & ((1 << ebits) - 1)
    bias = (1 << (ebits - 1)) - 1
    mag = torch.where(ex == 0, man * 2.0 ** (1 - bias - mbits), (1 + man / (1 << mbits)) * torch.exp2(ex.double() - bias))
    table = torch.where(c >> (ebits + mbits) == 1, -mag, mag)
    flat = codes.view(rows, -1).int()
    if fmt == "e2m1":
        flat = torch.stack((flat % 16, flat // 16), 2).view(rows, K)
    r = torch.arange(rows, device=codes.device).unsqueeze(1)
    b = torch.arange(K // BLOCK, device=codes.device).unsqueeze(0)
    at = ((r // 128) * ((K // BLOCK + 3) // 4) + b // 4) * 512 + (r % 32) * 16 + ((r % 128) // 32) * 4 + b % 4
    x = torch.exp2(scales[at].double() - 127)
    return table[flat] * x.repeat_interleave(BLOCK, 1)


def _quantize64(y, fmt):
    rows, L = y.shape
    kb = (L + BLOCK - 1) // BLOCK
    v = torch.zeros((rows, kb * BLOCK), dtype=torch.float64, device=y.device)
    v[:, :L] = y
    v = v.view(rows, kb, BLOCK)
    shared = torch.floor(torch.log2(v.abs().amax(2))) - EMAX[fmt]
    shared = torch.nan_to_num(shared, neginf=-127.0).clamp(min=-127.0)
    mbits, emin = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    codes = _round_to_grid(v / torch.exp2(shared).unsqueeze(2), mbits, emin, MAXN[fmt])
    chunks = torch.full(((rows + 127) // 128 * ((kb + 3) // 4) * 512,), 2.0 ** -127, dtype=torch.float64, device=y.device)
    r = torch.arange(rows, device=y.device).unsqueeze(1)
    b = torch.arange(kb, device=y.device).unsqueeze(0)
    chunks[((r // 128) * ((kb + 3) // 4) + b // 4) * 512 + (r % 32) * 16 + ((r % 128) // 32) * 4 + b % 4] = torch.exp2(shared)
    return codes.reshape(-1), chunks


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm_grad"):
        x, w = s["x"].double(), s["w"].double()
        if op == "norm":
            if s["res"] is not None:
                x = x + s["res"].double()
            y = x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + EPS) * w
            codes, scales = _quantize64(y, case["fmt"])
            out = {"codes": codes, "scales": scales}
            if s["res"] is not None:
                out["h"] = x
            return out
        dy, n = s["dy"].double(), x.shape[1]
        inv = 1 / torch.sqrt((x * x).sum(1, keepdim=True) / n + EPS)
        dh = dy * w * inv - x * inv ** 3 * (dy * w * x).sum(1, keepdim=True) / n
        if s["res"] is not None:
            dh = dh + s["res"].double()
        return {"dh": dh, "dw": (dy * x * inv).sum(0)}
    if op == "route":
        x = s["logits"].double()
        p = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
        c = p + s["bias"].double() if s["bias"] is not None else p
        if case["groups"] > 1:
            v = c.view(x.shape[0], case["groups"], -1)
            gs = torch.topk(v, min(2, v.shape[2]), 2).values.sum(2) if case["score"] == "sigmoid" else v.max(2).values
            worst = torch.argsort(gs, dim=1, descending=True, stable=True)[:, case["topk_groups"]:]
            v = v.clone().scatter_(1, worst.unsqueeze(2).expand(-1, -1, v.shape[2]), -1e300)
            c = v.view(x.shape)
        sel = p.gather(1, torch.argsort(c, dim=1, descending=True, stable=True)[:, :case["topk"]])
        return {"ids": None, "weights": ROUTED_SCALE * sel / sel.sum(1, keepdim=True)}
    if op == "route_grad":
        with torch.enable_grad():
            x = s["logits"].double().requires_grad_(True)
            p = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
            sel = p.gather(1, s["ids"].long())
            loss = (ROUTED_SCALE * sel / sel.sum(1, keepdim=True) * s["dweights"].double()).sum()
            return {"dlogits": torch.autograd.grad(loss, x)[0]}
    if op == "dispatch":
        T, D, E, k, R = case["tokens"], case["dim"], case["experts"], s["topk"], s["rows"]
        codes = torch.zeros((R, D), dtype=torch.float64, device="cuda")
        exps = torch.zeros((R, D // BLOCK), dtype=torch.uint8, device="cuda")
        values, scales = s["elems"].view(T, D).view(torch.float8_e4m3fn).double(), _unswizzle(s["scales"], T, D // BLOCK)
        start = 0
        for e in range(E):
            tokens = (s["ids"] == e).any(1).nonzero()[:, 0]
            codes[start:start + len(tokens)] = values[tokens]
            exps[start:start + len(tokens)] = scales[tokens]
            start += -(-len(tokens) // case["align"]) * case["align"]
        return {"offsets": None, "row_of": None, "codes": codes.view(-1), "scales": torch.exp2(_swizzle(exps).double() - 127)}
    if op in ("combine", "combine_grad"):
        at, w, y = s["row_of"].long(), s["weights"].double(), s["y"]
        if op == "combine":
            out = torch.zeros((at.shape[0], y.shape[1]), dtype=torch.float64, device="cuda")
            for j in range(at.shape[1]):
                out += w[:, j:j + 1] * y[at[:, j]].double()
            return {"out": out}
        dout = s["dout"].double()
        dy = torch.zeros(y.shape, dtype=torch.float64, device="cuda")
        dw = torch.empty_like(w)
        for j in range(at.shape[1]):
            dy[at[:, j]] = w[:, j:j + 1] * dout
            dw[:, j] = (dout * y[at[:, j]].double()).sum(1)
        return {"dy": dy, "dw": dw}
    off, R = s["offsets"].tolist(), s["rows_padded"]
    if op == "experts":
        E, N, K = case["experts"], case["n"], case["k"]
        a = _decode64(s["a"], s["sa"], R, K, case["fmt_a"])
        b = _decode64(s["b"], s["sb"], E * N, K, case["fmt_b"]).view(E, N, K)
        rest = torch.zeros((R - off[-1], N), dtype=torch.float64, device="cuda")
        return {"c": torch.cat([a[off[e]:off[e + 1]] @ b[e].T for e in range(E)] + [rest])}
    a = _decode64(s["a"], s["sa"], case["m"], R, case["fmt_a"])
    b = _decode64(s["b"], s["sb"], case["n"], R, case["fmt_b"])
    return {"c": torch.stack([a[:, off[e]:off[e + 1]] @ b[:, off[e]:off[e + 1]].T for e in range(case["experts"])])}
