"""Cases of the paged key-value cache in MX format: rows quantized as they are written, read back, and the
attention of one new token (or a few drafted ones) of every sequence over its cached tokens.

`own` false: every operator in elementary torch operations in FP32.  `own` true: the calls a user makes of the
library.  Sizes are generic: heads of 64 to 256 elements, pages of 16 to 128 tokens, 1 to 64 sequences of up to
131072 tokens."""
import math

import torch

own = False

BLOCK = 32
EMAX = {"e4m3": 8, "e5m2": 15, "e2m1": 2, "int8": 0}
MAXN = {"e4m3": 448.0, "e5m2": 57344.0, "e2m1": 6.0, "int8": 127.0 / 64.0}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "int8": torch.int8}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BITS = {"e4m3": 8, "e5m2": 8, "e2m1": 4, "int8": 8}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # one decoding step of 64 sequences writes its tokens; a few microseconds
        {"name": "append_decode", "op": "append", "tokens": 64, "skipped": 0, "heads": 8, "dim": 128, "page": 64, "fmt": "e4m3",
         "dtype": "bf16", "fused": True},
        # a prompt of 8192 tokens, rows inside the fused projection's output
        {"name": "append_prompt", "op": "append", "tokens": 8192, "skipped": 0, "heads": 8, "dim": 128, "page": 64, "fmt": "e4m3",
         "dtype": "bf16", "fused": True},
        # a padded batch: some tokens have no slot; odd counts, FP32
        {"name": "append_padded", "op": "append", "tokens": 1000, "skipped": 37, "heads": 5, "dim": 96, "page": 24, "fmt": "e5m2",
         "dtype": "f32", "fused": False},
        # a cached prefix of 16384 tokens for a prompt that continues it
        {"name": "read_prefix", "op": "read", "tokens": 16384, "heads": 8, "dim": 128, "page": 64, "fmt": "e4m3", "dtype": "bf16"},
        # a short one out of a 4-bit cache, in FP32
        {"name": "read_short", "op": "read", "tokens": 1003, "heads": 4, "dim": 64, "page": 16, "fmt": "e2m1", "dtype": "f32"},
        # one sequence at its start: latency
        {"name": "attend_first", "op": "attend", "batch": 1, "longest": 333, "heads": 2, "group": 4, "dim": 128, "page": 16, "new": 1,
         "window": 0, "fmt": "e4m3", "dtype": "bf16"},
        # a decoding step of 64 sequences of all lengths up to 8192
        {"name": "attend_batch", "op": "attend", "batch": 64, "longest": 8192, "heads": 8, "group": 4, "dim": 128, "page": 64, "new": 1,
         "window": 0, "fmt": "e4m3", "dtype": "bf16"},
        # one sequence of 131072 tokens: the work of a few rows, split over the length
        {"name": "attend_long", "op": "attend", "batch": 1, "longest": 131072, "heads": 8, "group": 8, "dim": 128, "page": 64, "new": 1,
         "window": 0, "fmt": "e4m3", "dtype": "bf16"},
        # a 4-bit cache
        {"name": "attend_fp4", "op": "attend", "batch": 32, "longest": 12000, "heads": 8, "group": 8, "dim": 128, "page": 32, "new": 1,
         "window": 0, "fmt": "e2m1", "dtype": "bf16"},
        # a key-value head for every query head, short rows
        {"name": "attend_single", "op": "attend", "batch": 16, "longest": 4096, "heads": 16, "group": 1, "dim": 64, "page": 128, "new": 1,
         "window": 0, "fmt": "e5m2", "dtype": "bf16"},
        # four drafted tokens to verify, a sliding window that starts inside a page
        {"name": "attend_drafts", "op": "attend", "batch": 32, "longest": 5000, "heads": 8, "group": 4, "dim": 128, "page": 16, "new": 4,
         "window": 1024, "fmt": "e4m3", "dtype": "bf16"},
        # FP32 queries and results, long rows of 8-bit integers, odd lengths
        {"name": "attend_f32", "op": "attend", "batch": 8, "longest": 2001, "heads": 4, "group": 4, "dim": 256, "page": 24, "new": 1,
         "window": 0, "fmt": "int8", "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend", "attend"])
    c = {"op": op, "dim": rng.choice([64, 96, 128, 128, 192, 256]), "page": rng.choice([16, 24, 32, 64, 128]),
         "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"])}
    if op != "attend":
        c["heads"] = rng.choice([1, 2, 5, 8])
        c["tokens"] = min(_log(rng, 16, 16384 if op == "read" else 8192), 16384 * 1024 // (c["heads"] * c["dim"]))
        c["fmt"] = rng.choice(["e4m3", "e4m3", "e5m2", "int8"] + (["e2m1"] if op == "read" else []))
        if op == "append":
            c["skipped"] = rng.choice([0, 0, c["tokens"] // 9])
            c["fused"] = rng.random() < 0.5
        return c
    c["fmt"] = rng.choice(["e4m3", "e4m3", "e5m2", "int8", "e2m1"])
    c["heads"] = rng.choice([1, 2, 4, 5, 8, 16])
    c["group"] = rng.choice([1, 2, 4, 5, 7, 8, 16])
    c["new"] = rng.choice([1, 1, 1, 2, 5])
    c["batch"] = _log(rng, 1, 64)
    most = 200_000_000 // (c["batch"] * c["heads"] * c["dim"])
    c["longest"] = _log(rng, 64, max(64, min(65536, most)))
    c["window"] = rng.choice([0, 0, 0, _log(rng, 33, 4096)])
    return c


# ---------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _encode(x, fmt):
    """Algorithm 1 along the last axis [..., dim] FP32: element values P as codes (one byte each, E2M1 two per byte)
    and scale bytes [..., blocks padded to whole words]."""
    shape = x.shape
    v = x.reshape(*shape[:-1], -1, BLOCK)
    amax = v.abs().amax(-1)
    byte = (torch.frexp(amax)[1] - 1 - EMAX[fmt] + 127).clamp(0, 254)
    byte = torch.where(amax >= 2.0 ** -126, byte, torch.zeros_like(byte))
    p = torch.ldexp(v, (127 - byte).unsqueeze(-1)).reshape(shape).clamp(-MAXN[fmt], MAXN[fmt])
    if fmt == "e2m1":
        grid = torch.tensor(E2M1, device=x.device)
        code = torch.bucketize(p.abs(), (grid[1:] + grid[:-1]) / 2).to(torch.uint8) | ((p < 0).to(torch.uint8) << 3)
        codes = code[..., 0::2] | (code[..., 1::2] << 4)
    elif fmt == "int8":
        codes = torch.round(p * 64).to(torch.int8).view(torch.uint8)
    else:
        codes = p.to(F8[fmt]).view(torch.uint8)
    byte = byte.to(torch.uint8)
    return codes.contiguous(), torch.nn.functional.pad(byte, (0, -byte.shape[-1] % 4))


def _lengths(case):
    """Cached tokens of each sequence, the new ones counted: between an eighth of the longest and the longest."""
    n = case["longest"]
    return [max(1, n - int((i * 0.6180339887) % 1.0 * 0.875 * n)) for i in range(case["batch"])]


def prepare(case, seed):
    g = _rng(seed)
    dev = "cuda"
    randn = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    s = dict(case)
    op, H, D, ps, fmt = case["op"], case["heads"], case["dim"], case["page"], case["fmt"]
    dt = DT[case["dtype"]]
    if op == "append":
        T = case["tokens"]
        pages = -(-T // ps) + 3
        width = (D * BITS[fmt]) // 8
        # what earlier tokens left in the cache
        s["ke"], s["ve"] = (torch.randint(0, 0x70, (pages, H, ps, width), generator=g, device=dev, dtype=torch.uint8) for _ in range(2))
        s["ks"], s["vs"] = (torch.randint(110, 130, (pages, H, ps, -(-D // 128) * 4), generator=g, device=dev, dtype=torch.uint8)
                            for _ in range(2))
        rows = randn(T, (4 if case["fused"] else 2) * H * D) * torch.exp(0.5 * randn((4 if case["fused"] else 2) * H * D))
        rows = rows.to(dt)
        # keys and values lie behind the queries in the projection's output
        k, v = rows[:, -2 * H * D:-H * D], rows[:, -H * D:]
        s["k"], s["v"] = (t.view(T, H, D) if case["fused"] else t.contiguous().view(T, H, D) for t in (k, v))
        slots = torch.randperm(pages, generator=g, device=dev).repeat_interleave(ps) * ps + torch.arange(pages * ps, device=dev) % ps
        slots = slots[:T].to(torch.int32)
        slots[torch.randperm(T, generator=g, device=dev)[:case["skipped"]]] = -1
        s["slots"] = slots
        return s
    lengths = [case["tokens"]] if op == "read" else _lengths(case)
    per = [-(-n // ps) for n in lengths]
    pages, most = sum(per) + 2, max(per)
    gain = torch.exp(0.5 * randn(H, 1, D))  # some channels of the keys are large
    s["ke"], s["ks"] = _encode(randn(pages, H, ps, D) * gain, fmt)
    s["ve"], s["vs"] = _encode(randn(pages, H, ps, D) * torch.exp(0.5 * randn(pages, 1, ps, 1)), fmt)
    order = torch.randperm(pages, generator=g, device=dev)
    if op == "read":
        slots = order.repeat_interleave(ps) * ps + torch.arange(pages * ps, device=dev) % ps
        s["slots"] = slots[:case["tokens"]].to(torch.int32)
        return s
    B, T, G = case["batch"], case["new"], case["group"]
    lens = torch.tensor(lengths, device=dev)[torch.randperm(B, generator=g, device=dev)]
    need = (lens + ps - 1) // ps
    first = need.cumsum(0) - need
    at = torch.arange(most, device=dev)
    s["table"] = torch.where(at < need[:, None], order[(first[:, None] + at).clamp(max=pages - 1)], -1).to(torch.int32)
    s["lengths"] = lens.to(torch.int32)
    s["scale"] = D ** -0.5
    s["q"] = (1.2 * randn(B, T, H, G, D) / gain.view(H, 1, D)).view(B, T, H * G, D).to(dt)
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


def _cache_values(s):
    """The cache as outputs: the values its codes and scales stand for."""
    f = F8[s["fmt"]]
    return {"k": s["ke"].view(f), "ks": s["ks"].view(torch.float8_e8m0fnu), "v": s["ve"].view(f), "vs": s["vs"].view(torch.float8_e8m0fnu)}


def _run_own(s):
    mx = _lib()
    cache = mx.KvCache(s["ke"], s["ks"], s["ve"], s["vs"], s["dim"], mx.FORMATS[s["fmt"]])
    if s["op"] == "append":
        mx.mx_kv_append(cache, s["k"], s["v"], s["slots"])
        return _cache_values(s)
    if s["op"] == "read":
        k, v = mx.mx_kv_read(cache, s["slots"], DT[s["dtype"]])
        return {"k": k, "v": v}
    out, lse = mx.mx_kv_attention(s["q"], cache, s["table"], s["lengths"], s["scale"], window=s["window"], return_lse=True)
    return {"out": out, "lse": lse}


def _decode(codes, scales, fmt):
    """FP32 values of rows of codes with their scale bytes."""
    if fmt == "e2m1":
        grid = torch.tensor(E2M1 + [-v for v in E2M1], device=codes.device)
        p = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).flatten(-2)
    elif fmt == "int8":
        p = codes.view(torch.int8).float() / 64
    else:
        p = codes.view(F8[fmt]).float()
    blocks = p.shape[-1] // BLOCK
    x = torch.exp2(scales[..., :blocks].float() - 127.0)
    return (p.unflatten(-1, (blocks, BLOCK)) * x.unsqueeze(-1)).flatten(-2)


def _run_plain(s):
    fmt, ps, H, D = s["fmt"], s["page"], s["heads"], s["dim"]
    if s["op"] == "append":
        slots = s["slots"].long()
        # a token without a slot repeats the first one that has one
        has = slots >= 0
        src = torch.where(has, torch.arange(len(slots), device=slots.device), torch.argmax(has.to(torch.uint8)))
        page, off = slots[src] // ps, slots[src] % ps
        for x, codes, scales in ((s["k"], s["ke"], s["ks"]), (s["v"], s["ve"], s["vs"])):
            c, b = _encode(x[src].float(), fmt)
            codes[page, :, off] = c
            scales[page, :, off] = b
        return _cache_values(s)
    if s["op"] == "read":
        page, off = s["slots"].long() // ps, s["slots"].long() % ps
        get = lambda c, b: _decode(c[page, :, off], b[page, :, off], fmt).to(DT[s["dtype"]])  # noqa: E731
        return {"k": get(s["ke"], s["ks"]), "v": get(s["ve"], s["vs"])}
    B, T, G = s["batch"], s["new"], s["group"]
    table, lens = s["table"].long(), s["lengths"].long()
    L = table.shape[1] * ps
    at = table.clamp(min=0)
    get = lambda c, b: _decode(c[at], b[at], fmt).transpose(1, 2).reshape(B, H, L, D)  # noqa: E731
    k, v = get(s["ke"], s["ks"]), get(s["ve"], s["vs"])
    q = s["q"].float().view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    sc = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    j = torch.arange(L, device=table.device)
    end = (lens[:, None] - T + 1 + torch.arange(T, device=table.device))[:, :, None]
    seen = (j < end) & (table >= 0).repeat_interleave(ps, 1)[:, None, :]
    if s["window"]:
        seen = seen & (j >= end - s["window"])
    seen = seen.repeat_interleave(G, 1)[:, None]
    sc = torch.where(seen, sc, torch.full_like(sc, -math.inf))
    top = sc.amax(3, keepdim=True)
    some = top > -math.inf
    e = torch.exp(sc - torch.where(some, top, torch.zeros_like(top)))
    total = e.sum(3, keepdim=True)
    out = torch.where(some, torch.matmul(e, v) / total, torch.zeros_like(top))
    lse = (top + torch.log(total)).squeeze(3)
    back = lambda t: t.unflatten(2, (T, G)).transpose(1, 2).flatten(2, 3)  # noqa: E731
    return {"out": back(out).to(s["q"].dtype).contiguous(), "lse": back(lse).contiguous()}


# ---------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------

def work(case):
    esz = {"bf16": 2, "f32": 4}[case["dtype"]]
    row = 2 * case["heads"] * case["dim"]  # a token's keys and values
    mx = BITS[case["fmt"]] / 8 + 1 / 32
    if case["op"] == "append":
        n = case["tokens"] - case["skipped"]
        return {"bytes": n * row * (esz + mx) + 4 * case["tokens"], "flops": 3 * n * row}
    if case["op"] == "read":
        return {"bytes": case["tokens"] * (row * (esz + mx) + 4), "flops": case["tokens"] * row}
    T, w = case["new"], case["window"]
    read = sum(min(n, w + T - 1) if w else n for n in _lengths(case))
    seen = sum(max(0, min(n - i, w) if w else n - i) for n in _lengths(case) for i in range(T))
    heads = case["heads"] * case["group"]
    return {"bytes": read * row * mx + 2 * case["batch"] * T * heads * case["dim"] * esz, "flops": 4 * seen * heads * case["dim"]}


# ---------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------

def _value_table(fmt):
    """What each code stands for, FP64, from its bit fields."""
    if fmt == "int8":
        n = torch.arange(256, device="cuda", dtype=torch.float64)
        return torch.where(n < 128, n, n - 256) / 64
    ebits, mbits = {"e4m3": (4, 3), "e5m2": (5, 2), "e2m1": (2, 1)}[fmt]
    c = torch.arange(1 << (1 + ebits + mbits), device="cuda")
    man, ex = (c & ((1 << mbits) - 1)).double(), (c >> mbits) & ((1 << ebits) - 1)
    bias = (1 << (ebits - 1)) - 1
    mag = torch.where(ex == 0, man * 2.0 ** (1 - bias - mbits), (1 + man / (1 << mbits)) * torch.exp2(ex.double() - bias))
    return torch.where(c >> (ebits + mbits) == 1, -mag, mag)


def _values64(codes, scales, fmt):
    flat = codes.int()
    if fmt == "e2m1":
        flat = torch.stack((flat % 16, flat // 16), -1).reshape(*codes.shape[:-1], -1)
    p = _value_table(fmt)[flat.long()]
    return p * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)[..., :p.shape[-1]]


def _quantized64(x, fmt):
    """Element and scale values of Algorithm 1, FP64."""
    v = x.double().unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1)
    shared = torch.where(amax < 2.0 ** -126, -127.0, torch.frexp(amax)[1].double() - 1 - EMAX[fmt]).clamp(min=-127.0)
    p = v / torch.exp2(shared).unsqueeze(-1)
    if fmt == "int8":
        return torch.round(p * 64).clamp(-127, 127).flatten(-2), torch.exp2(shared)
    mbits, emin = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    step = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** (emin - 60)))).clamp(min=emin) - mbits)
    return (torch.round(p / step) * step).clamp(-MAXN[fmt], MAXN[fmt]).flatten(-2), torch.exp2(shared)


def exact(case, seed):
    s = prepare(case, seed)
    op, fmt, ps, H, D = case["op"], case["fmt"], case["page"], case["heads"], case["dim"]
    if op == "append":
        out = {}
        slots = s["slots"].long()
        which = (slots >= 0).nonzero()[:, 0]
        page, off = slots[which] // ps, slots[which] % ps
        for name, x, codes, scales in (("k", s["k"], s["ke"], s["ks"]), ("v", s["v"], s["ve"], s["vs"])):
            p, b = _quantized64(x[which], fmt)
            values = codes.view(torch.int8).double() if fmt == "int8" else _value_table(fmt)[codes.long()]
            values[page, :, off] = p
            full = torch.exp2(scales.double() - 127)
            full[page, :, off] = torch.nn.functional.pad(b, (0, full.shape[3] - b.shape[2]), value=2.0 ** -127)
            out[name] = None if fmt == "int8" else values
            out[name + "s"] = full
        return out
    if op == "read":
        tokens = lambda t: t.transpose(1, 2).flatten(0, 1)[s["slots"].long()]  # noqa: E731
        return {name: _values64(tokens(codes), tokens(scales), fmt) for name, codes, scales in (("k", s["ke"], s["ks"]), ("v", s["ve"], s["vs"]))}
    T, G, w = case["new"], case["group"], case["window"]
    outs, lses = [], []
    for b, n in enumerate(s["lengths"].tolist()):
        pages = s["table"][b, :-(-n // ps)].long()
        k = _values64(s["ke"][pages], s["ks"][pages], fmt).transpose(0, 1).reshape(H, -1, D)[:, :n]
        v = _values64(s["ve"][pages], s["vs"][pages], fmt).transpose(0, 1).reshape(H, -1, D)[:, :n]
        for i in range(T):
            hi = n - (T - 1 - i)
            lo = max(0, hi - w) if w else 0
            if hi <= lo:
                outs.append(torch.zeros((H * G, D), dtype=torch.float64, device="cuda"))
                lses.append(torch.full((H * G,), -math.inf, dtype=torch.float64, device="cuda"))
                continue
            logits = torch.einsum("hgd,hnd->hgn", s["q"][b, i].double().view(H, G, D), k[:, lo:hi]) * s["scale"]
            outs.append(torch.einsum("hgn,hnd->hgd", torch.softmax(logits, 2), v[:, lo:hi]).reshape(H * G, D))
            lses.append(torch.logsumexp(logits, 2).reshape(H * G))
    B = case["batch"]
    return {"out": torch.stack(outs).view(B, T, H * G, D), "lse": torch.stack(lses).view(B, T, H * G)}
