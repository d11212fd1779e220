"""A paged cache for the tests: built from random codes and scales, and its definition in 64 bits."""
import math

import numpy as np
import torch

import paper_2310_10537_b200 as mx

FMT_NAME = {mx.MX_E4M3: (4, 3), mx.MX_E5M2: (5, 2), mx.MX_E2M1: (2, 1)}


def code_values(fmt):
    """Value of every code, FP64 (NaN / Inf codes of the FP8 formats as such)."""
    if fmt == mx.MX_INT8:
        n = np.arange(256, dtype=np.float64)
        return np.where(n < 128, n, n - 256) / 64
    e, m = FMT_NAME[fmt]
    c = np.arange(1 << (1 + e + m))
    man, ex = c & ((1 << m) - 1), (c >> m) & ((1 << e) - 1)
    bias = (1 << (e - 1)) - 1
    mag = np.where(ex == 0, man * 2.0 ** (1 - bias - m), (1 + man / (1 << m)) * 2.0 ** (ex - bias))
    if fmt == mx.MX_E4M3:
        mag = np.where((c & 0x7F) == 0x7F, np.nan, mag)
    if fmt == mx.MX_E5M2:
        mag = np.where(ex == 31, np.where(man == 0, np.inf, np.nan), mag)
    return np.where(c >> (e + m) == 1, -mag, mag)


def values(codes, scales, dim, fmt):
    """FP64 values [.., dim] of rows of codes and scale bytes (torch, any device)."""
    table = torch.from_numpy(code_values(fmt)).to(codes.device)
    if fmt == mx.MX_E2M1:
        codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    x = torch.where(scales == 255, torch.full((), math.nan, dtype=torch.float64, device=codes.device), torch.exp2(scales.double() - 127))
    return table[codes.long()] * x[..., :dim // 32].repeat_interleave(32, -1)


def random_cache(pages, page_size, heads, dim, fmt, g, spread=4, middle=None):
    """Codes over the whole format but its NaN and Inf; scale exponents within `spread` of `middle` (default: values
    of about 1)."""
    c = mx.mx_kv_cache(pages, page_size, heads, dim, fmt)
    middle = 127 - {mx.MX_E4M3: 7, mx.MX_E5M2: 13, mx.MX_E2M1: 1, mx.MX_INT8: 0}[fmt] if middle is None else middle
    for codes, scales in ((c.k_elems, c.k_scales), (c.v_elems, c.v_scales)):
        if fmt in (mx.MX_E4M3, mx.MX_E5M2):
            top = 0x7E if fmt == mx.MX_E4M3 else 0x7B
            r = torch.randint(0, top + 1, codes.shape, generator=g, device="cuda") + 128 * torch.randint(0, 2, codes.shape, generator=g, device="cuda")
        else:
            r = torch.randint(0, 256, codes.shape, generator=g, device="cuda")
        codes.copy_(r.to(torch.uint8))
        s = torch.randint(middle - spread, middle + spread + 1, scales.shape, generator=g, device="cuda").clamp(0, 254)
        s[..., dim // 32:] = 0
        scales.copy_(s.to(torch.uint8))
    return c


def attention64(q, cache, table, lengths, scale, window):
    """out, lse in FP64, and what the error bounds are made of: sum p |v|, the largest sum |q||k| scale (with
    2^-9 of max |q| sum |k| scale), and per block what FP16's smallest steps are relative to (see bounds)."""
    pages, heads, ps, _ = cache.k_elems.shape
    B, T, Hq, D = q.shape
    G = Hq // heads
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=q.device)
    absv, least = torch.zeros_like(out), torch.zeros_like(out)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(lse)
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * ps)
        j = torch.arange(n, device=q.device)
        page = table[b, j // ps].long() if n else j
        ok = (page >= 0) & (page < pages)
        for i in range(T):
            e = n - (T - 1 - i)
            see = ok & (j < e) & (j >= (e - window if window else 0))
            jj = j[see]
            if not len(jj):
                continue
            p, o = page[see], jj % ps
            k = values(cache.k_elems[p, :, o], cache.k_scales[p, :, o], D, cache.fmt)  # [n, heads, D]
            v = values(cache.v_elems[p, :, o], cache.v_scales[p, :, o], D, cache.fmt)
            x = q[b, i].double().view(heads, G, D)
            s = torch.einsum("hgd,nhd->hgn", x, k) * scale
            w = torch.softmax(s, 2)
            out[b, i] = torch.einsum("hgn,nhd->hgd", w, v).reshape(Hq, D)
            x_v = torch.exp2(cache.v_scales[p, :, o].double() - 127)[..., :D // 32]      # [n, heads, blocks]
            peak = (w.unsqueeze(3) * x_v.permute(1, 0, 2).unsqueeze(1)).amax(2)           # largest weight times scale [h, g, blocks]
            codes = (v / x_v.repeat_interleave(32, -1)).abs().sum(0)                      # sum of the elements [h, d]
            small = peak.repeat_interleave(32, -1) * codes.unsqueeze(1)
            absv[b, i] = torch.einsum("hgn,nhd->hgd", w, v.abs()).reshape(Hq, D)
            least[b, i] = small.reshape(Hq, D)
            lse[b, i] = torch.logsumexp(s, 2).reshape(Hq)
            size[b, i] = (torch.einsum("hgd,nhd->hgn", x.abs() + 2.0 ** -9 * x.abs().amax(2, keepdim=True), k.abs()) * abs(scale)).amax(2).reshape(Hq)
    return out, lse, absv, size, least


def bounds(dtype, want, absv, size, least, dim, tokens):
    """How far out and lse may be from the definition.

    Scores: `dim` products, exact in FP32, and their sum, scale and subtraction of the maximum: each step off by at
    most 2^-23 of sum |q||k| scale (the tensor core's additions may truncate), in all (dim + 16) 2^-23 size for the
    score in units of e.  A weight is off by that and by 2^-21 (the exponential), for its use in the products by half a step of FP16
    (BF16 results) or of two FP16 terms, 2^-22 (FP32).  The weights' sum and the sums over tokens add at most 2^-23 of sum p |v| for each 16 tokens and 64 more
    for the joins.  The result is rounded once.

    FP16 has steps of 2^-24 below 2^-14.  Queries enter with their largest element in [2^7, 2^8): smaller ones are off by at most
    2^-25 / 2^7 = 2^-32 of it, which in 2^-23 times `size` is 2^-9 max |q| sum |k|.  Weights w = p X F, X the value's block scale and
    p = e^(s - m) enter with a row's largest of a block in [2^12, 2^15]: F >= 2^12 / max p X, and each is off by at most
    2^-25 / F <= 2^-37 max p X, times the element P that it multiplies, divided by the sum of p.  Over tokens that is 2^-37 of `least`,
    the largest softmax weight times X, times the sum of |P|.
    (Both matter where a large weight meets a tiny element of its block and a tiny weight a large one.)"""
    u = 2.0 ** -23
    score = (dim + 16) * u * size.unsqueeze(3)
    half = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
    rel = 2 * score + 2.0 ** -20 + half + 2 * (tokens / 16 + 64) * u
    out = absv * rel + 2.0 ** -37 * least + want.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)
    lse = score.squeeze(3) + 2.0 ** -20 + (tokens / 16 + 64) * u
    return out + 1e-38, lse
