"""A mixture-of-experts block of a transformer on MX operands, forward and backward.

    h = x + residual;  y = norm(h);  route y;  out[t] = sum_j w[t, j] * down_e(silu(gate_e y) * up_e y)

Every matrix product but the small routing one runs on MX tensors that are quantized right before it: the
norm hands its result out in MX form, the gather moves those rows to their experts without requantizing, and
each product's gradients use the same tensors quantized along the axis that they reduce over.

Run `python examples/moe_block.py` on a B200: it compares a step with FP32 PyTorch and times it."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_10537_b200 as mx  # noqa: E402


class MoeBlock:
    def __init__(self, dim, ffn, experts, topk, fmt=mx.MX_E4M3, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.dim, self.ffn, self.experts, self.topk, self.fmt, self.eps = dim, ffn, experts, topk, fmt, 1e-6
        self.norm = (1 + 0.1 * randn(dim)).bfloat16()
        self.router = (randn(experts, dim) * dim ** -0.5).bfloat16()
        self.bias = torch.zeros(experts, device="cuda")               # moved by a load balancer, not by gradients
        self.up = (randn(experts, 2 * ffn, dim) * dim ** -0.5).bfloat16()   # gate rows, then up rows
        self.down = (randn(experts, dim, ffn) * ffn ** -0.5).bfloat16()
        self.quantize_weights()

    def quantize_weights(self):
        """Both MX forms of the experts' weights: along the input for the forward product, along the
        output for the gradient of its input.  Once per optimizer step."""
        self.up_q, self.up_t = (mx.mx_quantize(self.up, a, self.fmt) for a in (2, 1))
        self.down_q, self.down_t = (mx.mx_quantize(self.down, a, self.fmt) for a in (2, 1))

    def forward(self, x, residual):
        D, F, fmt = self.dim, self.ffn, self.fmt
        s = {"y": torch.empty_like(x)}
        e, sc, s["h"] = mx.mx_rmsnorm_quantize(x, self.norm, fmt, self.eps, residual=residual, y_out=s["y"])
        s["logits"] = s["y"] @ self.router.T
        s["ids"], s["w"] = mx.mx_route(s["logits"], self.topk, mx.MX_SCORE_SIGMOID, bias=self.bias)
        s["plan"] = p = mx.mx_moe_plan(s["ids"], self.experts, align=128)
        xe, xs = mx.mx_moe_gather(e, sc, D, fmt, p)
        s["u"] = mx.mx_gemm_grouped(xe, xs, *self.up_q, p.offsets, p.rows, 2 * F, D, fmt, fmt, out_dtype=torch.bfloat16)
        gate, up = s["u"].float().chunk(2, 1)
        s["a"] = (torch.nn.functional.silu(gate) * up).bfloat16()
        ae, asc = mx.mx_quantize(s["a"], 1, fmt)
        s["z"] = mx.mx_gemm_grouped(ae, asc, *self.down_q, p.offsets, p.rows, D, F, fmt, fmt, out_dtype=torch.bfloat16)
        return mx.mx_moe_combine(s["z"], s["w"], p), s

    def backward(self, dout, dh, s):
        """Gradients for the output's `dout` and the residual stream's `dh`."""
        D, F, fmt, p = self.dim, self.ffn, self.fmt, s["plan"]
        q = lambda t, axis: mx.mx_quantize(t, axis, fmt)  # noqa: E731
        dz, dw = mx.mx_moe_combine_backward(dout, s["z"], s["w"], p)
        da = mx.mx_gemm_grouped(*q(dz, 1), *self.down_t, p.offsets, p.rows, F, D, fmt, fmt, out_dtype=torch.bfloat16).float()
        ddown = mx.mx_gemm_grouped_k(*q(dz, 0), *q(s["a"], 0), p.offsets, D, F, p.rows, fmt, fmt)
        gate, up = s["u"].float().chunk(2, 1)
        sg = torch.sigmoid(gate)
        du = torch.cat([da * up * sg * (1 + gate * (1 - sg)), da * gate * sg], 1).bfloat16()
        dxp = mx.mx_gemm_grouped(*q(du, 1), *self.up_t, p.offsets, p.rows, D, 2 * F, fmt, fmt, out_dtype=torch.bfloat16)
        xp, _ = mx.mx_moe_combine_backward(s["y"], None, None, p)     # the float rows in expert order
        dup = mx.mx_gemm_grouped_k(*q(du, 0), *q(xp, 0), p.offsets, 2 * F, D, p.rows, fmt, fmt)
        dlogits = mx.mx_route_backward(dw, s["logits"], s["ids"], mx.MX_SCORE_SIGMOID)
        dy = mx.mx_moe_combine(dxp, None, p) + dlogits @ self.router
        dx, dnorm = mx.mx_rmsnorm_backward(dy, s["h"], self.norm, self.eps, dres=dh)
        return {"x": dx, "norm": dnorm, "router": dlogits.T @ s["y"], "up": dup, "down": ddown}


def reference(block, x, residual, ids, dout, dh):
    """The same step in FP32 PyTorch, the choice of experts given."""
    leaf = lambda t: t.float().detach().requires_grad_(True)  # noqa: E731
    p = {"x": leaf(x), "norm": leaf(block.norm), "router": leaf(block.router), "up": leaf(block.up), "down": leaf(block.down)}
    h = p["x"] + residual.float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + block.eps) * p["norm"]
    s = torch.sigmoid(y @ p["router"].T).gather(1, ids.long())
    w = s / s.sum(1, keepdim=True)
    out = torch.zeros_like(h)
    for e in range(block.experts):
        t, j = (ids == e).nonzero(as_tuple=True)
        gate, up = (y[t] @ p["up"][e].T).chunk(2, 1)
        z = (torch.nn.functional.silu(gate) * up) @ p["down"][e].T
        out = out.index_add(0, t, z * w[t, j].unsqueeze(1))
    grads = torch.autograd.grad((out * dout.float()).sum() + (h * dh.float()).sum(), list(p.values()))
    return out.detach(), dict(zip(p, grads))


def compare(tokens=512, dim=512, ffn=384, experts=8, topk=2, seed=1):
    """Relative 2-norm errors of a step's results against FP32."""
    block = MoeBlock(dim, ffn, experts, topk, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x, res, dout, dh = (torch.randn(tokens, dim, generator=g, device="cuda").bfloat16() for _ in range(4))
    out, saved = block.forward(x, res)
    grads = block.backward(dout, dh, saved)
    want, wgrads = reference(block, x, res, saved["ids"], dout, dh)
    rel = lambda a, b: float((a.float() - b.float()).norm() / b.float().norm())  # noqa: E731
    return {"out": rel(out, want), **{k: rel(grads[k], wgrads[k]) for k in grads}}


def main():
    for name, err in compare().items():
        print(f"{name:8s} relative error against FP32: {err:.4f}")
    tokens, dim = 8192, 4096
    block = MoeBlock(dim, 2048, 32, 4)
    x, res, dout, dh = (torch.randn(tokens, dim, device="cuda").bfloat16() for _ in range(4))
    for what, f in (("forward", lambda: block.forward(x, res)),
                    ("forward and backward", lambda: block.backward(dout, dh, block.forward(x, res)[1]))):
        for _ in range(3):
            f()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(10):
            f()
        b.record()
        torch.cuda.synchronize()
        print(f"{what}: {a.elapsed_time(b) / 10:.3f} ms for {tokens} tokens of {dim}, 4 of 32 experts of 2048")


if __name__ == "__main__":
    main()
