"""Requests with adapters of their own through a layer on frozen 4-bit weights, served and trained, with the operators of qmm.py.

  serving   rms_norm (residual added) -> mx_linear, with lora beside it for each row's adapter -> rms_norm -> router logits ->
            expert_route (sigmoid scores, balance bias, groups) -> mx_moe
  training  the adapters, the norm's weight and the router around the frozen projection: rms_norm_rows keeps x in 8 bits for the adapters' gradient, and
            lora_grad, rms_norm_grad and expert_route_grad are a torch.autograd.Function's backward pass each

Run on a B200:  python examples/adapted_layer.py [--tokens 64]
It prints how far the served layer is from the same layer in fp32, and the gradients from torch's own.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_00501_b200 import qmm  # noqa: E402

EPS = 1e-6


class Norm(torch.autograd.Function):
    """(x, residual, weight) -> (codes' values as x's type, h, codes, scales): the rows that the adapters read are kept in 8 bits."""

    @staticmethod
    def forward(ctx, x, residual, weight):
        y = torch.empty_like(x)
        codes, scales, h = qmm.rms_norm_rows(x, weight, EPS, residual=residual, y=y)
        ctx.save_for_backward(h, weight)
        ctx.mark_non_differentiable(codes, scales)
        return y, h, codes, scales

    @staticmethod
    def backward(ctx, dy, dh, _codes, _scales):
        h, weight = ctx.saved_tensors
        dx, dweight = qmm.rms_norm_grad(dy.contiguous(), h, weight, EPS, dh=dh.contiguous())
        return dx, dx, dweight.to(weight.dtype)


class Adapted(torch.autograd.Function):
    """y0 + scale * B A x of each row's adapter; y0 comes from the frozen projection w (dense here for its gradient), x8 is what is kept of x."""

    @staticmethod
    def forward(ctx, x, y0, a, b, idx, scale, codes, scales, w):
        s = torch.empty(x.shape[0], a.shape[1], device=x.device)
        y = qmm.lora(codes, idx, a, b, y0, scale=scale, x_scale=scales, s=s)
        ctx.save_for_backward(codes, scales, s, a, b, idx, scale, w)
        return y

    @staticmethod
    def backward(ctx, dy):
        codes, scales, s, a, b, idx, scale, w = ctx.saved_tensors
        dy = dy.contiguous()
        dx, da, db = qmm.lora_grad(dy, codes, s, idx, a, b, dy @ w, scale=scale, x_scale=scales)
        return dx, None, da.to(a.dtype), db.to(b.dtype), None, None, None, None, None


class Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, topk, bias):
        idx, weights = qmm.expert_route(logits, topk, qmm.SIGMOID, bias=bias, groups=4, top_groups=2, group_top=2)
        ctx.save_for_backward(logits, idx)
        ctx.mark_non_differentiable(idx)
        return idx, weights

    @staticmethod
    def backward(ctx, _idx, dweights):
        logits, idx = ctx.saved_tensors
        return qmm.expert_route_grad(dweights.contiguous(), logits, idx, qmm.SIGMOID), None, None


def adapters(n, r, K, N, dtype, gen):
    a = (torch.randn(n, r, K, generator=gen, device="cuda") * K**-0.5).to(dtype)
    return a, (torch.randn(n, N, r, generator=gen, device="cuda") * 0.1).to(dtype), torch.full((n,), 16.0 / r, device="cuda")


def lora_in_fp32(x, idx, a, b, scale):
    out = torch.zeros(x.shape[0], b.shape[1], device=x.device)
    for e in range(a.shape[0]):
        t = idx == e
        out[t] = scale[e] * (x[t] @ a[e].float().T @ b[e].float().T)
    return out


def norm_in_fp32(h, weight):
    return h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * weight


def serve(T, H, I, E, topk, n, r, gen):
    """Relative errors of the projection's adapters and of the whole layer's output against fp32 on the same 4-bit weights' values and the same routing."""
    dt = torch.bfloat16
    x, residual = (torch.randn(T, H, generator=gen, device="cuda").to(dt) for _ in range(2))
    weight = (1 + 0.1 * torch.randn(H, generator=gen, device="cuda")).to(dt)
    w = qmm.mx_quantize(qmm.MXFP4, torch.randn(H, H, generator=gen, device="cuda") * H**-0.5)
    a, b, scale = adapters(n, r, H, H, dt, gen)
    idx = torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32)      # -1: the base model alone
    y, h = qmm.rms_norm(x, weight, EPS, residual=residual)
    base = qmm.mx_linear(qmm.MXFP4, y, w, H)
    out = qmm.lora(y, idx, a, b, base, scale=scale)
    want = base.float() + lora_in_fp32(y.float(), idx, a, b, scale)
    adapted = float((out.float() - want).norm() / want.norm())
    # the routed part of the layer
    y2, h2 = qmm.rms_norm(out, weight, EPS, residual=h)
    gate, up, down = (torch.randn(E, p, q, generator=gen, device="cuda") * 0.05 for p, q in ((I, H), (I, H), (H, I)))
    packed = [torch.cat([qmm.mx_quantize(qmm.MXFP4, m) for m in v]) for v in (gate, up, down)]
    logits = y2.float() @ torch.randn(H, E, generator=gen, device="cuda") * H**-0.5
    chosen, weights = qmm.expert_route(logits, topk, qmm.SIGMOID, bias=torch.zeros(E, device="cuda"), groups=4, top_groups=2, group_top=2)
    z = qmm.mx_moe(qmm.MXFP4, y2, chosen, weights, *packed, I, E)
    xf, ref = norm_in_fp32(h2.float(), weight.float()), torch.zeros(T, H, device="cuda")
    for j in range(topk):
        e = chosen[:, j].long()
        g, u = (torch.einsum("th,tih->ti", xf, v[e]) for v in (gate, up))
        ref += weights[:, j, None] * torch.einsum("ti,thi->th", torch.nn.functional.silu(g) * u, down[e])
    return adapted, float((z.float() - ref).norm() / ref.norm())


def train(T, H, N, E, topk, n, r, gen):
    """Largest relative difference of the gradients (x, residual, norm weight, adapters, router) from torch's own in fp32 on the rows of 8 bits."""
    dt = torch.bfloat16
    leaf = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device="cuda") * std).to(dt).requires_grad_()  # noqa: E731
    x, residual, weight = leaf(T, H), leaf(T, H), (1 + 0.1 * torch.randn(H, generator=gen, device="cuda")).to(dt).requires_grad_()
    w = (torch.randn(N, H, generator=gen, device="cuda") * H**-0.5).to(dt)                  # the frozen projection's values
    packed = qmm.mx_quantize(qmm.MXFP4, w)
    a, b, scale = adapters(n, r, H, N, dt, gen)
    a.requires_grad_(), b.requires_grad_()
    router = (torch.randn(N, E, generator=gen, device="cuda") * N**-0.5).requires_grad_()
    idx = torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
    experts = torch.randn(E, generator=gen, device="cuda")                                  # each expert: a factor of its own
    target, to_h = torch.randn(T, N, generator=gen, device="cuda"), torch.randn(T, H, generator=gen, device="cuda")
    bias = torch.randn(E, generator=gen, device="cuda") * 0.05
    y, h, codes, scales = Norm.apply(x, residual, weight)
    base = qmm.mx_linear(qmm.MXFP4, y.detach(), packed, N)
    out = Adapted.apply(y, base, a, b, idx, scale, codes, scales, w)
    logits = out.float() @ router
    chosen, weights = Route.apply(logits, topk, bias)
    mixed = (weights * experts[chosen.long()]).sum(1, keepdim=True) * out.float()
    loss = ((mixed - target) ** 2).mean() + (h.float() * to_h).mean()
    leaves = (x, residual, weight, a, b, router)
    got = torch.autograd.grad(loss, leaves)

    # the same in fp32: the kept rows stand for y (their rounding passes the gradient on), the frozen product's value is the one that was computed
    f = [v.detach().float().requires_grad_() for v in leaves]
    hf = f[0] + f[1]
    hf = hf + (h.detach().float() - hf).detach()
    yf = norm_in_fp32(hf, f[2])
    kept = yf + (qmm.rows_dequantize(codes, scales) - yf).detach()
    linear = yf @ w.float().T
    delta = torch.zeros(T, N, device="cuda")
    for e in range(n):
        delta = delta + torch.where((idx == e)[:, None], scale[e] * (kept @ f[3][e].T @ f[4][e].T), 0.0)
    of = linear + delta
    of = of + (out.detach().float() - of).detach()
    s = torch.sigmoid(of @ f[5]).gather(1, chosen.long())
    mixed = (s / s.sum(1, keepdim=True) * experts[chosen.long()]).sum(1, keepdim=True) * of
    want = torch.autograd.grad(((mixed - target) ** 2).mean() + (hf * to_h).mean(), f)
    return max(float((p.float() - q).norm() / q.norm()) for p, q in zip(got, want))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=64)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    adapted, layer = serve(a.tokens, 512, 256, 16, 4, 6, 16, gen)
    trained = train(a.tokens, 512, 384, 16, 4, 3, 16, gen)
    print("adapters beside the projection: relative error %.2g; routed layer: %.3f; gradients against torch: %.2g" % (adapted, layer, trained))
    return adapted, layer, trained


if __name__ == "__main__":
    main()
