"""A routed feed-forward layer on 4-bit weights, served and trained through, with the operators of qmm.py.

  serving   router logits -> moe_route (top-k experts and weights) -> mx_moe (sort, quantise, gate / up, down, weighted sum)
  training  the same routing around experts of the program's own: expert_sort, expert_gather, expert_combine and their
            gradients as a torch.autograd.Function each

Run on a B200:  python examples/mx_moe_layer.py [--tokens 64] [--fmt mxfp4|nvfp4]
It prints how far the layer is from the same layer in fp32, and the gradients from torch's own.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_00501_b200 import qmm  # noqa: E402


def pack_experts(fmt, w):
    """fp32 [E, N, K] -> E packed matrices one after the other, and their tensor scales [E] (NVFP4; None for MXFP4)."""
    scales = w.abs().amax(dim=(1, 2)) / (448 * 6) if fmt == qmm.NVFP4 else None
    packed = [qmm.mx_quantize(fmt, m, tensor_scale=None if scales is None else scales[e:e + 1]) for e, m in enumerate(w)]
    return torch.cat(packed), scales


def route(logits, topk):
    """Top-k experts of each token (equal logits: lower index first) and the softmax over their logits."""
    T, E = logits.shape
    idx = torch.empty((T, topk), dtype=torch.int32, device=logits.device)
    weights = torch.empty((T, topk), dtype=torch.float32, device=logits.device)
    args = qmm.moe_args(qmm.Q4, T, 256, 256, E, topk, logits, None, None, None, None, None, topk_idx=idx, topk_w=weights)
    ws = torch.zeros(qmm.moe_workspace_bytes(args), dtype=torch.uint8, device=logits.device)
    qmm.moe_route(args, ws)
    qmm.status_check(ws)
    return idx, weights


class Gather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, plan):
        ctx.plan = plan
        return qmm.expert_gather(x, plan)

    @staticmethod
    def backward(ctx, dxs):
        return qmm.expert_gather_grad(dxs.contiguous(), ctx.plan), None


class Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ys, weights, plan):
        ctx.save_for_backward(ys, weights)
        ctx.plan = plan
        return qmm.expert_combine(ys, plan, weights)

    @staticmethod
    def backward(ctx, dy):
        ys, weights = ctx.saved_tensors
        dys, dw = qmm.expert_combine_grad(dy.contiguous(), ys, ctx.plan, weights)
        return dys, dw, None


def serve(fmt, T, H, I, E, topk, gen):
    """(relative error of the 4-bit layer against fp32 on the same routing, seconds are not measured here)."""
    dev = "cuda"
    gate, up, down = (torch.randn(E, n, k, generator=gen, device=dev) * 0.05 for n, k in ((I, H), (I, H), (H, I)))
    x = torch.randn(T, H, generator=gen, device=dev).half()
    idx, weights = route(torch.randn(T, E, generator=gen, device=dev), topk)
    (gp, gs), (up_p, us), (dp, ds) = (pack_experts(fmt, w) for w in (gate, up, down))
    scales = {}
    if fmt == qmm.NVFP4:                                   # activations' tensor scales: from their ranges, as a calibration would
        scales = {"x_scale": (x.abs().max() / (448 * 6)).float().reshape(1), "h_scale": torch.full((1,), 8.0 / (448 * 6), device=dev),
                  "gate_scale": gs, "up_scale": us, "down_scale": ds}
    out = torch.empty_like(x)
    args = qmm.mx_moe_args(fmt, x, idx, weights, gp, up_p, dp, I, E, out, **scales)
    ws = torch.zeros(qmm.mx_moe_workspace_bytes(args), dtype=torch.uint8, device=dev)
    qmm.mx_moe_run(args, ws)
    qmm.status_check(ws)
    xf, ref = x.float(), torch.zeros(T, H, device=dev)
    for j in range(topk):
        e = idx[:, j].long()
        g, u = (torch.einsum("th,tih->ti", xf, w[e]) for w in (gate, up))
        ref += weights[:, j, None] * torch.einsum("ti,thi->th", torch.nn.functional.silu(g) * u, down[e])
    return float((out.float() - ref).norm() / ref.norm())


def train(T, H, E, topk, gen):
    """Largest relative difference of the gradients (x, expert scale and bias, routing weights) from torch's own."""
    dev = "cuda"
    x = torch.randn(T, H, generator=gen, device=dev, requires_grad=True)
    idx, w0 = route(torch.randn(T, E, generator=gen, device=dev), topk)
    weights = w0.clone().requires_grad_()
    scale = torch.randn(E, H, generator=gen, device=dev, requires_grad=True)              # each expert: x -> tanh(scale_e * x)
    target = torch.randn(T, H, generator=gen, device=dev)
    plan = qmm.expert_sort(idx, E)
    rows_expert = idx.reshape(-1).long()[plan.order.long()]                               # (no pair is dropped here)
    ys = torch.tanh(scale[rows_expert] * Gather.apply(x, plan))
    loss = ((Combine.apply(ys, weights, plan) - target) ** 2).sum()
    got = torch.autograd.grad(loss, (x, weights, scale))
    plain = (torch.tanh(scale[idx.long()] * x[:, None, :]) * weights[..., None]).sum(1)
    want = torch.autograd.grad(((plain - target) ** 2).sum(), (x, weights, scale))
    return max(float((a - b).norm() / b.norm()) for a, b in zip(got, want))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--fmt", choices=("mxfp4", "nvfp4"), default="mxfp4")
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    served = serve(qmm.MXFP4 if a.fmt == "mxfp4" else qmm.NVFP4, a.tokens, 512, 256, 16, 4, gen)
    trained = train(a.tokens, 512, 16, 4, gen)
    print("4-bit layer against fp32: relative error %.3f; gradients against torch: %.2g" % (served, trained))
    return served, trained


if __name__ == "__main__":
    main()
