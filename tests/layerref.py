"""The router, the norm with 8-bit rows and the adapters in plain 64-bit torch, written from the definitions in include/qmm.h
(test infrastructure; shares no code with the library)."""
import math

import torch

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
STEP = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}       # half an ulp, relative
TINY = {torch.float16: 2.0**-25, torch.bfloat16: 2.0**-134, torch.float32: 2.0**-150}     # half the smallest subnormal
ROW8 = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}


def rounding(v, dtype):
    """Largest error of rounding the fp64 values v to dtype."""
    return STEP[dtype] * v.abs() + TINY[dtype]


# ------------------------------------------------------------------ router

def scores(l, sigmoid):
    live = l > -math.inf
    if sigmoid:
        return torch.where(live, 1 / (1 + torch.exp(-l)), 0.0)
    m = torch.where(live, l, -math.inf).amax(1, keepdim=True)
    e = torch.where(live, torch.exp(l - torch.where(m > -math.inf, m, 0.0)), 0.0)
    return e / e.sum(1, keepdim=True).clamp(min=1e-300)


def clean(logits):
    l = logits.double()
    l = torch.where(torch.isnan(l), -math.inf, l)
    return l.clamp(max=torch.finfo(torch.float32).max)


def route(logits, topk, sigmoid, bias, groups, top_groups, group_top, renorm, scale):
    """(idx [T, topk], weights fp64) token by token."""
    l = clean(logits.cpu())
    T, E = l.shape
    s = scores(l, sigmoid)
    b = None if bias is None else bias.double().cpu()
    idx, w = torch.full((T, topk), -1, dtype=torch.int64), torch.zeros(T, topk, dtype=torch.float64)
    per = E // groups
    sl, ll = s.tolist(), l.tolist()
    bl = [0.0] * E if b is None else b.tolist()
    for t in range(T):
        c = [sl[t][e] + bl[e] if ll[t][e] > -math.inf else -math.inf for e in range(E)]
        c = [-math.inf if v != v else v for v in c]
        key = c if b is not None else ll[t]
        stay = range(groups)
        if groups > 1:
            value = []
            for g in range(groups):
                best = sorted((c if b is not None or group_top == 2 else key)[g * per:(g + 1) * per], reverse=True)[:group_top]
                value.append(best[0] + (best[1] if len(best) > 1 and best[1] > -math.inf else 0.0))
            stay = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
        open_ = [e for g in stay for e in range(g * per, (g + 1) * per) if c[e] > -math.inf]
        chosen = sorted(open_, key=lambda e: (-key[e], e))[:topk]
        if not chosen:
            continue
        v = torch.tensor([sl[t][e] for e in chosen], dtype=torch.float64)
        if renorm:                                         # relative to the largest: the scores themselves may underflow
            x = torch.tensor([ll[t][e] for e in chosen], dtype=torch.float64)
            v = torch.nn.functional.logsigmoid(x) if sigmoid else x
            v = torch.exp(v - v.max())
            v = v / v.sum()
        idx[t, :len(chosen)] = torch.tensor(chosen)
        w[t, :len(chosen)] = scale * v
    return idx, w


def route_weights(l, idx, sigmoid, renorm, scale):
    """Differentiable weights of a given choice (fp64 logits, idx -1 dropped): for gradients by autograd."""
    live = idx >= 0
    s = torch.where(l > -math.inf, torch.sigmoid(l), 0.0) if sigmoid else torch.softmax(l, 1)
    v = torch.where(live, s.gather(1, idx.clamp(min=0)), 0.0)
    if renorm:
        x = l.gather(1, idx.clamp(min=0))
        x = torch.nn.functional.logsigmoid(x) if sigmoid else x
        x = torch.where(live, x, -1e300)
        v = torch.where(live, torch.softmax(x, 1), 0.0)
    return scale * v


# -------------------------------------------------------------------- norm

def add(x, residual):
    return x if residual is None else (x.float() + residual.float()).to(x.dtype)


def norm(h, weight, eps):
    """(rstd [rows, 1], y) in fp64."""
    h = h.double()
    rstd = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    return rstd, h * rstd * (1.0 if weight is None else weight.double())


def rows8(t, kind, rstd):
    """fp32 products t -> (codes, scales fp64): the codes bit for bit."""
    top = TOP[kind]
    amax = t.abs().amax(1, keepdim=True)
    fine = torch.isfinite(t).all(1, keepdim=True)
    some = fine & (amax >= 2.0**-118)
    inv = torch.where(some, torch.full_like(amax, top) / torch.where(some, amax, 1.0), 0.0)        # (a number / a tensor would be rounded twice)
    q = torch.where(some, (torch.where(some, t, 0.0) * inv).clamp(-top, top), 0.0)
    codes = q.to(kind) if kind == torch.float8_e4m3fn else torch.round(q).to(kind)
    scale = torch.where(some, amax.double() / top * rstd, 0.0)
    return codes, torch.where(fine, scale, math.nan)[:, 0]


# ---------------------------------------------------------------- adapters

def lora(x, idx, a, b, scale):
    """(S, U . B^T, and the sums of magnitudes sum |a x|, sum |B u|, |B| . sum |a x|) of fp64 inputs; rows without an adapter: zeros."""
    T, n, r, N = x.shape[0], a.shape[0], a.shape[1], b.shape[1]
    s, mag_s = (torch.zeros(T, r, dtype=torch.float64, device=x.device) for _ in range(2))
    d, mag_d, mag_ds = (torch.zeros(T, N, dtype=torch.float64, device=x.device) for _ in range(3))
    for e in range(n):
        t = torch.nonzero(idx == e)[:, 0]
        if t.numel() == 0:
            continue
        c = 1.0 if scale is None else float(scale[e])
        s[t] = x[t] @ a[e].T
        mag_s[t] = x[t].abs() @ a[e].abs().T
        d[t] = c * (s[t] @ b[e].T)
        mag_d[t] = abs(c) * (s[t].abs().amax(1, keepdim=True) * b[e].abs().sum(1))
        mag_ds[t] = abs(c) * (mag_s[t] @ b[e].abs().T)
    return s, d, mag_s, mag_d, mag_ds


def sum_error(terms):
    """Relative error (of the sum of magnitudes) of a fp32 sum of `terms` products on the tensor cores: a step adds 16 products and the sum so far, each
    cut to no less than 25 bits below the largest (17 * 2^-25 < 2^-20), and about 16 + 16 fp32 additions join the parts."""
    return (terms / 16 + 32) * 2.0**-20
