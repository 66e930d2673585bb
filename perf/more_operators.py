"""Cases and plain forms of the router, of the root-mean-square norm with 8-bit rows, and of low-rank adapters.

Three kinds of case, each one call sequence that a program makes around the quantised products and the experts:

  route  router logits -> each token's experts and weights; `train` adds the gradient of the logits
  norm   residual addition and root-mean-square norm; out in x's type, or in 8 bits with a scale per row (and back to the
         values that the codes stand for); `train` adds the gradients
  lora   low-rank adapters of many requests beside a shared projection; `train` adds the gradients, and x may be held in 8 bits
"""
import math

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}
_ROW8 = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_TOP = {"e4m3": 448.0, "int8": 127.0}
EPS = 1e-6


# ------------------------------------------------------------------ cases

def listed():
    return [
        # a decode step's router, four sequences: latency
        {"name": "route_decode", "kind": "route", "train": False, "dtype": "f32", "T": 4, "E": 128, "topk": 8, "scores": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_top": 1, "renorm": True, "masked": 0},
        # a prompt's router with a balance bias and groups; three experts switched off
        {"name": "route_prompt", "kind": "route", "train": False, "dtype": "bf16", "T": 2048, "E": 256, "topk": 8, "scores": "sigmoid", "bias": True,
         "groups": 8, "top_groups": 4, "group_top": 2, "renorm": True, "masked": 3},
        # a training step's router over a large batch, weights not renormalised, with the gradient
        {"name": "route_train", "kind": "route", "train": True, "dtype": "f32", "T": 16384, "E": 128, "topk": 8, "scores": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_top": 1, "renorm": False, "masked": 0},
        # the norm in front of a decode step's projection, four sequences: latency
        {"name": "norm_decode", "kind": "norm", "train": False, "dtype": "f16", "M": 4, "K": 2048, "residual": True, "rows": "same"},
        # a long prompt's norm into 8-bit rows and back: bandwidth
        {"name": "norm_rows8", "kind": "norm", "train": False, "dtype": "bf16", "M": 8192, "K": 8192, "residual": True, "rows": "e4m3"},
        # a small training batch of odd width
        {"name": "norm_train_small", "kind": "norm", "train": True, "dtype": "f32", "M": 500, "K": 1001, "residual": False, "rows": "same"},
        # a training step's norm
        {"name": "norm_train", "kind": "norm", "train": True, "dtype": "bf16", "M": 8192, "K": 4096, "residual": True, "rows": "same"},
        # a decode step, sixteen requests with adapters of their own beside the down projection
        {"name": "lora_decode", "kind": "lora", "train": False, "dtype": "f16", "T": 16, "K": 8192, "N": 2048, "n": 64, "r": 16, "rows": "same"},
        # an odd batch in decode, few adapters of high rank shared by many requests
        {"name": "lora_batch", "kind": "lora", "train": False, "dtype": "bf16", "T": 77, "K": 2048, "N": 2048, "n": 5, "r": 64, "rows": "same"},
        # prompts of several requests through the widest projection
        {"name": "lora_prompt", "kind": "lora", "train": False, "dtype": "f16", "T": 2048, "K": 4096, "N": 28672, "n": 8, "r": 16, "rows": "same"},
        # a small training batch of odd widths
        {"name": "lora_train_small", "kind": "lora", "train": True, "dtype": "bf16", "T": 500, "K": 1001, "N": 700, "n": 3, "r": 8, "rows": "same"},
        # a training step, x kept in 8 bits from its norm
        {"name": "lora_train", "kind": "lora", "train": True, "dtype": "bf16", "T": 8192, "K": 2048, "N": 8192, "n": 4, "r": 32, "rows": "e4m3"},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind, train = rng.choice(("route", "norm", "lora", "lora")), rng.random() < 0.5
    if kind == "route":
        G = rng.choice((1, 1, 2, 4, 8))
        E = G * rng.randint(8, 256 // G)
        top = rng.randint(1, G)
        return {"kind": kind, "train": train, "dtype": rng.choice(("f16", "bf16", "f32")), "T": _spread(rng, 1, 16000), "E": E,
                "topk": rng.randint(1, min(8, top * E // G)), "scores": rng.choice(("softmax", "sigmoid")), "bias": rng.random() < 0.5, "groups": G,
                "top_groups": top, "group_top": rng.randint(1, 2), "renorm": rng.random() < 0.7, "masked": rng.choice((0, 0, 1, 3))}
    if kind == "norm":
        return {"kind": kind, "train": train, "dtype": rng.choice(("f16", "bf16", "f32")), "M": _spread(rng, 1, 8000),
                "K": rng.choice((8 * _spread(rng, 8, 600), _spread(rng, 64, 5000))), "residual": rng.random() < 0.6,
                "rows": "same" if train else rng.choice(("same", "e4m3", "int8"))}
    T = _spread(rng, 1, 8000)
    K, N = (rng.choice((8 * _spread(rng, 16, 512), 256 * rng.randint(1, 16), _spread(rng, 100, 4000))) for _ in range(2))
    return {"kind": kind, "train": train, "dtype": rng.choice(("f16", "bf16")), "T": T, "K": K, "N": N, "n": _spread(rng, 1, 64),
            "r": rng.choice((8, 16, 16, 32, 64)), "rows": rng.choice(("same", "same", "e4m3", "int8"))}


# ----------------------------------------------------------------- inputs

def _requests(gen, T, n, dev):
    """The adapter of each row: of each row by itself in a decode step, of runs of rows (sequences) in a larger batch; 5 per cent have none."""
    runs = T if T <= 256 else min(T, 4 * n)
    cut = torch.sort(torch.randint(0, T, (runs - 1,), generator=gen, device=dev)).values if T > 256 else torch.arange(1, T, device=dev)
    of_run = torch.randint(0, n, (runs,), generator=gen, device=dev, dtype=torch.int32)
    of_run = torch.where(torch.rand(runs, generator=gen, device=dev) < 0.05, torch.full_like(of_run, -1), of_run)
    return of_run[torch.searchsorted(cut, torch.arange(T, device=dev), right=True)].contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    st = {"case": case}
    kind, dt = case["kind"], _DT[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * std).to(dt)

    if kind == "route":
        T, E, topk = case["T"], case["E"], case["topk"]
        st["logits"] = normal(T, E, std=1.5)
        if case["masked"]:                                 # experts that are switched off, for every token
            off = torch.randperm(E, generator=gen, device=dev)[: case["masked"]]
            st["logits"][:, off] = -math.inf
        st["bias"] = torch.randn(E, generator=gen, device=dev) * 0.05 if case["bias"] else None
        st["idx"] = torch.empty(T, topk, dtype=torch.int32, device=dev)
        st["weights"] = torch.empty(T, topk, device=dev)
        if case["train"]:
            st["dweights"], st["dlogits"] = torch.randn(T, topk, generator=gen, device=dev), torch.empty_like(st["logits"])
    elif kind == "norm":
        M, K = case["M"], case["K"]
        st["x"], st["weight"] = normal(M, K), (1 + 0.1 * torch.randn(K, generator=gen, device=dev)).to(dt)
        st["residual"] = normal(M, K, std=2.0) if case["residual"] else None
        st["h"] = torch.empty_like(st["x"]) if case["residual"] else None
        st["y"] = torch.empty_like(st["x"])
        if case["rows"] != "same":
            st["codes"], st["scales"] = torch.empty(M, K, dtype=_ROW8[case["rows"]], device=dev), torch.empty(M, device=dev)
        if case["train"]:
            st["dy"], st["dx"], st["dweight"] = normal(M, K), torch.empty_like(st["x"]), torch.empty(K, device=dev)
            st["dh"] = normal(M, K) if case["residual"] else None
    else:
        T, K, N, n, r = (case[k] for k in ("T", "K", "N", "n", "r"))
        st["idx"] = _requests(gen, T, n, dev)
        kept = st["idx"][st["idx"] >= 0].long()
        st["most"] = int(torch.bincount(kept, minlength=n).max()) if kept.numel() else 0
        st["a"], st["b"] = normal(n, r, K, std=K ** -0.5), normal(n, N, r, std=0.1)
        st["scale"] = torch.full((n,), 16.0 / r, device=dev)
        x = torch.randn(T, K, generator=gen, device=dev)
        if case["rows"] == "same":
            st["x"], st["x_scale"] = x.to(dt), None
        else:                                              # rows of 8 bits with a scale each, as a norm leaves them
            top = _TOP[case["rows"]]
            st["x_scale"] = x.abs().amax(1) / top
            q = (x / st["x_scale"][:, None]).clamp(-top, top)
            st["x"] = q.to(_ROW8[case["rows"]]) if case["rows"] == "e4m3" else q.round().to(torch.int8)
        del x
        st["y0"], st["y"] = normal(T, N), torch.empty(T, N, dtype=dt, device=dev)
        if case["train"]:
            st["s"] = torch.zeros(T, r, device=dev)
            st["dy"], st["dx0"], st["dx"] = normal(T, N), normal(T, K), torch.empty(T, K, dtype=dt, device=dev)
            st["da"], st["db"] = torch.empty(n, r, K, device=dev), torch.empty(n, N, r, device=dev)
    return st


# --------------------------------------------------------------- one pass

def _own_run(st):
    from paper_2607_00501_b200 import qmm
    case, kind = st["case"], st["case"]["kind"]
    if kind == "route":
        scores = qmm.SOFTMAX if case["scores"] == "softmax" else qmm.SIGMOID
        idx, weights = qmm.expert_route(st["logits"], case["topk"], scores=scores, bias=st["bias"], groups=case["groups"], top_groups=case["top_groups"],
                                        group_top=case["group_top"], renormalize=case["renorm"], scale=2.5, idx=st["idx"], weights=st["weights"])
        out = {"idx": idx, "weights": weights}
        if case["train"]:
            out["dlogits"] = qmm.expert_route_grad(st["dweights"], st["logits"], idx, scores=scores, renormalize=case["renorm"], scale=2.5, out=st["dlogits"])
        return out
    if kind == "norm":
        if case["rows"] == "same":
            y, h = qmm.rms_norm(st["x"], st["weight"], EPS, residual=st["residual"], h=st["h"], y=st["y"])
        else:
            codes, scales, h = qmm.rms_norm_rows(st["x"], st["weight"], EPS, residual=st["residual"], h=st["h"], codes=st["codes"], scales=st["scales"])
            y = qmm.rows_dequantize(codes, scales, out=st["y"])
        out = {"y": y}
        if case["residual"]:
            out["h"] = h
        if case["train"]:
            if "ws" not in st:                             # the workspace that a program keeps
                st["ws"] = torch.empty(qmm.rms_norm_grad_workspace_bytes(case["M"], case["K"]), dtype=torch.uint8, device=h.device)
            out["dx"], out["dweight"] = qmm.rms_norm_grad(st["dy"], h, st["weight"], EPS, dh=st["dh"], dx=st["dx"], dweight=st["dweight"], ws=st["ws"])
        return out
    if "ws" not in st:
        st["ws"] = torch.empty(qmm.lora_workspace_bytes(case["T"], case["n"], case["r"]), dtype=torch.uint8, device=st["y"].device)
        st["plan"] = qmm.ExpertPlan(case["T"], 1, case["n"]) if case["train"] else None
    plan = st["plan"]
    if plan is not None:                                   # the rows sorted by adapter once for both directions
        qmm.expert_sort(st["idx"].view(-1, 1), case["n"], out=plan)
    y = qmm.lora(st["x"], st["idx"], st["a"], st["b"], st["y0"], scale=st["scale"], x_scale=st["x_scale"], s=st.get("s"), plan=plan, ws=st["ws"], out=st["y"])
    if not case["train"]:
        return y
    dx, da, db = qmm.lora_grad(st["dy"], st["x"], st["s"], st["idx"], st["a"], st["b"], st["dx0"], scale=st["scale"], x_scale=st["x_scale"], plan=plan, ws=st["ws"],
                               dx=st["dx"], da=st["da"], db=st["db"])
    return {"y": y, "s": st["s"], "dx": dx, "da": da, "db": db}


def _route_plain(st):
    case = st["case"]
    l = st["logits"].float()
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    there = l > -math.inf
    T, E, G, topk = case["T"], case["E"], case["groups"], case["topk"]
    sigmoid = case["scores"] == "sigmoid"

    def scores(v, live):
        if sigmoid:
            return torch.where(live, 1 / (1 + torch.exp(-v)), torch.zeros_like(v))
        e = torch.where(live, torch.exp(v - v.amax(-1, keepdim=True)), torch.zeros_like(v))
        return e / e.sum(-1, keepdim=True).clamp(min=1e-300 if v.dtype == torch.float64 else 1e-38)

    # who is chosen is decided in 64 bits: neighbours in the order may be nearer to one another than 32 bits tell
    c = scores(l.double(), there)
    by_logit = st["bias"] is None                          # the order of the scores is that of the logits
    if not by_logit:
        c = c + st["bias"].double()
    key = torch.where(there, l.double() if by_logit else c, torch.full_like(c, -math.inf))
    if G > 1:
        of_group = torch.where(there, c, torch.full_like(c, -math.inf)).view(T, G, E // G) if not by_logit or case["group_top"] == 2 else key.view(T, G, E // G)
        best = torch.sort(of_group, dim=2, descending=True).values[:, :, : case["group_top"]]
        first = best[..., 0]
        value = first if case["group_top"] == 1 else first + torch.where(best[..., 1] > -math.inf, best[..., 1], torch.zeros_like(first))
        stay = torch.sort(value, dim=1, descending=True, stable=True).indices[:, : case["top_groups"]]
        open_ = torch.zeros(T, G, dtype=torch.bool, device=l.device).scatter_(1, stay, True)
        key = torch.where(open_[..., None].expand(T, G, E // G).reshape(T, E), key, torch.full_like(key, -math.inf))
    val, idx = torch.sort(key, dim=1, descending=True, stable=True)
    val, idx = val[:, :topk], idx[:, :topk]
    live = val > -math.inf
    at = l.gather(1, idx)
    if not case["renorm"]:
        w = scores(l, there).gather(1, idx)
    elif sigmoid:
        w = 1 / (1 + torch.exp(-at))
    else:
        w = torch.exp(at - torch.where(live, at, torch.full_like(at, -math.inf)).amax(1, keepdim=True))
    w = torch.where(live, w, torch.zeros_like(w))
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-38)
    out = {"idx": torch.where(live, idx, torch.full_like(idx, -1)).int(), "weights": 2.5 * w}
    if case["train"]:
        g = torch.where(live, 2.5 * st["dweights"], torch.zeros_like(w))
        if sigmoid:
            one_less = torch.where(live, 1 / (1 + torch.exp(at)), torch.zeros_like(at))
            d = w * (g - (g * w).sum(1, keepdim=True) if case["renorm"] else g) * one_less
        else:
            d = w * (g - (g * w).sum(1, keepdim=True))
        d = torch.where(live, d, torch.zeros_like(d))
        if sigmoid or case["renorm"]:
            full = torch.zeros_like(l)
        else:
            full = scores(l, there) * -(g * w).sum(1, keepdim=True)
            full.scatter_(1, torch.where(live, idx, idx[:, :1]), 0.0)
        out["dlogits"] = full.scatter_add_(1, idx, d).to(st["logits"].dtype)
    return out


def _norm_plain(st):
    case, dt = st["case"], st["x"].dtype
    x = st["x"].float()
    h = (x + st["residual"].float()).to(dt) if case["residual"] else st["x"]
    hf, w = h.float(), st["weight"].float()
    rstd = 1 / torch.sqrt((hf * hf).mean(1, keepdim=True) + EPS)
    if case["rows"] == "same":
        out = {"y": (hf * rstd * w).to(dt)}
    else:
        top = _TOP[case["rows"]]
        t = hf * w
        amax = t.abs().amax(1, keepdim=True)
        q = (t * (torch.full_like(amax, top) / amax)).clamp(-top, top)          # (a number / a tensor is a reciprocal and a product: two roundings)
        codes = q.to(torch.float8_e4m3fn).float() if case["rows"] == "e4m3" else torch.round(q)
        out = {"y": (codes * (amax / top * rstd)).to(dt)}
    if case["residual"]:
        out["h"] = h
    if case["train"]:
        dy, xhat = st["dy"].float(), hf * rstd
        g = dy * w
        dx = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True))
        out["dx"] = (dx + st["dh"].float() if case["residual"] else dx).to(dt)
        out["dweight"] = (dy * xhat).sum(0)
    return out


def _lora_plain(st):
    case = st["case"]
    T, n = case["T"], case["n"]
    idx, dt = st["idx"].long(), st["y"].dtype
    x = st["x"].float() if st["x_scale"] is None else st["x"].float() * st["x_scale"][:, None]
    # rows of each adapter, padded to the longest: [n, most]
    key, order = torch.sort(torch.where((idx >= 0) & (idx < n), idx, torch.full_like(idx, n)), stable=True)
    offsets = torch.searchsorted(key, torch.arange(n + 1, device=idx.device))
    at = torch.arange(st["most"], device=idx.device)[None, :] + offsets[:n, None]
    inside = (at < offsets[1:, None])[..., None]
    row = order[at.clamp(max=T - 1)]
    scale = st["scale"][:, None, None]
    a, b = st["a"].float(), st["b"].float()

    def back(rows, width):                                 # [n, most, width] -> [T, width], zeros where a row has no adapter
        out = torch.zeros(T, width, device=idx.device)
        out[row[inside[..., 0]]] = rows[inside[..., 0]]
        return out

    xs = x[row] * inside
    s = xs @ a.transpose(1, 2)
    y = (st["y0"].float() + back((scale * s) @ b.transpose(1, 2), case["N"])).to(dt)
    if not case["train"]:
        return y
    dys = st["dy"].float()[row] * inside
    ds = scale * (dys @ b)
    return {"y": y, "s": back(s, case["r"]), "dx": (st["dx0"].float() + back(ds @ a, case["K"])).to(dt), "da": ds.transpose(1, 2) @ xs,
            "db": dys.transpose(1, 2) @ (scale * s)}


def run(state):
    if own:
        return _own_run(state)
    return {"route": _route_plain, "norm": _norm_plain, "lora": _lora_plain}[state["case"]["kind"]](state)


# ------------------------------------------------------------------- work

def work(case):
    kind, size = case["kind"], _SIZE[case["dtype"]]
    if kind == "route":
        n, k = case["T"] * case["E"], case["T"] * case["topk"]
        return {"bytes": n * size * (2 if case["train"] else 1) + k * 8 + (k * 4 if case["train"] else 0), "flops": n * 4}
    if kind == "norm":
        n = case["M"] * case["K"]
        moved = n * size * (4 if case["residual"] else 2)
        if case["rows"] != "same":
            moved += 2 * n + 8 * case["M"]                 # the codes written and read
        if case["train"]:
            moved += n * size * (3 if case["residual"] else 2) + 4 * case["K"]
        return {"bytes": moved + case["K"] * size, "flops": n * (12 if case["train"] else 4)}
    T, K, N, n, r = (case[k] for k in ("T", "K", "N", "n", "r"))
    used = n * (1 - (1 - 1 / n) ** T)                      # adapters that get a row, on average
    moved = T * K * (size if case["rows"] == "same" else 1) + 2 * T * N * size + int(used * r * (K + N) * size) + 4 * T
    flops = 2 * T * r * (K + N)
    if case["train"]:
        moved += T * N * size + 2 * T * K * size + 4 * n * r * (K + N) + 4 * T * r
        flops *= 3
    return {"bytes": moved, "flops": flops}


# ----------------------------------------------- the definition in 64 bits

def _f32(x):
    return x.to(torch.float32).double()                    # a value that the definition rounds to fp32


def _route_exact(st):
    case, E, topk, G = st["case"], st["case"]["E"], st["case"]["topk"], st["case"]["groups"]
    l = torch.nan_to_num(st["logits"].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    off = l == -math.inf
    s = torch.sigmoid(l) if case["scores"] == "sigmoid" else torch.softmax(l, 1)
    s = torch.where(off, torch.zeros_like(s), s)
    none = torch.full_like(l, -math.inf)
    c = l if st["bias"] is None else torch.where(off, none, s + st["bias"].double())
    if G > 1:
        v = torch.where(off, none, s) if st["bias"] is None and case["group_top"] == 2 else c
        v = torch.topk(v.unflatten(1, (G, E // G)), case["group_top"], dim=2).values
        v = torch.where((v == -math.inf) & (torch.arange(v.shape[2], device=v.device) > 0), torch.zeros_like(v), v).sum(2)
        order = torch.argsort(-v, dim=1, stable=True)
        rank = torch.empty_like(order).scatter_(1, order, torch.arange(G, device=v.device).expand_as(order))
        c = torch.where((rank < case["top_groups"]).repeat_interleave(E // G, 1), c, none)
    idx = torch.argsort(-c, dim=1, stable=True)[:, :topk]
    chosen = torch.zeros_like(off).scatter_(1, idx, True) & (c > -math.inf)
    p = torch.where(chosen, s, torch.zeros_like(s))
    if case["renorm"]:
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    idx = torch.where(chosen.gather(1, idx), idx, torch.full_like(idx, -1))
    at = idx.clamp(min=0)
    out = {"idx": idx.int(), "weights": torch.where(idx >= 0, 2.5 * p.gather(1, at), torch.zeros_like(at, dtype=torch.float64))}
    if case["train"]:
        g = torch.zeros_like(l).scatter_add_(1, at, torch.where(idx >= 0, 2.5 * st["dweights"].double(), torch.zeros(1, dtype=torch.float64, device=l.device)))
        dot = (g * p).sum(1, keepdim=True)
        if case["scores"] == "softmax":
            out["dlogits"] = (p * (g - dot)) if case["renorm"] else s * (g - dot)
        else:
            out["dlogits"] = p * ((g - dot) if case["renorm"] else g) * torch.sigmoid(-l)
        out["dlogits"] = torch.where(off, torch.zeros_like(l), out["dlogits"])
    return out


def _exact_8(t, kind):
    """The nearest value of 8 bits, ties to even, of |t| <= its largest."""
    if kind == "int8":
        return torch.round(t)
    grid = torch.exp2((torch.frexp(t.abs()).exponent - 1).clamp(min=-6).double() - 3)
    return torch.round(t / grid) * grid


def _norm_exact(st):
    case, dt = st["case"], st["x"].dtype
    h = _f32(st["x"].double() + st["residual"].double()).to(dt).double() if case["residual"] else st["x"].double()
    w = st["weight"].double()
    rstd = (h.square().mean(1, keepdim=True) + EPS).rsqrt()
    if case["rows"] == "same":
        out = {"y": h * w * rstd}
    else:
        top = _TOP[case["rows"]]
        t = _f32(h * w)
        amax = t.abs().max(1, keepdim=True).values
        out = {"y": _exact_8(_f32(t * _f32(top / amax)).clamp(-top, top), case["rows"]) * amax / top * rstd}
    if case["residual"]:
        out["h"] = h
    if case["train"]:
        dy = st["dy"].double()
        out["dweight"] = torch.einsum("mk,mk,m->k", dy, h, rstd[:, 0])
        out["dx"] = rstd * dy * w - h * rstd ** 3 * torch.einsum("mk,mk,k->m", dy, h, w)[:, None] / case["K"]
        if case["residual"]:
            out["dx"] = out["dx"] + st["dh"].double()
    return out


def _lora_exact(st):
    case = st["case"]
    x = st["x"].double()
    if st["x_scale"] is not None:
        x = x * st["x_scale"].double()[:, None]
    y = st["y0"].double()
    if case["train"]:
        s, dx = torch.zeros(case["T"], case["r"], dtype=torch.float64, device=x.device), st["dx0"].double()
        da, db = torch.zeros_like(st["a"], dtype=torch.float64), torch.zeros_like(st["b"], dtype=torch.float64)
    for e in range(case["n"]):
        t = torch.nonzero(st["idx"] == e)[:, 0]
        if t.numel() == 0:
            continue
        A, B, c = st["a"][e].double(), st["b"][e].double(), st["scale"][e].double()
        u = torch.einsum("tk,rk->tr", x[t], A)
        y[t] += c * torch.einsum("tr,nr->tn", u, B)
        if case["train"]:
            dy = st["dy"][t].double()
            du = c * torch.einsum("tn,nr->tr", dy, B)
            s[t] = u
            dx[t] += torch.einsum("tr,rk->tk", du, A)
            da[e], db[e] = torch.einsum("tr,tk->rk", du, x[t]), c * torch.einsum("tn,tr->nr", dy, u)
    return {"y": y, "s": s, "dx": dx, "da": da, "db": db} if case["train"] else y


def exact(case, seed):
    return {"route": _route_exact, "norm": _norm_exact, "lora": _lora_exact}[case["kind"]](prepare(case, seed))
