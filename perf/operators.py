"""Cases and plain forms of the microscaled 4-bit floating-point operators and of the expert sort.

Four kinds of case, each one call sequence that a program makes:

  quantize  activations or weights to MXFP4 / NVFP4 and back to the values that the codes stand for
  linear    y = x W^T with W held in 4 bits and x quantised on the way in, from one token to long prompts
  experts   a routed feed-forward layer in 4 bits: sort, gather and quantise, gate / up, down, weighted sum
  route     tokens sorted by expert and back with the routing weights; `train` adds the gradients

MXFP4: e2m1 codes, one e8m0 scale 2^(floor(log2 amax) - 2) per 32 elements along K.  NVFP4: e2m1 codes, one
e4m3 scale rn(amax / (6 g)) per 16 elements and one fp32 scale g per tensor.  Codes are the nearest e2m1
value, ties to the even code, saturating at 6; quotients are IEEE fp32.
"""
import math

import torch

own = False

MXFP4, NVFP4 = 32, 16                     # the format's number is its block length
_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ cases

def listed():
    return [
        # a handful of ragged rows on the way into a product: latency
        {"name": "quantize_small", "kind": "quantize", "fmt": NVFP4, "dtype": "bf16", "M": 33, "K": 1000},
        # a weight matrix or a long prompt's activations: bandwidth
        {"name": "quantize_large", "kind": "quantize", "fmt": MXFP4, "dtype": "f16", "M": 8192, "K": 8192},
        # a decode step's q projection
        {"name": "linear_decode", "kind": "linear", "fmt": MXFP4, "dtype": "f16", "M": 1, "N": 2048, "K": 2048},
        # the output head for one token: one read of the weights
        {"name": "linear_head", "kind": "linear", "fmt": MXFP4, "dtype": "f16", "M": 1, "N": 128256, "K": 2048},
        # an odd batch of sequences in decode
        {"name": "linear_batch", "kind": "linear", "fmt": NVFP4, "dtype": "bf16", "M": 77, "N": 8192, "K": 2048},
        # a prompt through the down projection
        {"name": "linear_prompt", "kind": "linear", "fmt": MXFP4, "dtype": "f16", "M": 2048, "N": 2048, "K": 8192},
        # many prompts at once: the tensor cores' rate
        {"name": "linear_prefill", "kind": "linear", "fmt": NVFP4, "dtype": "bf16", "M": 8192, "N": 8192, "K": 8192},
        # a routed layer in decode, four sequences
        {"name": "experts_decode", "kind": "experts", "fmt": MXFP4, "dtype": "f16", "T": 4, "H": 2048, "I": 768, "E": 128, "topk": 8},
        # the same layer on a prompt
        {"name": "experts_prompt", "kind": "experts", "fmt": MXFP4, "dtype": "f16", "T": 2048, "H": 2048, "I": 768, "E": 128, "topk": 8},
        # the way to the experts and back for a small batch, some pairs dropped
        {"name": "route_serve", "kind": "route", "train": False, "dtype": "f16", "T": 61, "H": 2048, "E": 128, "topk": 8, "dropped": 5},
        # a training step's share of it
        {"name": "route_train_small", "kind": "route", "train": True, "dtype": "f32", "T": 500, "H": 1000, "E": 16, "topk": 2, "dropped": 0},
        {"name": "route_train_large", "kind": "route", "train": True, "dtype": "bf16", "T": 8192, "H": 2048, "E": 128, "topk": 8, "dropped": 2},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantize", "linear", "linear", "experts", "route"))
    fmt, dtype = rng.choice((MXFP4, NVFP4)), rng.choice(("f16", "bf16"))
    if kind == "quantize":
        return {"kind": kind, "fmt": fmt, "dtype": rng.choice(("f16", "bf16", "f32")), "M": _spread(rng, 1, 8000), "K": _spread(rng, 64, 8192)}
    if kind == "linear":
        return {"kind": kind, "fmt": fmt, "dtype": dtype, "M": _spread(rng, 1, 8000), "N": _spread(rng, 100, 8192),
                "K": rng.choice((8 * _spread(rng, 16, 1000), 256 * rng.randint(1, 32)))}
    if kind == "experts":
        return {"kind": kind, "fmt": fmt, "dtype": dtype, "T": _spread(rng, 1, 2000), "H": 64 * rng.randint(2, 32), "I": 32 * rng.randint(2, 24),
                "E": rng.randint(8, 128), "topk": rng.randint(1, 8)}
    return {"kind": kind, "train": rng.random() < 0.6, "dtype": rng.choice(("f16", "bf16", "f32")), "T": _spread(rng, 1, 8000), "H": _spread(rng, 60, 2048),
            "E": rng.randint(8, 256), "topk": rng.randint(1, 8), "dropped": rng.choice((0, 3, 20))}


# ----------------------------------------------------- quantisation, plain form (32 bits)

def _blocks(x, fmt):
    k = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -k % fmt))
    return x.reshape(*x.shape[:-1], -1, fmt)


def _quantize_plain(x, fmt, g):
    """x fp32 [..., K] -> (codes [..., nb, fmt] in 0..15, scale bytes [..., nb], step D [..., nb]); g: the tensor's scale."""
    xb = _blocks(x, fmt)
    amax = xb.abs().amax(-1)
    if fmt == MXFP4:
        byte = ((amax.view(torch.int32) >> 23) - 2).clamp(min=0)
        step = torch.ldexp(torch.ones_like(amax), byte - 127)
        scaled = torch.ldexp(xb, (127 - byte)[..., None])
    else:
        s = (amax / (6.0 * g)).clamp(max=448.0).to(torch.float8_e4m3fn)
        byte = s.view(torch.uint8).to(torch.int32)
        step = s.float() * g
        scaled = torch.where(step[..., None] > 0, xb / step[..., None], torch.zeros_like(xb))
    a = scaled.abs()
    idx = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte()
           + (a > 5.0).byte())
    return idx | (torch.signbit(xb).to(torch.uint8) << 3), byte.to(torch.uint8), step


def _values(codes, step):
    levels = torch.tensor(_LEVELS + tuple(-v for v in _LEVELS), dtype=torch.float32, device=codes.device)
    return (levels[codes.int()] * step[..., None]).flatten(-2)


def _step_of(byte, fmt, g):
    if fmt == MXFP4:
        return torch.ldexp(torch.ones(byte.shape, device=byte.device), byte.int() - 127)
    return byte.view(torch.float8_e4m3fn).float() * g


def _through_4_bits(x, fmt, g):
    """fp32 -> the fp32 values that its codes stand for, same shape."""
    codes, _, step = _quantize_plain(x, fmt, g)
    return _values(codes, step)[..., : x.shape[-1]]


# ----------------------------------------------------------- inputs

def _weights(gen, fmt, count, rows, K, dev):
    """`count` weight matrices N(0, 0.02) in 4 bits: canonical codes [count, rows, nb fmt / 2] and scale bytes [count, rows, nb],
    the tensors' scales [count], and the library's device layout of the same, matrix after matrix (units of 128 rows x 256 k:
    codes in 16-byte chunks, chunk c of row r at place c ^ (r mod 8), then the scale bytes, 4 of row r at 16 (r mod 32) + 4 (r / 32))."""
    g = torch.full((count,), 0.1 / (448 * 6), device=dev) if fmt == NVFP4 else torch.ones(count, device=dev)
    units, ku = -(-rows // 128), -(-K // 256)
    codes = torch.zeros(count, units * 128, ku * 128, dtype=torch.uint8, device=dev)
    scale = torch.zeros(count, units * 128, ku * (256 // fmt), dtype=torch.uint8, device=dev)
    many = max(1, (1 << 25) // (K * rows))                 # matrices, or rows of one, at a time
    per = rows if many > 1 else max(1, (1 << 25) // K)
    for e in range(0, count, many):
        for r in range(0, rows, per):
            n, m = min(per, rows - r), min(many, count - e)
            q, s, _ = _quantize_plain(torch.randn(m, n, K, generator=gen, device=dev) * 0.02, fmt, g[0])
            q = q.flatten(-2)
            codes[e:e + m, r:r + n, : q.shape[-1] // 2] = q[..., 0::2] | (q[..., 1::2] << 4)
            scale[e:e + m, r:r + n, : s.shape[-1]] = s
    chunk = torch.arange(8, device=dev)[None, :] ^ (torch.arange(128, device=dev)[:, None] & 7)
    c = codes.reshape(count * units, 128, ku, 8, 16).permute(0, 2, 1, 3, 4)
    c = torch.gather(c, 3, chunk[None, None, :, :, None].expand(count * units, ku, 128, 8, 16)).reshape(count * units, ku, -1)
    s = scale.reshape(count * units, 4, 32, ku, 64 // fmt, 4).permute(0, 3, 4, 2, 1, 5).reshape(count * units, ku, -1)
    nb = -(-K // fmt)
    return {"codes": codes[:, :rows, : nb * fmt // 2], "scales": scale[:, :rows, :nb], "g": g, "packed": torch.cat([c, s], dim=2).reshape(-1)}


def _dense(w, fmt, K):
    """The fp32 values of canonical 4-bit weights, [count, rows, K]."""
    c = torch.stack([w["codes"] & 15, w["codes"] >> 4], dim=-1)
    return _values(c.flatten(-2).unflatten(-1, (-1, fmt)), _step_of(w["scales"], fmt, w["g"][:, None, None]))[..., :K]


def _routing(gen, T, E, topk, dropped, dev):
    """Router's choice: the topk largest of N(0,1) logits per token, softmax weights over them; `dropped` per cent of the pairs at -1."""
    val, idx = torch.randn(T, E, generator=gen, device=dev).topk(min(topk, E), dim=1)
    idx = idx.to(torch.int32)
    if dropped:
        idx = torch.where(torch.rand(idx.shape, generator=gen, device=dev) * 100 < dropped, torch.full_like(idx, -1), idx)
    return idx.contiguous(), torch.softmax(val, dim=1).contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    st = {"case": case}
    kind, dt = case["kind"], _DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev).to(dt)

    if kind == "quantize":
        M, K = case["M"], case["K"]
        st["x"], st["values"] = normal(M, K), torch.empty(M, K, dtype=dt, device=dev)
        st["g"] = torch.full((1,), 6.0 / (448 * 6), device=dev) if case["fmt"] == NVFP4 else torch.ones(1, device=dev)
        st["packed"] = torch.empty(-(-M // 128) * -(-K // 256) * (16384 + 32768 // case["fmt"]), dtype=torch.uint8, device=dev)
    elif kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        st["w"] = _weights(gen, case["fmt"], 1, N, K, dev)
        st["x"], st["y"] = normal(M, K), torch.empty(M, N, dtype=dt, device=dev)
        st["g"] = torch.full((1,), 6.0 / (448 * 6), device=dev) if case["fmt"] == NVFP4 else torch.ones(1, device=dev)
    elif kind == "experts":
        T, H, I, E, topk = (case[k] for k in ("T", "H", "I", "E", "topk"))
        for name, rows, K in (("gate", I, H), ("up", I, H), ("down", H, I)):
            st[name] = _weights(gen, case["fmt"], E, rows, K, dev)
        st["x"], st["y"] = normal(T, H), torch.empty(T, H, dtype=dt, device=dev)
        st["g"] = torch.full((1,), 6.0 / (448 * 6), device=dev) if case["fmt"] == NVFP4 else torch.ones(1, device=dev)
        st["gh"] = torch.full((1,), 4.0 / (448 * 6), device=dev) if case["fmt"] == NVFP4 else torch.ones(1, device=dev)
        st["idx"], st["w"] = _routing(gen, T, E, topk, 0, dev)
        st["most"] = int(torch.bincount(st["idx"].flatten().long(), minlength=E).max())
    else:
        T, H, E, topk = (case[k] for k in ("T", "H", "E", "topk"))
        st["idx"], st["w"] = _routing(gen, T, E, topk, case["dropped"], dev)
        topk = st["idx"].shape[1]
        st["x"], st["ys"] = normal(T, H), normal(T * topk, H)
        st["xs"], st["y"] = torch.empty_like(st["ys"]), torch.empty_like(st["x"])
        if case["train"]:
            st["dy"], st["dxs"] = normal(T, H), normal(T * topk, H)
            st["dys"], st["dx"], st["dw"] = torch.empty_like(st["ys"]), torch.empty_like(st["x"]), torch.empty_like(st["w"])
    return st


# ------------------------------------------------------------- one pass

def _own_run(st):
    from paper_2607_00501_b200 import qmm
    case, kind = st["case"], st["case"]["kind"]
    if kind == "quantize":
        g = st["g"] if case["fmt"] == NVFP4 else None
        qmm.mx_quantize(case["fmt"], st["x"], out=st["packed"], tensor_scale=g)
        return qmm.mx_dequantize(case["fmt"], st["packed"], case["M"], case["K"], out=st["values"], tensor_scale=g)
    if kind == "linear":
        g, gw = (st["g"], st["w"]["g"]) if case["fmt"] == NVFP4 else (None, None)
        if "ws" not in st:                                 # the workspace that a program keeps beside its weights
            st["ws"] = torch.zeros(qmm.mx_linear_workspace_bytes(case["fmt"], case["M"], case["N"], case["K"]), dtype=torch.uint8, device=st["x"].device)
        return qmm.mx_linear(case["fmt"], st["x"], st["w"]["packed"], case["N"], Y=st["y"], x_scale=g, w_scale=gw, ws=st["ws"])
    if kind == "experts":
        scales = {}
        if case["fmt"] == NVFP4:
            scales = {"x_scale": st["g"], "gate_scale": st["gate"]["g"], "up_scale": st["up"]["g"], "down_scale": st["down"]["g"], "h_scale": st["gh"]}
        args = qmm.mx_moe_args(case["fmt"], st["x"], st["idx"], st["w"], st["gate"]["packed"], st["up"]["packed"], st["down"]["packed"],
                               case["I"], case["E"], st["y"], **scales)
        if "ws" not in st:
            st["ws"] = torch.zeros(qmm.mx_moe_workspace_bytes(args), dtype=torch.uint8, device=st["x"].device)
        qmm.mx_moe_run(args, st["ws"])
        return st["y"]
    if "plan" not in st:                                   # the plan's buffers; every pass sorts into them anew
        st["plan"] = qmm.ExpertPlan(case["T"], st["idx"].shape[1], case["E"])
    plan = qmm.expert_sort(st["idx"], case["E"], out=st["plan"])
    xs = qmm.expert_gather(st["x"], plan, out=st["xs"])
    y = qmm.expert_combine(st["ys"], plan, st["w"], out=st["y"])
    out = {"order": plan.order, "offsets": plan.offsets, "xs": xs, "y": y}
    if case["train"]:
        out["dys"], out["dw"] = qmm.expert_combine_grad(st["dy"], st["ys"], plan, st["w"], dys=st["dys"], dw=st["dw"])
        out["dx"] = qmm.expert_gather_grad(st["dxs"], plan, out=st["dx"])
    return out


def _sorted_plain(idx, E):
    """order [P] (-1 past the routed pairs), offsets [E + 1], place [P] (-1: dropped) of the pairs' stable order by expert."""
    flat = idx.flatten().long()
    P = flat.numel()
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    sorted_key, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(sorted_key, torch.arange(E + 1, device=flat.device))
    at = torch.arange(P, device=flat.device)
    place = torch.empty_like(order).scatter_(0, order, torch.where(sorted_key < E, at, torch.full_like(at, -1)))
    return torch.where(sorted_key < E, order, torch.full_like(order, -1)), offsets, place


def _rows(x, index):
    """x[index] as fp32, zeros where index < 0."""
    return torch.where((index >= 0)[:, None], x[index.clamp(min=0)].float(), torch.zeros((), device=x.device))


def run(state):
    if own:
        return _own_run(state)
    st = state
    case, kind = st["case"], st["case"]["kind"]
    if kind == "quantize":
        return _through_4_bits(st["x"].float(), case["fmt"], st["g"]).to(st["x"].dtype)
    if kind == "linear":
        x = _through_4_bits(st["x"].float(), case["fmt"], st["g"])
        return (x @ _dense(st["w"], case["fmt"], case["K"])[0].T).to(st["x"].dtype)
    if kind == "experts":
        fmt, T, H, I, E = (case[k] for k in ("fmt", "T", "H", "I", "E"))
        order, offsets, place = _sorted_plain(st["idx"], E)
        topk, most = st["idx"].shape[1], st["most"]

        x = _through_4_bits(st["x"].float(), fmt, st["g"])
        at = torch.arange(most, device=order.device)[None, :] + offsets[:E, None]                  # [E, most]: sorted rows of each expert
        inside = at < offsets[1:, None]
        pair = order[at.clamp(max=order.numel() - 1)]
        rows = x[pair // topk] * inside[..., None]
        g = rows @ _dense(st["gate"], fmt, H).transpose(1, 2)
        u = rows @ _dense(st["up"], fmt, H).transpose(1, 2)
        h = _through_4_bits(g / (1.0 + torch.exp(-g)) * u, fmt, st["gh"])
        d = h @ _dense(st["down"], fmt, I).transpose(1, 2)
        flat = torch.zeros(order.numel(), H, device=x.device)
        flat[pair[inside]] = d[inside]
        return (flat.reshape(T, topk, H) * st["w"][..., None]).sum(1).to(st["x"].dtype)
    T, topk = st["idx"].shape
    order, offsets, place = _sorted_plain(st["idx"], case["E"])
    dt = st["x"].dtype
    token = torch.where(order >= 0, order // topk, order)
    xs = _rows(st["x"], token).to(dt)
    w = torch.where(place.reshape(T, topk) >= 0, st["w"], torch.zeros((), device=st["w"].device))
    back = _rows(st["ys"], place).reshape(T, topk, -1)
    out = {"order": order.int(), "offsets": offsets.int(), "xs": xs, "y": (back * w[..., None]).sum(1).to(dt)}
    if case["train"]:
        dy = st["dy"].float()
        wr = torch.where(order >= 0, st["w"].flatten()[order.clamp(min=0)], torch.zeros((), device=dy.device))
        out["dys"] = (_rows(st["dy"], token) * wr[:, None]).to(dt)
        out["dw"] = (back * dy[:, None, :]).sum(2)
        out["dx"] = _rows(st["dxs"], place).reshape(T, topk, -1).sum(1).to(dt)
    return out


# ------------------------------------------------------------------ work

def _q_bytes(rows, K, fmt):
    return rows * K // 2 + rows * -(-K // fmt)


def work(case):
    kind, size = case["kind"], _SIZE[case["dtype"]]
    if kind == "quantize":
        n = case["M"] * case["K"]
        return {"bytes": 2 * n * size + 2 * _q_bytes(case["M"], case["K"], case["fmt"]), "flops": 4 * n}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M * K + M * N) * size + _q_bytes(N, K, case["fmt"]), "flops": 2 * M * N * K}
    if kind == "experts":
        T, H, I, E, fmt = (case[k] for k in ("T", "H", "I", "E", "fmt"))
        topk = min(case["topk"], E)
        used = E * (1 - (1 - topk / E) ** T)               # experts that get a token, on average
        per = 2 * _q_bytes(I, H, fmt) + _q_bytes(H, I, fmt)
        return {"bytes": int(used * per) + 2 * T * H * size + 8 * T * topk, "flops": 6 * T * topk * H * I}
    T, H, P = case["T"], case["H"], case["T"] * min(case["topk"], case["E"])
    rows = (T + P) + (P + T)                               # x -> xs, ys -> y
    flops = 2 * P * H
    if case["train"]:
        rows += (T + P + P) + (P + T)                      # dy, ys -> dys, dw; dxs -> dx
        flops += 4 * P * H
    return {"bytes": rows * H * size + P * 16, "flops": flops}


# ----------------------------------------------- the definition in 64 bits

def _f32(x):
    return x.to(torch.float32).double()                    # a quotient or product that the definition rounds to fp32


def _exact_values(x, fmt, g):
    """float64 [..., K] -> the values of its 4-bit codes, from the definition: nearest multiple of the step of the binade."""
    k = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -k % fmt)).unflatten(-1, (-1, fmt))
    top = x.abs().max(-1, keepdim=True).values
    if fmt == 32:
        d = torch.exp2((torch.frexp(top).exponent - 1 - 2).clamp(-127, 127).double())
        r = (x / d).abs()
    else:
        s = _f32(top / _f32(6.0 * g.double())).clamp(max=448.0)
        grid = torch.exp2((torch.frexp(s).exponent - 1).clamp(min=-6).double() - 3)
        d = _f32(torch.round(s / grid) * grid * g.double())
        r = torch.where(d > 0, _f32(x / torch.where(d > 0, d, torch.ones_like(d))).abs(), torch.zeros_like(x))
    unit = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)).double()
    v = (torch.round(r / unit) * unit).clamp(max=6.0) * torch.sign(x) * d
    return v.flatten(-2)[..., :k]


def _exact_dense(codes, scales, g, fmt, K):
    mag = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=codes.device) / 2
    lo, hi = codes & 15, codes >> 4
    v = torch.stack([mag[(c & 7).long()] * (1 - 2 * (c >> 3).double()) for c in (lo, hi)], dim=-1).flatten(-2)
    if fmt == 32:
        d = torch.exp2(scales.double() - 127)
    else:
        e, m = (scales >> 3 & 15).double(), (scales & 7).double()
        d = _f32(torch.where(e > 0, torch.exp2(e - 7) * (1 + m / 8), m * 2.0 ** -9) * g.double())
    return (v.unflatten(-1, (-1, fmt)) * d[..., None]).flatten(-2)[..., :K]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return _exact_values(st["x"].double(), case["fmt"], st["g"])
    if kind == "linear":
        w = st["w"]
        x = _exact_values(st["x"].double(), case["fmt"], st["g"])
        out = torch.empty(case["M"], case["N"], dtype=torch.float64, device=x.device)
        for n in range(0, case["N"], 16384):
            out[:, n:n + 16384] = x @ _exact_dense(w["codes"][0, n:n + 16384], w["scales"][0, n:n + 16384], w["g"], case["fmt"], case["K"]).T
        return out
    if kind == "experts":
        fmt, H, I = case["fmt"], case["H"], case["I"]
        x = _exact_values(st["x"].double(), fmt, st["g"])
        out = torch.zeros(case["T"], H, dtype=torch.float64, device=x.device)
        for e in range(case["E"]):
            t, j = torch.nonzero(st["idx"] == e, as_tuple=True)
            if t.numel() == 0:
                continue
            mat = lambda m, K: _exact_dense(m["codes"][e], m["scales"][e], m["g"][e], fmt, K)  # noqa: E731
            g, u = x[t] @ mat(st["gate"], H).T, x[t] @ mat(st["up"], H).T
            d = _exact_values(g * torch.sigmoid(g) * u, fmt, st["gh"]) @ mat(st["down"], I).T
            out.index_add_(0, t, d * st["w"][t, j].double()[:, None])
        return out
    idx, w, E = st["idx"].cpu(), st["w"].double(), case["E"]
    T, topk = idx.shape
    pairs = sorted((int(e), p) for p, e in enumerate(idx.flatten().tolist()) if 0 <= e < E)
    order = torch.full((T * topk,), -1, dtype=torch.int32)
    order[: len(pairs)] = torch.tensor([p for _, p in pairs], dtype=torch.int32)
    offsets = torch.tensor([sum(1 for q, _ in pairs if q < e) for e in range(E + 1)] if len(pairs) < 2000 else
                           torch.cumsum(torch.bincount(torch.tensor([q + 1 for q, _ in pairs]), minlength=E + 1), 0).tolist(), dtype=torch.int32)
    pair = torch.tensor([p for _, p in pairs], dtype=torch.long, device=w.device)
    n, x64, ys = len(pairs), st["x"].double(), st["ys"].double()
    zero = torch.zeros(T * topk, case["H"], dtype=torch.float64, device=w.device)
    xs, y = zero.clone(), torch.zeros_like(x64)
    xs[:n] = x64[pair // topk]
    y.index_add_(0, pair // topk, ys[:n] * w.flatten()[pair][:, None])
    out = {"order": order, "offsets": offsets, "xs": xs, "y": y}
    if case["train"]:
        dy = st["dy"].double()
        dys, dw, dx = zero.clone(), torch.zeros(T * topk, dtype=torch.float64, device=w.device), torch.zeros_like(x64)
        dys[:n] = dy[pair // topk] * w.flatten()[pair][:, None]
        dw[pair] = (dy[pair // topk] * ys[:n]).sum(1)
        dx.index_add_(0, pair // topk, st["dxs"].double()[:n])
        out.update(dys=dys, dw=dw.reshape(T, topk), dx=dx)
    return out
