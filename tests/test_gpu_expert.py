"""GPU parity: tokens sorted by expert and back, their gradients, and the routed layer on microscaled operands."""
import numpy as np
import pytest
import torch

from tests import mxref
from tests.test_gpu_mx import DTYPES, HALF_ULP, check_product, f64, scale_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def routing(T, topk, E, kind, seed):
    rng = np.random.default_rng(seed)
    idx = rng.integers(0, E, (T, topk))
    if kind == "dropped":
        idx = np.where(rng.random((T, topk)) < 0.2, rng.choice([-1, E, 2**31 - 1, -2**31], (T, topk)), idx)
    elif kind == "one":
        idx[:] = E - 1
    elif kind == "none":
        idx[:] = -1
    elif kind == "skewed":
        idx = np.where(rng.random((T, topk)) < 0.7, 0, idx)
    return idx.astype(np.int32)


def check_plan(plan, idx, E):
    order, place, offsets, units = mxref.sort(idx, E)
    for got, want in ((plan.order, order), (plan.place, place), (plan.offsets, offsets), (plan.units, units)):
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("kind", ["uniform", "dropped", "one", "none", "skewed"])
@pytest.mark.parametrize("T,topk,E", [(1, 1, 1), (1, 8, 128), (4, 8, 128), (31, 1, 3), (512, 2, 16), (513, 2, 318), (1024, 8, 128), (8193, 1, 1024),
                                      (3000, 3, 319), (8192, 8, 128), (20000, 6, 160), (40, 32, 1024), (50000, 4, 500)])
def test_sort(qmm, kind, T, topk, E):
    idx = routing(T, topk, E, kind, T + E)
    plan = qmm.expert_sort(torch.from_numpy(idx).cuda(), E)
    check_plan(plan, idx, E)
    idx2 = routing(T, topk, E, "dropped", 5)                                       # the same buffers again
    check_plan(qmm.expert_sort(torch.from_numpy(idx2).cuda(), E, out=plan), idx2, E)


def test_sort_of_no_tokens(qmm):
    plan = qmm.expert_sort(torch.empty(0, 4, dtype=torch.int32, device="cuda"), 9)
    assert not plan.offsets.any() and not plan.units.any()


def rows_of(T, topk, H, dt, seed, pitch=None, off=0):
    gen = torch.Generator().manual_seed(seed)

    def make(rows):
        x = torch.randn(rows, H, generator=gen).to(dt)
        if pitch is None:
            return x.cuda()
        buf = torch.full((rows * pitch + off + 8,), 7.0, dtype=dt, device="cuda")
        v = buf[off: off + rows * pitch].view(rows, pitch)[:, :H]
        v.copy_(x)
        return v
    return make(T), make(T * topk), make(T), make(T * topk)


@pytest.mark.parametrize("dt", list(DTYPES))
@pytest.mark.parametrize("kind", ["uniform", "dropped", "none"])
@pytest.mark.parametrize("T,topk,E,H,pitch,off", [(1, 1, 1, 1, None, 0), (5, 2, 3, 64, None, 0), (61, 8, 128, 2048, None, 0), (300, 3, 7, 1001, 1003, 1),
                                                  (200, 11, 16, 130, 136, 8), (33, 32, 64, 500, 512, 2), (40, 4, 8, 4096, None, 0)])
def test_moves_and_gradients(qmm, dt, kind, T, topk, E, H, pitch, off):
    dtype = DTYPES[dt]
    idx = routing(T, topk, E, kind, T)
    plan = qmm.expert_sort(torch.from_numpy(idx).cuda(), E)
    order, place, _, _ = mxref.sort(idx, E)
    x, ys, dy, dxs = rows_of(T, topk, H, dtype, T + H, pitch, off)
    w = torch.rand(T, topk, generator=torch.Generator().manual_seed(3)) * 2 - 0.5
    w[0, 0] = 0
    dropped = torch.from_numpy(place.reshape(T, topk) < 0)
    wn = w.clone()
    wn[dropped] = float("nan")                                                     # a dropped pair's weight is not read
    wd = wn.cuda()
    kept = order >= 0
    token = np.where(kept, order, 0) // topk

    # copies are exact; a weighted copy is the fp32 product rounded once
    xs = qmm.expert_gather(x, plan)
    assert np.array_equal(f64(xs), np.where(kept[:, None], f64(x)[token], 0))
    xw = qmm.expert_gather(x, plan, weights=wd)
    want = (x.float().cpu()[token] * w.reshape(-1)[np.where(kept, order, 0)][:, None]).to(dtype)
    assert np.array_equal(f64(xw), np.where(kept[:, None], f64(want), 0))

    # sums of topk fp32 terms: topk + 1 roundings of 2^-24 of sum |w y|, then the output's own
    rows = np.where(place >= 0, place, 0).reshape(T, topk)
    mask = (place >= 0).reshape(T, topk)[..., None]

    def check_sum(got, terms):
        ref = terms.sum(1)
        tol = (topk + 1) * 2.0**-24 * np.abs(terms).sum(1) + HALF_ULP[dtype] * 1.001 * np.abs(ref) + (2.0**-25 if dtype == torch.float16 else 0)
        assert (np.abs(f64(got) - ref) <= tol).all()
    w64 = np.where(mask[..., 0], f64(w), 0)
    check_sum(qmm.expert_combine(ys, plan, wd), np.where(mask, f64(ys)[rows], 0) * w64[..., None])
    check_sum(qmm.expert_combine(ys, plan), np.where(mask, f64(ys)[rows], 0))
    check_sum(qmm.expert_gather_grad(dxs, plan), np.where(mask, f64(dxs)[rows], 0))

    # gradients of the weighted sum.  A dot product over H <= 4096 runs through at most 2 * 8 (thread) + 5 (warp) + 8
    # (block) additions with 16-byte vectors, 16 + 13 with single elements: 40 roundings of 2^-24 of sum |dy ys| cover both
    dys, dw = qmm.expert_combine_grad(dy, ys, plan, wd)
    want = (dy.float().cpu()[token] * w.reshape(-1)[np.where(kept, order, 0)][:, None]).to(dtype)
    assert np.array_equal(f64(dys), np.where(kept[:, None], f64(want), 0))
    prod = np.where(mask, f64(ys)[rows], 0) * f64(dy)[:, None, :]
    assert (np.abs(f64(dw) - prod.sum(2)) <= 40 * 2.0**-24 * np.abs(prod).sum(2)).all()
    assert not f64(dw)[~mask[..., 0]].any()
    again = qmm.expert_combine_grad(dy, ys, plan, wd)
    assert torch.equal(again[0], dys) and torch.equal(again[1], dw)


def test_gradients_against_differences(qmm):
    """The weighted sum is linear in ys and in w, the gather in x: differences of the loss over whole steps are the gradients,
    up to the fp32 rounding of the sums (2^-20 of the sum of magnitudes is far above it)."""
    T, topk, E, H = 6, 3, 4, 40
    idx = routing(T, topk, E, "dropped", 2)
    plan = qmm.expert_sort(torch.from_numpy(idx).cuda(), E)
    x, ys, dy, dxs = rows_of(T, topk, H, torch.float32, 1)
    w = torch.rand(T, topk, device="cuda")
    dys, dw = qmm.expert_combine_grad(dy, ys, plan, w)
    dx = qmm.expert_gather_grad(dxs, plan)
    loss = lambda ys_, w_: float((qmm.expert_combine(ys_, plan, w_).double() * dy.double()).sum())  # noqa: E731
    tol = 2.0**-20 * float(ys.abs().sum() * dy.abs().max() + 1)
    for t in range(T):
        for j in range(topk):
            up, dn = w.clone(), w.clone()
            up[t, j] += 1
            dn[t, j] -= 1
            assert abs((loss(ys, up) - loss(ys, dn)) / 2 - float(dw[t, j])) <= tol
    rng = np.random.default_rng(0)
    for _ in range(20):
        r, h = int(rng.integers(T * topk)), int(rng.integers(H))
        up, dn = ys.clone(), ys.clone()
        up[r, h] += 1
        dn[r, h] -= 1
        assert abs((loss(up, w) - loss(dn, w)) / 2 - float(dys[r, h])) <= tol
        t = int(rng.integers(T))
        up, dn = x.clone(), x.clone()
        up[t, h] += 1
        dn[t, h] -= 1
        g = lambda x_: float((qmm.expert_gather(x_, plan).double() * dxs.double()).sum())  # noqa: E731
        assert abs((g(up) - g(dn)) / 2 - float(dx[t, h])) <= 2.0**-20 * float(x.abs().sum() * dxs.abs().max() * topk + 1)


def expert_weights(fmt, E, N, K, seed, g):
    """Packed matrices [E], their float64 values [E, N, K] and tensor scales."""
    x = torch.randn(E, N, K, generator=torch.Generator().manual_seed(seed)) * 0.1
    from paper_2607_00501_b200 import qmm
    gs = [g * (1 + 0.25 * e) for e in range(E)]
    packed = torch.cat([qmm.mx_quantize(fmt, x[e].cuda(), tensor_scale=scale_of(fmt, gs[e])) for e in range(E)])
    vals = np.stack([mxref.values(*mxref.quantize(f64(x[e]), fmt, gs[e]), fmt, K, gs[e]) for e in range(E)])
    return packed, vals, None if fmt == mxref.MXFP4 else torch.tensor(gs, device="cuda")


@pytest.mark.parametrize("rows", [None, "64", "128"])
@pytest.mark.parametrize("fmt", [mxref.MXFP4, mxref.NVFP4])
@pytest.mark.parametrize("T,topk,E,H,I,kind", [(1, 1, 1, 32, 32, "uniform"), (1, 4, 16, 256, 128, "uniform"), (3, 8, 16, 320, 96, "dropped"), (40, 2, 4, 512, 384, "skewed"),
                                               (300, 2, 3, 300, 200, "uniform"), (700, 1, 2, 256, 640, "one"), (5, 2, 4, 64, 64, "none"), (400, 2, 3, 257, 90, "dropped"), (90, 3, 5, 131, 70, "uniform")])
def test_expert_products(qmm, fmt, rows, T, topk, E, H, I, kind):
    qmm.debug_config("mx_tile", rows)                                              # weight rows per tile: the plan's, or each of them
    idx = routing(T, topk, E, kind, T + E)
    order, place, offsets, units = mxref.sort(idx, E)
    idx_d = torch.from_numpy(idx).cuda()
    plan = qmm.expert_sort(idx_d, E)
    X = torch.randn(T, H, generator=torch.Generator().manual_seed(1)).half().cuda()
    gx, gh = (1.0, 1.0) if fmt == mxref.MXFP4 else (0.003, 0.0017)
    gate, vg, sg = expert_weights(fmt, E, I, H, 2, 0.0004)
    up, vu, su = expert_weights(fmt, E, I, H, 3, 0.0005)
    down, vd, sd = expert_weights(fmt, E, H, I, 4, 0.0003)

    # rows grouped by expert, quantised bit for bit
    xq = torch.full((qmm.mx_experts_bytes(fmt, T, topk, E, H),), 0xFF, dtype=torch.uint8, device="cuda")
    qmm.mx_quantize_experts(fmt, X, idx_d, plan, out=xq, tensor_scale=scale_of(fmt, gx))
    codes, scale = mxref.quantize(f64(X), fmt, gx)
    for e in range(E):
        n = int(offsets[e + 1] - offsets[e])
        if n:
            c, s = mxref.unpack(xq.cpu().numpy(), fmt, n, H, int(units[e]))
            tok = order[offsets[e]: offsets[e + 1]] // topk
            assert np.array_equal(s[:, : scale.shape[1]], scale[tok]) and np.array_equal(np.where(c == 8, 0, c)[:, : scale.shape[1] * fmt],
                                                                                        np.where(codes == 8, 0, codes)[tok].reshape(n, -1))

    # gate / up: the stored block is the quantisation of the exact h up to the fp32 roundings of the two products and of silu (relative
    # 2^-17 of the products' sums of magnitudes and of h): every stored value is within half a gap of its grid of the exact one
    h = qmm.mx_experts_gate_up(fmt, xq, plan, gate, up, I, H, h=torch.full((qmm.mx_experts_bytes(fmt, T, topk, E, I),), 0xFF, dtype=torch.uint8, device="cuda"),
                               a_scale=scale_of(fmt, gx), gate_scale=sg, up_scale=su, h_scale=scale_of(fmt, gh))
    Y = qmm.mx_experts_gemm(fmt, h, plan, down, H, I, a_scale=scale_of(fmt, gh), w_scale=sd, dtype=torch.float32)
    xv = mxref.values(codes, scale, fmt, H, gx)
    for e in range(E):
        n = int(offsets[e + 1] - offsets[e])
        if not n:
            continue
        a = xv[order[offsets[e]: offsets[e + 1]] // topk]
        G, U = a @ vg[e].T, a @ vu[e].T
        hv = mxref.silu(G) * U
        slack = 2.0**-17 * (1.1 * (np.abs(a) @ np.abs(vg[e]).T) * np.abs(U) + np.abs(mxref.silu(G)) * (np.abs(a) @ np.abs(vu[e]).T)) + 2.0**-17 * np.abs(hv)
        c, s = mxref.unpack(h.cpu().numpy(), fmt, n, I, int(units[e]))
        nb = -(-I // fmt)
        assert not s[:, nb:].any() and not c[:, nb * fmt:].any() and not c[:, I:].any()
        D = mxref.step(s[:, :nb], fmt, gh)
        hb, sl = mxref.blocks_of(hv, fmt), mxref.blocks_of(slack, fmt)
        lo = mxref.quantize((np.sign(hb) * np.maximum(np.abs(hb) - sl, 0)).reshape(n, -1), fmt, gh)[1]
        hi = mxref.quantize((np.sign(hb) * (np.abs(hb) + sl)).reshape(n, -1), fmt, gh)[1]
        assert ((lo <= s[:, :nb]) & (s[:, :nb] <= hi)).all()
        v = mxref.VALUE[c[:, : nb * fmt]].reshape(n, nb, fmt)
        q = hb / np.where(D > 0, D, 1)[..., None]
        gap = np.where(np.abs(q) < 2, 0.25, np.where(np.abs(q) < 4, 0.5, 1.0)) + sl / np.where(D > 0, D, 1)[..., None] + 1e-6
        ok = (np.abs(v - q) <= gap) | (np.abs(q) > 6) & (np.abs(v) == 6) | (D == 0)[..., None]
        assert ok.all()
        # down, from the codes as stored
        hq = mxref.values(c[:, : nb * fmt].reshape(n, nb, fmt), s[:, :nb], fmt, I, gh)
        check_product(Y[int(offsets[e]): int(offsets[e + 1])], hq, vd[e], I)

    # the whole layer is the sequence of its parts, bit for bit
    w = torch.rand(T, topk, device="cuda")
    out = torch.empty(T, H, dtype=torch.float16, device="cuda")
    args = qmm.mx_moe_args(fmt, X, idx_d, w, gate, up, down, I, E, out, x_scale=scale_of(fmt, gx), gate_scale=sg, up_scale=su, down_scale=sd, h_scale=scale_of(fmt, gh))
    ws = torch.zeros(qmm.mx_moe_workspace_bytes(args), dtype=torch.uint8, device="cuda")
    qmm.mx_moe_run(args, ws)
    qmm.status_check(ws)
    Y16 = torch.zeros(T * topk, H, dtype=torch.float16, device="cuda")
    qmm.mx_experts_gemm(fmt, h, plan, down, H, I, Y=Y16, a_scale=scale_of(fmt, gh), w_scale=sd)
    assert torch.equal(out, qmm.expert_combine(Y16, plan, w))
    out2 = out.clone()
    qmm.mx_moe_run(args, ws)
    assert torch.equal(out, out2)


def test_layer_with_strided_bf16_rows(qmm):
    fmt, T, topk, E, H, I = mxref.MXFP4, 50, 2, 4, 288, 160
    idx = torch.from_numpy(routing(T, topk, E, "dropped", 1)).cuda()
    gate, _, _ = expert_weights(fmt, E, I, H, 2, 1.0)
    up, _, _ = expert_weights(fmt, E, I, H, 3, 1.0)
    down, _, _ = expert_weights(fmt, E, H, I, 4, 1.0)
    w = torch.rand(T, topk, device="cuda")
    X = torch.randn(T, H, device="cuda").bfloat16()
    want = qmm.mx_moe(fmt, X, idx, w, gate, up, down, I, E)
    buf = torch.full((T, H + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    Xs = torch.zeros(T, H + 5, dtype=torch.bfloat16, device="cuda")[:, 1: H + 1]
    Xs.copy_(X)
    qmm.mx_moe(fmt, Xs, idx, w, gate, up, down, I, E, out=buf[:, :H])
    assert torch.equal(buf[:, :H], want) and bool((buf[:, H:] == 7).all())


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_example_layer(qmm, fmt):
    """The example serves a layer and trains through the moves.  Two 4-bit operands per product, each off by a relative rms of about
    0.12 (the e2m1 grid under one scale per block): sqrt(2) * 0.12 per product, two products in sequence and the product g u in between
    leave about 0.35 (0.45 with the spread of a single token); the gradients differ by the order of fp32 sums."""
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("mx_moe_layer", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mx_moe_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for tokens in (1, 64, 300):
        served, trained = example.main(["--tokens", str(tokens), "--fmt", fmt])
        assert 0 < served < 0.45 and trained < 1e-5


def test_offsets_past_32_bits(qmm):
    T, topk, H = 4, 1, 64
    pitch = (1 << 30) + 8
    plan = qmm.expert_sort(torch.tensor([[3], [0], [1], [2]], dtype=torch.int32, device="cuda"), 4)
    big = [torch.empty(3 * pitch + 64, dtype=torch.float16, device="cuda").as_strided((4, H), (pitch, 1)) for _ in range(3)]
    x, dy = torch.randn(T, H, device="cuda").half(), torch.randn(T, H, device="cuda").half()
    w = torch.rand(T, topk, device="cuda")
    big[0].copy_(x)
    xs = qmm.expert_gather(big[0], plan, out=big[1])
    assert torch.equal(xs, qmm.expert_gather(x, plan))
    assert torch.equal(qmm.expert_combine(big[1], plan, w, out=big[2]), qmm.expert_combine(xs.contiguous(), plan, w))
    dys, dw = qmm.expert_combine_grad(dy, big[1], plan, w, dys=big[2])
    dys2, dw2 = qmm.expert_combine_grad(dy, xs.contiguous(), plan, w)
    assert torch.equal(dys, dys2) and torch.equal(dw, dw2)
