"""Calls of the router, the norm and the adapters as programs make them: other streams, captured and replayed, shared workspaces, long offsets, one after the other, the example."""
import math

import pytest
import torch

from tests import layerref as ref
from tests.test_gpu_lora import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def step(qmm, s):
    """One pass of everything over the tensors of s, into its buffers."""
    qmm.expert_route(s["logits"], 4, qmm.SIGMOID, bias=s["bias"], groups=4, top_groups=2, group_top=2, idx=s["idx"], weights=s["w"])
    qmm.expert_route_grad(s["dw"], s["logits"], s["idx"], qmm.SIGMOID, out=s["dl"])
    qmm.rms_norm_rows(s["x"], s["weight"], residual=s["r"], h=s["h"], codes=s["codes"], scales=s["scales"], y=s["y"])
    qmm.lora(s["codes"], s["who"], s["a"], s["b"], s["y0"], scale=s["scale"], x_scale=s["scales"], s=s["s"], ws=s["ws"], out=s["out"])
    qmm.lora_grad(s["dy"], s["codes"], s["s"], s["who"], s["a"], s["b"], s["dx0"], scale=s["scale"], x_scale=s["scales"], ws=s["ws"], dx=s["dx"], da=s["da"], db=s["db"])
    qmm.rms_norm_grad(s["dx"], s["h"], s["weight"], dx=s["dh"], dweight=s["dweight"], ws=s["ws2"])
    return [s[k] for k in ("idx", "w", "dl", "h", "y", "scales", "s", "out", "dx", "da", "db", "dh", "dweight")]


def tensors(qmm, T, seed, share=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, K, N, n, r, E = torch.bfloat16, 264, 200, 5, 16, 32
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    e = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    s = dict(logits=f(T, E), bias=f(E) * 0.1, dw=f(T, 4), x=f(T, K).to(dt), r=f(T, K).to(dt), weight=f(K).to(dt), a=(f(n, r, K) / 16).to(dt), b=f(n, N, r).to(dt), scale=f(n),
             who=torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32), y0=f(T, N).to(dt), dy=f(T, N).to(dt), dx0=f(T, K).to(dt))
    s.update(idx=e(T, 4, dtype=torch.int32), w=e(T, 4, dtype=torch.float32), dl=e(T, E, dtype=torch.float32), h=e(T, K), y=e(T, K), codes=e(T, K, dtype=torch.float8_e4m3fn),
             scales=e(T, dtype=torch.float32), s=torch.zeros(T, r, device="cuda"), out=e(T, N), dx=e(T, K), da=e(n, r, K, dtype=torch.float32), db=e(n, N, r, dtype=torch.float32),
             dh=e(T, K), dweight=e(K, dtype=torch.float32))
    s["ws"] = share["ws"] if share else torch.empty(qmm.lora_workspace_bytes(T, n, r), dtype=torch.uint8, device="cuda")
    s["ws2"] = share["ws2"] if share else torch.empty(qmm.rms_norm_grad_workspace_bytes(T, K), dtype=torch.uint8, device="cuda")
    return s


@pytest.mark.parametrize("T", [40, 700])
def test_other_streams_and_graphs_that_share_workspaces(qmm, T):
    one = tensors(qmm, T, 1)
    two = tensors(qmm, T, 2, share=one)
    want = [[t.clone() for t in step(qmm, s)] for s in (one, two)]
    stream = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(stream):
        for s, w in zip((one, two), want):
            for t in step(qmm, s):
                t.record_stream(stream)
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(step(qmm, s), w))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                step(qmm, s)
            graphs.append(g)
        for i in (0, 1, 1, 0):
            s = (one, two)[i]
            for t in (s["out"], s["dx"], s["da"], s["w"], s["y"]):
                t.zero_()
            graphs[i].replay()
            stream.synchronize()
            got = [s[k] for k in ("idx", "w", "dl", "h", "y", "scales", "s", "out", "dx", "da", "db", "dh", "dweight")]
            assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
        # other inputs in the same places: the replay reads them, other adapters among them
        fresh = tensors(qmm, T, 3)
        for k in ("logits", "x", "who", "a", "dy"):
            one[k].copy_(fresh[k])
        graphs[0].replay()
        stream.synchronize()
        got = [one[k].clone() for k in ("idx", "out", "dx", "da", "dweight")]
        step(qmm, one)
        stream.synchronize()
        assert all(torch.equal(a, one[k]) for a, k in zip(got, ("idx", "out", "dx", "da", "dweight")))


def test_offsets_past_32_bits(qmm):
    """Three rows that lie 1.2e9 elements apart."""
    pitch, T, K, N = 1_200_000_000, 3, 96, 64
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    big = torch.empty(2 * pitch + 512, dtype=torch.float16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)

    def far(at, cols, v=None):
        t = big.as_strided((T, cols), (pitch, 1), at)
        if v is not None:
            t.copy_(v)
        return t
    x, y0 = torch.randn(T, K, generator=gen, device="cuda").half(), torch.randn(T, N, generator=gen, device="cuda").half()
    a, b = torch.randn(2, 8, K, generator=gen, device="cuda").half() / 8, torch.randn(2, N, 8, generator=gen, device="cuda").half()
    idx = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    want = qmm.lora(x, idx, a, b, y0)
    assert torch.equal(qmm.lora(far(0, K, x), idx, a, b, far(128, N, y0), out=far(128, N)), want) and torch.equal(far(128, N), want)
    yn, xn = qmm.rms_norm(x)[0], far(0, K, x)
    assert torch.equal(qmm.rms_norm(xn, y=far(0, K))[0], yn)
    l = torch.randn(T, 64, generator=gen, device="cuda").half()
    i1, w1 = qmm.expert_route(l, 4)
    i2, w2 = qmm.expert_route(far(0, 64, l), 4)
    assert torch.equal(i1, i2) and torch.equal(w1, w2)
    codes, scales = qmm.rows_quantize(far(0, K, x))
    c2, s2 = qmm.rows_quantize(x)
    assert torch.equal(codes.view(torch.uint8), c2.view(torch.uint8)) and torch.equal(scales, s2)
    dx, da, db = qmm.lora_grad(y0, x, torch.ones(T, 8, device="cuda"), idx, a, b)
    dx2, da2, db2 = qmm.lora_grad(far(128, N, y0), far(0, K, x), torch.ones(T, 8, device="cuda"), idx, a, b, dx=far(300, K))
    assert torch.equal(dx, dx2) and torch.equal(da, da2) and torch.equal(db, db2)


def test_many_rows_far_apart(qmm):
    """The two-launch form with rows 4e6 elements apart: 2.4e9 elements between the first and the last."""
    pitch, T, K, N = 4_000_000, 600, 64, 64
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    big = torch.empty((T - 1) * pitch + 512, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, y0 = torch.randn(T, K, generator=gen, device="cuda").bfloat16(), torch.randn(T, N, generator=gen, device="cuda").bfloat16()
    a, b = (torch.randn(3, 16, K, generator=gen, device="cuda") / 8).bfloat16(), torch.randn(3, N, 16, generator=gen, device="cuda").bfloat16()
    idx = torch.randint(-1, 3, (T,), generator=gen, device="cuda", dtype=torch.int32)
    s = torch.zeros(T, 16, device="cuda")
    want = qmm.lora(x, idx, a, b, y0, s=s)
    far = lambda at: big.as_strided((T, 64), (pitch, 1), at)  # noqa: E731
    fx, fy, fo = far(0), far(64), far(128)
    fx.copy_(x), fy.copy_(y0)
    assert torch.equal(qmm.lora(fx, idx, a, b, fy, out=fo), want) and torch.equal(fo, want)
    grads = qmm.lora_grad(y0, x, s, idx, a, b, x)
    assert all(torch.equal(p, q) for p, q in zip(grads, qmm.lora_grad(fy, fx, s, idx, a, b, fx, dx=fo)))


def test_norm_into_adapters_beside_a_frozen_product(qmm):
    """rms_norm into 16 and 8 bits at once, the 4-bit product of the one, the adapters on the other, in place beside it; all of it back."""
    for T in (30, 600):
        p = Problem(qmm, "bf16", T, 512, 384, 3, 16, "dropped")
        weight = torch.randn(512, device="cuda").bfloat16()
        y = torch.empty_like(p.x)
        codes, scales, h = qmm.rms_norm_rows(p.x, weight, residual=p.dx0, y=y)
        packed = qmm.mx_quantize(qmm.MXFP4, torch.randn(384, 512, device="cuda") * 0.05)
        base = qmm.mx_linear(qmm.MXFP4, y, packed, 384)
        p.x, p.x_scale, p.x64 = codes, scales, codes.double() * scales.double()[:, None]
        y0 = base.clone()
        p.check_forward(p.forward(y0=base, out=base), y0)
        dx0 = (p.dy.float() @ qmm.mx_dequantize(qmm.MXFP4, packed, 384, 512)).bfloat16()
        dx, da, db = p.backward(dx0=dx0, dx=None)
        p.check_backward(dx, da, db, dx0)
        from tests.test_gpu_norm import check_grad
        dh, dweight = qmm.rms_norm_grad(dx, h, weight)
        check_grad(dh, dweight, dx, h, weight, 1e-6, None)


def test_route_and_adapters_by_the_same_sort(qmm):
    """An adapter per expert: rows gathered in expert order are the adapters' rows, by a router's choice of one."""
    T, E, K, N = 700, 12, 128, 96
    gen = torch.Generator(device="cuda").manual_seed(1)
    l = torch.randn(T, E, generator=gen, device="cuda")
    l[5] = -math.inf
    idx, w = qmm.expert_route(l, 1, renormalize=False)
    plan = qmm.expert_sort(idx, E)
    x = torch.randn(T, K, generator=gen, device="cuda").half()
    a, b = (torch.randn(E, 16, K, generator=gen, device="cuda") / 8).half(), torch.randn(E, N, 16, generator=gen, device="cuda").half()
    y = qmm.lora(x, idx.view(-1), a, b, None, plan=plan)
    s, d, mag_s, mag_d, mag_ds = ref.lora(x.double(), idx.view(-1), a.double(), b.double(), None)
    tol = ref.sum_error(K) * mag_ds + (ref.sum_error(16) + 2.0**-16) * (mag_d + mag_ds) + ref.rounding(d, torch.float16) * 1.01
    assert bool(((y.double() - d).abs() <= tol).all()) and not y[5].any()


def test_the_example(qmm):
    """It runs; its gradients are torch's up to the roundings of bf16 rows (half an ulp 2^-8 each, a handful of them in a row)."""
    from examples import adapted_layer
    adapted, layer, trained = adapted_layer.main(["--tokens", "96"])
    assert adapted < 2 * 2.0**-8 and layer < 0.5 and trained < 8 * 2.0**-8
