"""GPU parity of microscaled calls in company: workspaces shared between operators and between batch sizes, calls without rows."""
import numpy as np
import pytest
import torch

from tests import mxref
from tests.test_gpu_mx import FMTS, f64, scale_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def layer(qmm, T=6, H=256, I=128, E=8, topk=2, dtype=torch.float16, scale=0.05):
    gen = torch.Generator(device="cuda").manual_seed(1)
    make = lambda n, k: torch.cat([qmm.mx_quantize(32, torch.randn(n, k, generator=gen, device="cuda") * scale) for _ in range(E)])  # noqa: E731
    idx = torch.randint(0, E, (T, topk), generator=gen, dtype=torch.int32, device="cuda")
    X = torch.randn(T, H, generator=gen, device="cuda").to(dtype)
    w = torch.rand(T, topk, generator=gen, device="cuda")
    return X, idx, w, make(I, H), make(I, H), make(H, I), I, E


def test_experts_rows_in_32_bits(qmm):
    """With rows_dtype = float32 the experts' rows reach the weighted sum unrounded: out is within one rounding of the sum of the fp32 rows,
    and a row beyond fp16 comes back where its weight brings it back."""
    for dtype, T, H, I in ((torch.float16, 6, 256, 128), (torch.bfloat16, 300, 320, 96), (torch.float16, 50, 257, 90), (torch.float32, 20, 64, 64)):
        X, idx, w, gate, up, down, I, E = args = layer(qmm, T=T, H=H, I=I, dtype=dtype)
        out = qmm.mx_moe(32, *args, rows_dtype=torch.float32)
        plan = qmm.expert_sort(idx, E)
        h = qmm.mx_experts_gate_up(32, qmm.mx_quantize_experts(32, X, idx, plan), plan, gate, up, I, H)
        Y = qmm.mx_experts_gemm(32, h, plan, down, H, I, dtype=torch.float32)
        assert torch.equal(out, qmm.expert_combine(Y, plan, w).to(dtype))            # the fp32 sum, rounded once
        buf = torch.full((T, H + 5), 7.0, dtype=dtype, device="cuda")              # rows of any alignment
        qmm.mx_moe(32, *args, out=buf[:, 1:H + 1], rows_dtype=torch.float32)
        assert torch.equal(buf[:, 1:H + 1], out) and bool((buf[:, 0] == 7).all()) and bool((buf[:, H + 1:] == 7).all())
    X, idx, w, gate, up, down, I, E = layer(qmm, scale=4.0)
    w = w * 1e-4
    plain = qmm.mx_moe(32, X, idx, w, gate, up, down, I, E)
    kept = qmm.mx_moe(32, X, idx, w, gate, up, down, I, E, rows_dtype=torch.float32)
    assert torch.isfinite(kept).all() and not torch.isfinite(plain).all()
    with pytest.raises(AssertionError):
        qmm.mx_moe(32, X, idx, w, gate, up, down, I, E, rows_dtype=torch.bfloat16)


def test_one_workspace_for_layers_and_products(qmm):
    """A product that shares a tile's K keeps counters in its workspace's header; another operator's data there must not count."""
    args = layer(qmm)
    out = torch.empty_like(args[0])
    a = qmm.mx_moe_args(32, *args, out)
    ws = torch.zeros(max(qmm.mx_moe_workspace_bytes(a), 1 << 24), dtype=torch.uint8, device="cuda")
    want_layer = qmm.mx_moe(32, *args)
    canon = torch.zeros(qmm.canonical_bytes(qmm.Q4, 512, 4096), dtype=torch.uint8, device="cuda")
    q4, Xg = qmm.pack(qmm.Q4, canon, 512, 4096), torch.randn(100, 4096, device="cuda").half()
    for M, N, K in ((1, 2048, 8192), (16, 512, 8192), (40, 300, 5000)):
        X, w = torch.randn(M, K, device="cuda").half(), qmm.mx_quantize(32, torch.randn(N, K, device="cuda"))
        want = qmm.mx_linear(32, X, w, N)
        xq = qmm.mx_quantize(32, X)
        for other in (lambda: qmm.mx_moe_run(a, ws), lambda: qmm.gemm(qmm.Q4, q4, 512, 4096, Xg, ws=ws)):
            for _ in range(2):
                other()
                Y = torch.full_like(want, 7.0)
                qmm.mx_linear(32, X, w, N, Y=Y, ws=ws)
                assert torch.equal(Y, want)
                other()
                Y = torch.full_like(want, 7.0)
                qmm.mx_gemm(32, xq, M, w, N, K, Y=Y, ws=ws)
                assert torch.equal(Y, want)
                out.fill_(7.0)
                qmm.mx_moe_run(a, ws)
                assert torch.equal(out, want_layer)
        qmm.status_check(ws)
        assert not ws[:256].any(), "status word and counters are zero between calls"


@pytest.mark.parametrize("fmt", FMTS)
def test_workspace_of_the_largest_batch_serves_smaller_ones(qmm, fmt):
    N, K = 2048, 8192
    w = qmm.mx_quantize(fmt, torch.randn(N, K, device="cuda") * 0.05)
    ws = torch.zeros(qmm.mx_linear_workspace_bytes(fmt, 256, N, K), dtype=torch.uint8, device="cuda")
    wg = torch.zeros(qmm.mx_gemm_workspace_bytes(fmt, 256, N, K), dtype=torch.uint8, device="cuda")
    for M in (256, 1, 33, 16, 64, 128, 17, 200):
        X = torch.randn(M, K, device="cuda").half()
        want = qmm.mx_linear(fmt, X, w, N)
        assert torch.equal(qmm.mx_linear(fmt, X, w, N, ws=ws), want)
        assert torch.equal(qmm.mx_gemm(fmt, qmm.mx_quantize(fmt, X), M, w, N, K, ws=wg), want)
    qmm.status_check(ws)
    qmm.status_check(wg)


def test_experts_rows_of_another_routing_are_not_stored(qmm):
    """mx_quantize_experts on an idx that is not the sorted one stores the pairs that agree and writes nowhere else."""
    T, topk, E, K = 70, 3, 5, 300
    rng = np.random.default_rng(3)
    idx = rng.integers(0, E, (T, topk)).astype(np.int32)
    plan = qmm.expert_sort(torch.from_numpy(idx).cuda(), E)
    x = torch.randn(T, K, device="cuda").half()
    other = np.where(rng.random((T, topk)) < 0.5, idx, rng.choice([-1, E, 2**30, -2**31, 0, E - 1], (T, topk))).astype(np.int32)
    need = qmm.mx_experts_bytes(32, T, topk, E, K)
    want = qmm.mx_quantize_experts(32, x, torch.from_numpy(idx).cuda(), plan).cpu().numpy()
    buf = torch.full((need + 8192,), 0xAB, dtype=torch.uint8, device="cuda")
    qmm.mx_quantize_experts(32, x, torch.from_numpy(other).cuda(), plan, out=buf[4096: 4096 + need])
    got = buf.cpu().numpy()
    assert (got[:4096] == 0xAB).all() and (got[4096 + need:] == 0xAB).all()
    order, place, offsets, units = mxref.sort(idx, E)
    for e in range(E):
        n = int(offsets[e + 1] - offsets[e])
        (c, s), (cw, sw) = (mxref.unpack(b, 32, n, K, int(units[e])) for b in (got[4096: 4096 + need], want))
        stored = other.reshape(-1)[order[offsets[e]: offsets[e + 1]]] == e
        assert np.array_equal(c[stored], cw[stored]) and np.array_equal(s[stored], sw[stored])
        assert (s[~stored] == 0xAB).all() and (c[~stored][:, 0::2] == 0xB).all()


def test_no_tokens(qmm):
    """Calls without rows return empty results, whichever wrapper they go through."""
    E, H, I = 4, 256, 128
    idx = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    plan = qmm.expert_sort(idx, E)
    gu, dn = torch.zeros(E * qmm.mx_bytes(32, I, H), dtype=torch.uint8, device="cuda"), torch.zeros(E * qmm.mx_bytes(32, H, I), dtype=torch.uint8, device="cuda")
    x = torch.empty(0, H, dtype=torch.float16, device="cuda")
    a = qmm.mx_quantize_experts(32, x, idx, plan)
    h = qmm.mx_experts_gate_up(32, a, plan, gu, gu, I, H)
    assert a.numel() == 0 and h.numel() == 0
    assert qmm.mx_experts_gemm(32, h, plan, dn, H, I).shape == (0, H)
    assert qmm.mx_moe(32, x, idx, torch.empty(0, 2, device="cuda"), gu, gu, dn, I, E).shape == (0, H)
    assert qmm.mx_pack(32, torch.empty(0, 128, dtype=torch.uint8, device="cuda"), torch.empty(0, 8, dtype=torch.uint8, device="cuda"), 256).numel() == 0
    assert qmm.mx_dequantize(32, a, 0, H).shape == (0, H)
    assert qmm.mx_gemm(32, a, 0, gu, I, H).shape == (0, I)
    assert qmm.expert_gather(x, plan).shape == (0, H) and qmm.expert_combine(x, plan).shape == (0, H)
    with pytest.raises(qmm.QmmError):
        qmm.mx_experts_gate_up(8, a, plan, gu, gu, I, H)                           # (an unknown format is still refused)


def test_plan_before_its_first_sort(qmm):
    """A plan that has not been sorted into drops every pair; its arrays never hold places that are none."""
    T, topk, E, H = 9, 3, 5, 300
    for _ in range(3):                                                             # (memory that others have used)
        torch.full((1 << 20,), 0x7F, dtype=torch.uint8, device="cuda")
    plan = qmm.ExpertPlan(T, topk, E)
    x, ys, w = torch.randn(T, H, device="cuda"), torch.randn(T * topk, H, device="cuda"), torch.rand(T, topk, device="cuda")
    assert bool((plan.order == -1).all()) and bool((plan.place == -1).all()) and not plan.offsets.any() and not plan.units.any()
    assert not qmm.expert_gather(x, plan).any() and not qmm.expert_combine(ys, plan, w).any()
    dys, dw = qmm.expert_combine_grad(x, ys, plan, w)
    assert not dys.any() and not dw.any()
    idx = torch.zeros(T, topk, dtype=torch.int32, device="cuda")
    a = torch.full((qmm.mx_experts_bytes(32, T, topk, E, H),), 0xAB, dtype=torch.uint8, device="cuda")
    qmm.mx_quantize_experts(32, x, idx, plan, out=a)
    Y = torch.full((T * topk, 64), 7.0, device="cuda")
    qmm.mx_experts_gemm(32, a, plan, torch.zeros(E * qmm.mx_bytes(32, 64, H), dtype=torch.uint8, device="cuda"), 64, H, Y=Y)
    assert bool((a == 0xAB).all()) and bool((Y == 7).all())
