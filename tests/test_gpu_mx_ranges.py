"""GPU parity at the ends of the exponent range, and microscaled products on workspaces that other calls have used."""
import numpy as np
import pytest
import torch

from tests import mxref
from tests.test_gpu_mx import DTYPES, FMTS, check_quantized, f64, scale_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


# ---- gate / up

def one_expert(qmm, rows):
    idx = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    return idx, qmm.expert_sort(idx, 1)


def stored(h, fmt, rows, N, g):
    c, s = mxref.unpack(h.cpu().numpy(), fmt, rows, N)
    nb = -(-N // fmt)
    return mxref.values(c[:, : nb * fmt].reshape(rows, nb, fmt), s[:, :nb], fmt, N, g)


@pytest.mark.parametrize("rows", ["64", "128"])
def test_gate_far_below_zero_closes_whatever_up_is(qmm, rows):
    """silu(-2^66) is -0 in 32 bits and closes a feature with u = 2^66, although g u is beyond fp32.  The open features of the block are
    exact: silu(64) = 64 in fp32, and 64 / 16 = 4 is a code under the scale 1.  At g = -88 the factor 1 / (1 + e^88) is a subnormal of fp32, but
    silu = -5.3e-37 is not: times u = 2^120 it is -0.71, whose code under the scale 1 is -0.5."""
    qmm.debug_config("mx_tile", rows)
    K, N = 32, 96
    x = torch.zeros(2, K, device="cuda")
    x[:, 0] = 1
    x[1, 0] = -1
    gate, up = torch.zeros(N, K), torch.zeros(N, K)
    gate[:, 0], up[:, 0] = 64, 1 / 16
    gate[5, 0], up[5, 0] = -2.0**66, 2.0**66
    gate[40, 0], up[40, 0] = -2.0**66, -2.0**66
    up[70, 0] = 2.0**120
    gate[70, 0], gate[70, 1] = -64, -24                                            # (88 is no 4-bit number)
    x[0, 1] = 1
    idx, plan = one_expert(qmm, 2)
    a = qmm.mx_quantize_experts(32, x, idx, plan)
    h = qmm.mx_experts_gate_up(32, a, plan, qmm.mx_quantize(32, gate.cuda()), qmm.mx_quantize(32, up.cuda()), N, K)
    got = stored(h, 32, 2, N, 1.0)
    want = np.full(N, 4.0)
    want[[5, 40]] = 0
    want[70] = -0.5
    assert np.array_equal(np.abs(got[0]), np.abs(want)) and (got[0] * want >= 0).all()
    # the other token has -g and -u: its features of g = -64 are closed, 2^66 * -2^66 is beyond fp32 and its block NaN
    assert np.isnan(got[1, :64]).all() and np.isfinite(got[1, 64:70]).all()


def far_operand(fmt, rows, K, g, seed):
    """Values of about 100 tensor scales: blocks of scales near 16."""
    x = torch.randn(rows, K, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 100 * g
    x = x.float()
    return x, mxref.values(*mxref.quantize(f64(x), fmt, g), fmt, K, g)


@pytest.mark.parametrize("ga,gg,gu,gh", [(1.0, 1e-20, 1e-20, 1e-33), (1e-15, 1e-8, 1e-9, 1e-39), (1e-25, 1e25, 1e20, 1e2), (1e25, 1e-30, 1e-20, 1e7), (1e-25, 1e20, 1e25, 1e2),
                                         (1e20, 1e-20, 1e-25, 1e2), (1e18, 1e-22, 1e12, 1e33)])
def test_gate_up_far_tensor_scales(qmm, ga, gg, gu, gh):
    """g, u and h are fp32 numbers, whatever the product of the tensor scales is.  Tolerance: half a gap of the stored grid (at most the step D, a sixth of the
    block's largest value but for the scale's own rounding: 1/16 of it, or 2^-10 where it is subnormal, six times that at the largest value) and 2^-10 for
    the fp32 products and silu."""
    rows, N, K = 3, 64, 256
    (x, xv), (wg, vg), (wu, vu) = far_operand(16, rows, K, ga, 1), far_operand(16, N, K, gg, 2), far_operand(16, N, K, gu, 3)
    idx, plan = one_expert(qmm, rows)
    a = qmm.mx_quantize_experts(16, x.cuda(), idx, plan, tensor_scale=scale_of(16, ga))
    h = qmm.mx_experts_gate_up(16, a, plan, qmm.mx_quantize(16, wg.cuda(), tensor_scale=scale_of(16, gg)), qmm.mx_quantize(16, wu.cuda(), tensor_scale=scale_of(16, gu)), N, K,
                               a_scale=scale_of(16, ga), gate_scale=scale_of(16, gg), up_scale=scale_of(16, gu), h_scale=scale_of(16, gh))
    got = stored(h, 16, rows, N, gh)
    with np.errstate(over="ignore"):
        hv = mxref.silu(xv @ vg.T) * (xv @ vu.T)
    hv = np.clip(hv, -448 * 6 * gh, 448 * 6 * gh)
    top = np.abs(hv).reshape(rows, -1, 16).max(-1, keepdims=True)
    assert np.isfinite(got).all()
    assert (np.abs(got - hv).reshape(rows, -1, 16) <= (1 / 6 + 1 / 16 + 2.0**-10) * top + 2.0**-7 * gh).all()
    assert (top > 0.02 * gh).all()                                                 # (the case says something)


# ---- dense products

@pytest.mark.parametrize("M,N,K", [(3, 100, 512), (40, 130, 512), (2, 256, 8192), (70, 130, 16384), (300, 400, 512)])
def test_product_far_tensor_scales(qmm, M, N, K):
    """Sums of codes times scales run from 2^-20 to 7e6 K: y = a_scale w_scale sum is an fp32 number where the product of the two scales is not."""
    nb = K // 16

    def operand(rows, code, scale):
        codes = torch.full((rows, nb * 8), code * 17, dtype=torch.uint8, device="cuda")
        return qmm.mx_pack(16, codes, torch.full((rows, nb), scale, dtype=torch.uint8, device="cuda"), K)

    def forms(a, w, ga, gw):
        for knob in (None, ("mx_pair", "1"), ("mx_pair", "2"), ("mx_no_split", "1")):
            if knob and ((knob[0] == "mx_pair") != (M > 128) or (knob[0] == "mx_no_split" and K < 4096)):
                continue
            if knob:
                qmm.debug_config(*knob)
            yield qmm.mx_gemm(16, a, M, w, N, K, a_scale=scale_of(16, ga), w_scale=scale_of(16, gw), dtype=torch.float32)
            qmm.debug_config(None)

    big_a, big_w = operand(M, 7, 0x7E), operand(N, 7, 0x7E)                        # codes 6, scales 448
    sum_big = (6 * 448.0) ** 2 * K
    tol = (K / 64 + 8) * 2.0**-23
    for ga, gw in ((1e-25, 1e-20), (1e-20, 1e-25), (2e-45, 1.0), (1e-45, 3.0)):
        want = sum_big * float(np.float32(ga)) * float(np.float32(gw))
        for Y in forms(big_a, big_w, ga, gw):
            assert (np.abs(f64(Y) - want) <= tol * want + 2.0**-148).all(), (ga, gw, float(Y[0, 0]), want)
    small_a, small_w = operand(M, 1, 1), operand(N, 1, 1)                          # codes 0.5, scales 2^-9
    sum_small = 2.0**-20 * K
    for ga, gw in ((1e20, 1e20), (1e25, 1e14), (1e14, 1e25)):
        want = sum_small * float(np.float32(ga)) * float(np.float32(gw))
        if want > 3e38:
            continue
        for Y in forms(small_a, small_w, ga, gw):
            assert (np.abs(f64(Y) - want) <= tol * want).all(), (ga, gw, float(Y[0, 0]), want)
    none = operand(M, 0, 0)                                                        # a sum of nothing is zero under any scales
    for Y in forms(none, big_w, 1e25, 1e25):
        assert not Y.any() and torch.isfinite(Y).all()


def test_linear_far_tensor_scales(qmm):
    K = 512
    for M, N in ((3, 100), (200, 130)):
        for ga, gw in ((1e-25, 1e-20), (1e-20, 1e-25)):
            X, W = torch.full((M, K), 6 * 448 * ga, device="cuda"), torch.full((N, K), 6 * 448 * gw, device="cuda")
            Y = qmm.mx_linear(16, X, qmm.mx_quantize(16, W, tensor_scale=scale_of(16, gw)), N, x_scale=scale_of(16, ga), w_scale=scale_of(16, gw))
            want = (6 * 448.0) ** 2 * K * float(np.float32(ga)) * float(np.float32(gw))
            assert (np.abs(f64(Y) - want) <= 2.0**-18 * want).all(), (ga, gw, float(Y[0, 0]), want)
        Y = qmm.mx_linear(16, torch.zeros(M, K, device="cuda"), qmm.mx_quantize(16, W, tensor_scale=scale_of(16, gw)), N, x_scale=scale_of(16, 1e25), w_scale=scale_of(16, 1e25))
        assert not Y.any() and torch.isfinite(Y).all()


def test_experts_product_far_tensor_scales(qmm):
    K, N, rows = 512, 100, 5
    idx, plan = one_expert(qmm, rows)
    for ga, gw in ((1e-25, 1e-20), (1e-20, 1e-25)):
        X, W = torch.full((rows, K), 6 * 448 * ga, device="cuda"), torch.full((N, K), 6 * 448 * gw, device="cuda")
        a = qmm.mx_quantize_experts(16, X, idx, plan, tensor_scale=scale_of(16, ga))
        Y = qmm.mx_experts_gemm(16, a, plan, qmm.mx_quantize(16, W, tensor_scale=scale_of(16, gw)), N, K, a_scale=scale_of(16, ga), w_scale=scale_of(16, gw), dtype=torch.float32)
        want = (6 * 448.0) ** 2 * K * float(np.float32(ga)) * float(np.float32(gw))
        assert (np.abs(f64(Y) - want) <= 2.0**-18 * want).all(), (ga, gw, float(Y[0, 0]), want)


# ---- quantisation

@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
def test_scales_of_lanes_that_took_different_branches(qmm, fmt, dt):
    """Four neighbouring blocks of a row share a word of scales: here a row's end, blocks beyond 2^40 (true divisions), zeros and infinities meet in it."""
    dtype = DTYPES[dt]
    for rows, K in ((40, 40), (33, 296), (64, 264), (9, 1000), (5, 2024)):
        x = torch.randn(rows, K, generator=torch.Generator().manual_seed(rows))
        b = torch.arange(K) // fmt
        r = torch.arange(rows)[:, None]
        x = x * torch.where((b + r) % 3 == 0, 2.0**41 if dt != "f16" else 2.0**10, 1.0)
        x = torch.where((b + r) % 7 == 3, torch.zeros(()), x)
        x = torch.where(((b + 2 * r) % 11 == 5) & (torch.arange(K) % fmt == 1), torch.full((), float("inf")), x).to(dtype)
        for g in ((1.0,) if fmt == mxref.MXFP4 else (0.01, 2.0**-41)):
            check_quantized(qmm.mx_quantize(fmt, x.cuda(), tensor_scale=scale_of(fmt, g)), f64(x), fmt, g)
