"""GPU: products of 4-bit integers under power-of-two scales are exact in every form of the kernel.

Codes 0, 1, 2, 3, 4, 6 with either sign and scales 1, 2 or 4: every product is an integer, and sums of up to 36 * 16 * K < 2^24 (K <= 16384) stay integers of fp32
whatever the order of additions, so outputs are the integer result, rounded once to their type."""
import numpy as np
import pytest
import torch

from tests import mxref
from tests.test_gpu_mx import DTYPES, FMTS, f64

pytestmark = pytest.mark.gpu
INTEGERS = np.array([0, 2, 4, 5, 6, 7])                                            # codes of 0, 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def integers(fmt, rows, K, seed):
    """Codes [rows, nb, fmt] and scale bytes [rows, nb] of integers (zero past K), and the integers [rows, K]."""
    rng = np.random.default_rng(seed)
    nb = -(-K // fmt)
    codes = rng.choice(INTEGERS, (rows, nb, fmt)) | (rng.integers(0, 2, (rows, nb, fmt)) << 3)
    codes.reshape(rows, -1)[:, K:] = 0
    power = rng.integers(0, 3, (rows, nb))
    scale = power + 127 if fmt == mxref.MXFP4 else (power + 7) << 3                # e8m0, e4m3 bytes of 1, 2, 4
    return codes, scale, mxref.values(codes, scale, fmt, K)


def packed(qmm, fmt, codes, scale, K):
    flat = codes.reshape(codes.shape[0], -1).astype(np.uint8)
    return qmm.mx_pack(fmt, torch.from_numpy(flat[:, 0::2] | (flat[:, 1::2] << 4)).cuda(), torch.from_numpy(scale.astype(np.uint8)).cuda(), K)


def rounded(v, dtype):
    return torch.from_numpy(v.astype(np.float32)).to(dtype).double().numpy()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", [(1, 128, 256), (5, 130, 272), (128, 300, 800), (129, 257, 1000), (300, 1000, 512), (600, 2100, 768), (1, 2048, 8192), (40, 300, 5000), (70, 130, 16384)])
def test_integer_products_are_exact(qmm, fmt, M, N, K):
    (ca, sa, a), (cw, sw, w) = integers(fmt, M, K, M), integers(fmt, N, K, N + 1)
    want = a @ w.T
    assert np.abs(a).max() * np.abs(w).max() * K < 2**24 and np.array_equal(want, np.round(want))
    ap, wp = packed(qmm, fmt, ca, sa, K), packed(qmm, fmt, cw, sw, K)
    for dt in DTYPES.values():
        for knob in (None, ("mx_pair", "1"), ("mx_pair", "2"), ("mx_no_split", "1")):
            if knob:
                qmm.debug_config(*knob)
            assert np.array_equal(f64(qmm.mx_gemm(fmt, ap, M, wp, N, K, dtype=dt)), rounded(want, dt)), (dt, knob)
            qmm.debug_config(None)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", [(1, 130, 272), (3, 2048, 2048), (16, 300, 800), (9, 500, 8192), (40, 300, 512), (200, 300, 512)])
def test_integer_activations_are_exact(qmm, fmt, M, N, K):
    """A block whose largest magnitude is 6 is quantised under the scale 1: integer activations go through the product's own quantisation unchanged."""
    cw, sw, w = integers(fmt, N, K, 1)
    rng = np.random.default_rng(2)
    x = rng.choice([0, 1, 2, 3, 4, 6], (M, K)) * rng.choice([1, -1], (M, K))
    x[:, ::fmt] = 6
    wp = packed(qmm, fmt, cw, sw, K)
    for dt in DTYPES.values():
        for knob in (None, ("mx_no_few", "1"), ("mx_no_split", "1")):
            if knob:
                qmm.debug_config(*knob)
            Y = qmm.mx_linear(fmt, torch.from_numpy(x).to(dt).cuda(), wp, N)
            assert np.array_equal(f64(Y), rounded(x @ w.T, dt)), (dt, knob)
            qmm.debug_config(None)


@pytest.mark.parametrize("fmt", FMTS)
def test_integer_experts_are_exact(qmm, fmt):
    T, topk, E, N, K = 90, 3, 5, 200, 520
    rng = np.random.default_rng(4)
    idx = rng.integers(-1, E, (T, topk)).astype(np.int32)
    x = rng.choice([0, 1, 2, 3, 4, 6], (T, K)) * rng.choice([1, -1], (T, K))
    x[:, ::fmt] = 6
    ws = [integers(fmt, N, K, 10 + e) for e in range(E)]
    idx_d = torch.from_numpy(idx).cuda()
    plan = qmm.expert_sort(idx_d, E)
    a = qmm.mx_quantize_experts(fmt, torch.from_numpy(x).half().cuda(), idx_d, plan)
    Y = f64(qmm.mx_experts_gemm(fmt, a, plan, torch.cat([packed(qmm, fmt, c, s, K) for c, s, _ in ws]), N, K, dtype=torch.float32))
    order, _, offsets, _ = mxref.sort(idx, E)
    for e in range(E):
        rows = slice(int(offsets[e]), int(offsets[e + 1]))
        assert np.array_equal(Y[rows], x[order[rows] // topk] @ ws[e][2].T)
