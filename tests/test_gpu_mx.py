"""GPU parity: microscaled 4-bit floating point -- quantisation bit for bit, products against 64 bits.

Products of 4-bit codes and block scales are exact; the tensor core adds 64 of them per step and keeps 32 bits, so an
fp32 output of K elements is within (K / 64 + 8) roundings of 2^-23 of sum |a w| (the 8: the sums inside a step,
the split over blocks and the tensor scales).  Narrower outputs add half an ulp of their type."""
import numpy as np
import pytest
import torch

from tests import mxref

pytestmark = pytest.mark.gpu
FMTS = [mxref.MXFP4, mxref.NVFP4]
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_ULP = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def f64(t):
    return t.detach().double().cpu().numpy()


def scale_of(fmt, g):
    return None if fmt == mxref.MXFP4 else torch.full((1,), g, dtype=torch.float32, device="cuda")


def same_codes(a, b):
    """Codes equal, the two zeros taken for one."""
    return np.array_equal(np.where(a == 8, 0, a), np.where(b == 8, 0, b))


def check_quantized(packed, x, fmt, g):
    rows, K = x.shape
    codes, scale = mxref.quantize(x, fmt, g)
    got_c, got_s = mxref.unpack(packed.cpu().numpy(), fmt, rows, K)
    nb = scale.shape[1]
    assert np.array_equal(got_s[:, :nb], scale)
    assert same_codes(got_c[:, : nb * fmt], codes.reshape(rows, -1))
    assert not got_s[:, nb:].any() and not got_c[:, nb * fmt:].any(), "padding along K is zero"


def hard_values(dtype, rows, K, seed):
    """Ordinary values, ties of the grid, powers of two, zeros, the type's ends, and blocks of very different sizes."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, -0.0, 7.0, 4.0])
    pick = rng.random((rows, K)) < 0.3
    x = np.where(pick, rng.choice(ties, (rows, K)) * rng.choice([1, -1], (rows, K)) * np.exp2(rng.integers(-3, 3, (rows, 1))), x)
    t = torch.from_numpy(x).to(dtype)
    info = torch.finfo(dtype)
    if rows > 4:
        t[1, : K // 2] = 0
        t[2] = t[2] * info.tiny
        t[3, 0] = info.max
        t[3, K - 1] = -info.max
        t[4] = (t[4].double() * info.tiny * 0.25).to(dtype)                       # subnormals of the type
    return t


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", list(DTYPES))
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (5, 31), (7, 257), (33, 1000), (129, 256), (130, 300), (300, 2048)])
def test_quantize_bit_for_bit(qmm, fmt, dt, rows, K):
    for g in ((1.0,) if fmt == mxref.MXFP4 else (1.0, 2.0**-9, 0.00223, 3.7)):
        x = hard_values(DTYPES[dt], rows, K, rows + K)
        packed = qmm.mx_quantize(fmt, x.cuda(), tensor_scale=scale_of(fmt, g))
        check_quantized(packed, f64(x), fmt, g)


@pytest.mark.parametrize("g", [1e-30, 1e-25, 1e25, 1e36])
def test_quantize_far_tensor_scales(qmm, g):
    """Steps near the ends of the exponent range take true divisions."""
    x = hard_values(torch.float32, 9, 320, 5)
    x[5:] = (x[5:].double() * g).float()
    check_quantized(qmm.mx_quantize(mxref.NVFP4, x.cuda(), tensor_scale=scale_of(mxref.NVFP4, g)), f64(x), mxref.NVFP4, g)


def test_quantize_quotients_are_correctly_rounded(qmm):
    """The quotient x / D decides ties: every e4m3 scale against numerators on, just below and just above every tie."""
    for g in (1.0, 0.00223, 1.7):
        scales = mxref.E4M3[1:]                                                    # every positive scale
        D = scales.astype(np.float32) * np.float32(g)
        amax = (np.float32(6) * np.float32(g) * scales.astype(np.float32)).astype(np.float32)
        ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
        num = (ties[None, :] * D[:, None]).astype(np.float32)
        x = np.zeros((len(D), 32), np.float32)
        x[:, 0], x[:, 16] = amax, -amax
        x[:, 1:8], x[:, 8:15] = num, np.nextafter(num, np.float32(0))
        x[:, 17:24] = np.nextafter(num, np.float32(1e30))
        check_quantized(qmm.mx_quantize(mxref.NVFP4, torch.from_numpy(x).cuda(), tensor_scale=scale_of(mxref.NVFP4, g)), x.astype(np.float64), mxref.NVFP4, g)


@pytest.mark.parametrize("fmt", FMTS)
def test_infinities_and_nans_poison_their_block_only(qmm, fmt):
    for dt in DTYPES.values():
        x = torch.randn(6, 256, generator=torch.Generator().manual_seed(1)).to(dt)
        x[0, 3], x[1, 40], x[2, 255], x[3, 100] = float("inf"), float("-inf"), float("nan"), -float("nan")
        packed = qmm.mx_quantize(fmt, x.cuda(), tensor_scale=scale_of(fmt, 0.01))
        check_quantized(packed, f64(x), fmt, 0.01)
        v = f64(qmm.mx_dequantize(fmt, packed, 6, 256, tensor_scale=scale_of(fmt, 0.01)))
        for r, k in ((0, 3), (1, 40), (2, 255), (3, 100)):
            b = k // fmt * fmt
            assert np.isnan(v[r, b: b + fmt]).all() and np.isfinite(np.delete(v[r], np.arange(b, b + fmt))).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dt", list(DTYPES))
def test_strides_and_alignment(qmm, fmt, dt):
    """Row pitches and base addresses that allow 32-byte, 16-byte and element-wise access give the same codes."""
    base = hard_values(DTYPES[dt], 37, 640, 3).cuda()
    want = qmm.mx_quantize(fmt, base, tensor_scale=scale_of(fmt, 0.02))
    for pitch, off in ((640, 0), (648, 8), (641, 1), (700, 3), (656, 16)):
        buf = torch.full((38 * pitch,), float("nan"), dtype=base.dtype, device="cuda")
        view = buf[off: off + 37 * pitch].view(37, pitch)[:, :640]
        view.copy_(base)
        got = qmm.mx_quantize(fmt, view, tensor_scale=scale_of(fmt, 0.02))
        a, b = mxref.unpack(got.cpu().numpy(), fmt, 37, 640), mxref.unpack(want.cpu().numpy(), fmt, 37, 640)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
        out = torch.full((38 * pitch,), 7.0, dtype=base.dtype, device="cuda")
        ov = out[off: off + 37 * pitch].view(37, pitch)
        qmm.mx_dequantize(fmt, want, 37, 640, out=ov[:, :640], tensor_scale=scale_of(fmt, 0.02))
        assert torch.equal(ov[:, :640], qmm.mx_dequantize(fmt, want, 37, 640, tensor_scale=scale_of(fmt, 0.02), dtype=base.dtype))
        assert bool((ov[:, 640:] == 7).all()) and bool((out[:off] == 7).all())


@pytest.mark.parametrize("fmt", FMTS)
def test_pack_and_dequantize(qmm, fmt):
    rng = np.random.default_rng(2)
    for rows, K in ((1, 16), (130, 272), (128, 256), (5, 1000)):
        nb = -(-K // fmt)
        codes = rng.integers(0, 16, (rows, nb, fmt))
        codes.reshape(rows, -1)[:, K:] = 0
        scale = rng.integers(1, 127, (rows, nb)) if fmt == mxref.NVFP4 else rng.integers(100, 150, (rows, nb))
        scale[0, 0] = 127 if fmt == mxref.NVFP4 else 255
        if rows > 1:
            scale[1, 0] = 0
        flat = codes.reshape(rows, -1).astype(np.uint8)
        canon = torch.from_numpy(flat[:, 0::2] | (flat[:, 1::2] << 4)).cuda()
        out = torch.full((qmm.mx_bytes(fmt, rows, K),), 0xA5, dtype=torch.uint8, device="cuda")
        qmm.mx_pack(fmt, canon, torch.from_numpy(scale.astype(np.uint8)).cuda(), K, out=out)
        assert np.array_equal(out.cpu().numpy(), mxref.pack(codes, scale, fmt))
        ref = mxref.values(codes, scale, fmt, K, 0.37)
        for dt in DTYPES.values():
            got = qmm.mx_dequantize(fmt, out, rows, K, tensor_scale=scale_of(fmt, 0.37), dtype=dt)
            want = torch.from_numpy(ref.astype(np.float32)).to(dt)                 # code * D in fp32, rounded once
            assert np.array_equal(f64(got), f64(want), equal_nan=True)


def operands(fmt, M, N, K, seed, g=(0.004, 0.0003)):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for rows, std, gs in ((M, 1.0, g[0]), (N, 0.05, g[1])):
        x = torch.randn(rows, K, generator=gen) * std * torch.exp2(torch.randint(-2, 3, (rows, 1), generator=gen).float())
        x = x * torch.exp2(torch.randint(-3, 3, (1, K), generator=gen).float())    # block scales differ along K
        codes, scale = mxref.quantize(f64(x), fmt, gs)
        out.append((x, mxref.values(codes, scale, fmt, K, gs), scale_of(fmt, gs)))
    return out


def check_product(Y, a, w, K, what=""):
    ref, mag = a @ w.T, np.abs(a) @ np.abs(w).T
    tol = (K / 64 + 8) * 2.0**-23 * mag + HALF_ULP[Y.dtype] * np.abs(ref) * 1.001 + (2.0**-25 if Y.dtype == torch.float16 else 0)
    err = np.abs(f64(Y) - ref)
    assert np.isfinite(f64(Y)).all() and (err <= tol).all(), "%s: worst %.3f of the bound" % (what, float((err / tol).max()))


# one tile; K tails; few and many weight tiles; several token tiles; more tiles than SMs, ragged both ways
SHAPES = [(1, 1, 1), (1, 128, 256), (3, 100, 32), (5, 130, 272), (128, 128, 512), (17, 256, 1024), (1, 2048, 2048), (9, 512, 2304), (127, 640, 1000),
          (129, 1000, 520), (300, 384, 768), (1, 20000, 256), (200, 10000, 300), (700, 4100, 544), (2500, 3000, 288), (130, 129, 4000), (300, 301, 600), (1500, 2051, 300), (513, 998, 256), (1, 2048, 8192), (40, 300, 5000), (128, 129, 4096), (200, 777, 6000), (14, 1900, 7000), (50, 515, 16384)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(qmm, fmt, M, N, K):
    (xa, a, ga), (xw, w, gw) = operands(fmt, M, N, K, M + N + K)
    wp = qmm.mx_quantize(fmt, xw.cuda(), tensor_scale=gw)
    ap = qmm.mx_quantize(fmt, xa.cuda(), tensor_scale=ga)
    ws = torch.zeros(qmm.mx_gemm_workspace_bytes(fmt, M, N, K), dtype=torch.uint8, device="cuda")
    for dt in DTYPES.values():
        Y = qmm.mx_gemm(fmt, ap, M, wp, N, K, a_scale=ga, w_scale=gw, ws=ws, dtype=dt)
        qmm.status_check(ws)
        check_product(Y, a, w, K, "M=%d N=%d K=%d fmt=%d %s" % (M, N, K, fmt, dt))
        assert torch.equal(Y, qmm.mx_gemm(fmt, ap, M, wp, N, K, a_scale=ga, w_scale=gw, ws=ws, dtype=dt)), "same bits on every call"
        if M > 128:                                                                # both tile forms, whichever the plan took
            for form in ("1", "2"):
                qmm.debug_config("mx_pair", form)
                check_product(qmm.mx_gemm(fmt, ap, M, wp, N, K, a_scale=ga, w_scale=gw, ws=ws, dtype=dt), a, w, K, "form " + form)
                qmm.status_check(ws)
        qmm.debug_config(None)
        if K >= 4096:                                                              # without blocks that share a tile's K
            qmm.debug_config("mx_no_split", "1")
            check_product(qmm.mx_gemm(fmt, ap, M, wp, N, K, a_scale=ga, w_scale=gw, ws=ws, dtype=dt), a, w, K, "whole K")
            qmm.debug_config(None)
            assert not ws[256:1024].any(), "the counters are zero between calls"


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 64, 100, 128, 130, 256, 257, 400])
def test_linear_is_quantize_then_product(qmm, fmt, M):
    """qmm_mx_linear gives the bits of qmm_mx_quantize followed by qmm_mx_gemm, whatever form it takes."""
    for N, K in ((384, 800), (2048, 512), (200, 4096), (130, 9000), (1100, 5000)):
        (xa, _, ga), (xw, _, gw) = operands(fmt, M, N, K, M + N)
        wp = qmm.mx_quantize(fmt, xw.cuda(), tensor_scale=gw)
        for dt in DTYPES.values():
            X = xa.to(dt).cuda()
            ws = torch.zeros(qmm.mx_linear_workspace_bytes(fmt, M, N, K), dtype=torch.uint8, device="cuda")
            Y = qmm.mx_linear(fmt, X, wp, N, x_scale=ga, w_scale=gw, ws=ws)
            qmm.status_check(ws)
            codes, scale = mxref.quantize(f64(X), fmt, 0.004)
            check_product(Y, mxref.values(codes, scale, fmt, K, 0.004), mxref.values(*mxref.quantize(f64(xw), fmt, 0.0003), fmt, K, 0.0003), K)
            assert torch.equal(Y, qmm.mx_gemm(fmt, qmm.mx_quantize(fmt, X, tensor_scale=ga), M, wp, N, K, a_scale=ga, w_scale=gw, dtype=dt))
            for pitch, off in ((K + 8, 8), (K + 3, 1)):                            # rows that allow 16-byte and element-wise loads
                view = torch.zeros(M * pitch + off, dtype=dt, device="cuda")[off:].view(M, pitch)[:, :K]
                view.copy_(X)
                assert torch.equal(Y, qmm.mx_linear(fmt, view, wp, N, x_scale=ga, w_scale=gw, ws=ws))
            qmm.status_check(ws)


@pytest.mark.parametrize("fmt", FMTS)
def test_output_strides(qmm, fmt):
    for M, N, K in ((5, 200, 512), (130, 300, 256), (260, 520, 512), (513, 5000, 256)):
        (xa, a, ga), (xw, w, gw) = operands(fmt, M, N, K, 9)
        ap, wp = qmm.mx_quantize(fmt, xa.cuda(), tensor_scale=ga), qmm.mx_quantize(fmt, xw.cuda(), tensor_scale=gw)
        for dt in DTYPES.values():
            want = qmm.mx_gemm(fmt, ap, M, wp, N, K, a_scale=ga, w_scale=gw, dtype=dt)
            for pitch, off in ((N + 8, 8), (N + 1, 1), (N + 16, 0)):
                buf = torch.full(((M + 1) * pitch,), 7.0, dtype=dt, device="cuda")
                view = buf[off: off + M * pitch].view(M, pitch)
                qmm.mx_gemm(fmt, ap, M, wp, N, K, Y=view[:, :N], a_scale=ga, w_scale=gw)
                assert torch.equal(view[:, :N], want)
                assert bool((view[:, N:] == 7).all()) and bool((buf[:off] == 7).all()) and bool((buf[off + M * pitch:] == 7).all())


@pytest.mark.parametrize("fmt", FMTS)
def test_nan_blocks_reach_exactly_the_outputs_that_read_them(qmm, fmt):
    for M, N, K in ((6, 256, 512), (300, 512, 512), (600, 4096, 512)):
        gen = torch.Generator().manual_seed(4)
        xa, xw = torch.randn(M, K, generator=gen), torch.randn(N, K, generator=gen)
        xa[2, 77], xw[130, 500] = float("nan"), float("inf")
        Y = f64(qmm.mx_gemm(fmt, qmm.mx_quantize(fmt, xa.cuda()), M, qmm.mx_quantize(fmt, xw.cuda()), N, K, dtype=torch.float32))
        want = np.zeros((M, N), bool)
        want[2], want[:, 130] = True, True
        assert np.array_equal(np.isnan(Y), want) and np.isfinite(Y[~want]).all()


def test_rows_past_the_matrix_are_not_data(qmm):
    """The rows that pad the last unit may hold anything, NaN scales included."""
    for fmt in FMTS:
        for M, N, K in ((5, 130, 512), (200, 300, 256), (300, 400, 512), (385, 4225, 512)):
            (xa, a, ga), (xw, w, gw) = operands(fmt, M, N, K, 2)
            ap, wp = (torch.full((qmm.mx_bytes(fmt, r, K),), 0xFF, dtype=torch.uint8, device="cuda") for r in (M, N))
            qmm.mx_quantize(fmt, xa.cuda(), out=ap, tensor_scale=ga)
            qmm.mx_quantize(fmt, xw.cuda(), out=wp, tensor_scale=gw)
            check_product(qmm.mx_gemm(fmt, ap, M, wp, N, K, a_scale=ga, w_scale=gw, dtype=torch.float32), a, w, K)


def test_other_streams_and_graphs(qmm):
    fmt, M, N, K = mxref.MXFP4, 40, 512, 1024
    (xa, a, _), (xw, w, _) = operands(fmt, M, N, K, 6)
    X, Wd = xa.cuda(), xw.cuda()
    Y = torch.empty(M, N, device="cuda")
    ws = torch.zeros(qmm.mx_linear_workspace_bytes(fmt, M, N, K), dtype=torch.uint8, device="cuda")
    wp = torch.empty(qmm.mx_bytes(fmt, N, K), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):                                                     # weights quantised and used in stream order
        qmm.mx_quantize(fmt, Wd, out=wp)
        qmm.mx_linear(fmt, X, wp, N, Y=Y, ws=ws)
    s.synchronize()
    check_product(Y, a, w, K)
    first = Y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qmm.mx_quantize(fmt, Wd, out=wp)
        qmm.mx_linear(fmt, X, wp, N, Y=Y, ws=ws)
    for _ in range(3):
        Y.zero_()
        wp.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, first)


def test_offsets_past_32_bits(qmm):
    fmt, K, N = mxref.NVFP4, 512, 128
    (xa, a, ga), (xw, w, gw) = operands(fmt, 4, N, K, 8)
    pitch = (1 << 30) + 8
    big = torch.empty(3 * pitch + 1024, dtype=torch.float16, device="cuda")        # 6.4 GB; the last row starts past 2^31 elements
    view = big.as_strided((4, K), (pitch, 1))
    view.copy_(xa.half())
    wp = qmm.mx_quantize(fmt, xw.cuda(), tensor_scale=gw)
    want = qmm.mx_linear(fmt, xa.half().cuda(), wp, N, x_scale=ga, w_scale=gw)
    out = torch.empty(3 * pitch + 1024, dtype=torch.float16, device="cuda").as_strided((4, N), (pitch, 1))
    qmm.mx_linear(fmt, view, wp, N, Y=out, x_scale=ga, w_scale=gw)
    assert torch.equal(out, want)
    back = qmm.mx_dequantize(fmt, qmm.mx_quantize(fmt, view, tensor_scale=ga), 4, K, out=view, tensor_scale=ga)
    assert np.array_equal(f64(back), mxref.values(*mxref.quantize(f64(xa.half()), fmt, 0.004), fmt, K, 0.004).astype(np.float32).astype(np.float16).astype(np.float64))


@pytest.mark.parametrize("fmt", FMTS)
def test_nan_token_in_a_few_rows(qmm, fmt):
    xw = torch.randn(256, 512, generator=torch.Generator().manual_seed(1)).cuda()
    X = torch.randn(5, 512, generator=torch.Generator().manual_seed(2)).cuda()
    X[3, 100] = float("inf")
    Y = qmm.mx_linear(fmt, X, qmm.mx_quantize(fmt, xw), 256)
    assert bool(torch.isnan(Y[3]).all()) and bool(torch.isfinite(Y[[0, 1, 2, 4]]).all())


def test_no_rows(qmm):
    w = qmm.mx_quantize(mxref.MXFP4, torch.randn(128, 256, device="cuda"))
    assert qmm.mx_linear(mxref.MXFP4, torch.empty(0, 256, dtype=torch.float16, device="cuda"), w, 128).shape == (0, 128)
    assert qmm.mx_quantize(mxref.NVFP4, torch.empty(0, 64, device="cuda"), out=w) is w
