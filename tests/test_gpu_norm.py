"""GPU parity: the root-mean-square norm, its gradient, and rows of 8 bits."""
import math

import pytest
import torch

from tests import layerref as ref

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 2048), (4, 4096), (130, 64), (33, 1001), (700, 1000), (5, 8192), (2, 16384), (2, 32768), (3, 20001), (1200, 4096), (9, 32)]


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def rows(M, K, dtype, gen, std=1.0, pitch=None, off=0):
    x = (torch.randn(M, K, generator=gen, device="cuda") * std).to(dtype)
    if pitch is None:
        return x
    buf = torch.full((M * pitch + off + 8,), 7.0, dtype=dtype, device="cuda")
    v = buf[off: off + M * pitch].view(M, pitch)[:, :K]
    v.copy_(x)
    return v


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# squares added 32 at most by a thread, 10 steps over threads: 42 roundings of a positive sum, halved by the root; root, division, two products
STAT = 48 * 2.0**-24


def check_y(y, h, weight, eps):
    rstd, want = ref.norm(h, weight, eps)
    err = (y.double() - want).abs()
    assert bool((err <= STAT * want.abs() + ref.rounding(want, y.dtype)).all())


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("residual,weighted", [(False, True), (True, True), (True, False)])
def test_norm(qmm, dt, M, K, residual, weighted):
    dtype, gen = ref.DTYPES[dt], gen_of(M + K)
    x = rows(M, K, dtype, gen)
    r = rows(M, K, dtype, gen, 3.0) if residual else None
    w = rows(1, K, dtype, gen)[0] if weighted else None
    y, h = qmm.rms_norm(x, w, 1e-5, residual=r)
    assert torch.equal(h, ref.add(x, r))
    check_y(y, h, w, 1e-5)
    again, _ = qmm.rms_norm(x, w, 1e-5, residual=r)
    assert torch.equal(y, again)


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("pitch,off", [(136, 8), (131, 1), (130, 2), (132, 4)])
def test_strides_and_places(qmm, dt, pitch, off):
    dtype, gen = ref.DTYPES[dt], gen_of(pitch)
    x, r = rows(50, 128, dtype, gen, 1, pitch, off), rows(50, 128, dtype, gen, 1, pitch, off)
    w = rows(1, 128, dtype, gen)[0]
    want_h = ref.add(x, r)
    y, h = qmm.rms_norm(x, w, residual=r, h=r, y=x)                                # in place, both ways
    assert h is r and y is x and torch.equal(h, want_h)
    check_y(y, want_h, w, 1e-6)
    assert bool((x.as_strided((50 * pitch - (pitch - 128),), (1,))[128:pitch] == 7.0).all())          # between the rows


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-30, 1e-21, 1e19, 1e30])
def test_ends_of_the_range(qmm, dt, size):
    """Squares outside fp32's range: the statistics are those of 64 bits."""
    dtype, gen = ref.DTYPES[dt], gen_of(3)
    x, w = rows(6, 300, dtype, gen, size), rows(1, 300, dtype, gen)[0]
    x[2] = 0
    x[3] = 1.0
    eps = 1e-6 if size > 1 else 1e-38
    y, _ = qmm.rms_norm(x, w, eps)
    check_y(y, x, w, float(torch.tensor(eps, dtype=torch.float32)))
    dy = rows(6, 300, dtype, gen)
    dx, dw = qmm.rms_norm_grad(dy, x, w, eps)
    check_grad(dx, dw, dy, x, w, float(torch.tensor(eps, dtype=torch.float32)), None)


def test_infinities_and_nan(qmm):
    x = torch.randn(4, 256, device="cuda")
    x[1, 3] = math.inf
    x[2, 4] = math.nan
    y, _ = qmm.rms_norm(x)
    codes, scales, _ = qmm.rms_norm_rows(x)
    assert torch.isfinite(y[0]).all() and torch.isnan(y[1, 3]) and not y[1, :3].any() and torch.isnan(y[2]).all() and torch.isfinite(y[3]).all()
    assert torch.isnan(scales[1:3]).all() and torch.isfinite(scales[[0, 3]]).all() and not codes[1:3].float().any()
    assert torch.isnan(qmm.rows_dequantize(codes, scales)[1:3]).all()


def check_grad(dx, dw, dy, h, w, eps, dh):
    h64, dy64 = h.double(), dy.double()
    w64 = torch.ones_like(h64[0]) if w is None else w.double()
    M, K = h.shape
    rstd = 1 / torch.sqrt(h64.square().mean(1, keepdim=True) + eps)
    xhat = h64 * rstd
    g = w64 * dy64
    mean = (g * xhat).mean(1, keepdim=True)
    want = rstd * (g - xhat * mean)
    size = rstd * (g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    if dh is not None:
        want = want + dh.double()
        size = size + dh.double().abs()
    err = (dx.double() - want).abs()
    # the statistics twice (rstd, mean), the products and sums of an element: five roundings
    assert bool((err <= (3 * STAT + 8 * 2.0**-24) * size + ref.rounding(want, dx.dtype)).all())
    if dw is not None:
        want, size = (dy64 * xhat).sum(0), (dy64 * xhat).abs().sum(0)
        assert bool(((dw.double() - want).abs() <= (STAT + (M + 16) * 2.0**-24) * size + 2.0**-126).all())


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("weighted,with_dh", [(True, False), (True, True), (False, True)])
def test_gradient(qmm, dt, M, K, weighted, with_dh):
    dtype, gen = ref.DTYPES[dt], gen_of(M * K)
    h, dy = rows(M, K, dtype, gen, 2.0), rows(M, K, dtype, gen)
    w = rows(1, K, dtype, gen)[0] if weighted else None
    dh = rows(M, K, dtype, gen) if with_dh else None
    dx, dw = qmm.rms_norm_grad(dy, h, w, 1e-5, dh=dh)
    check_grad(dx, dw, dy, h, w, 1e-5, dh)
    dx2, dw2 = qmm.rms_norm_grad(dy, h, w, 1e-5, dh=dh)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    only, none = qmm.rms_norm_grad(dy, h, w, 1e-5, dh=dh, dx=dy, want_dweight=False)  # in place of dy
    assert none is None and torch.equal(only, dx)


@pytest.mark.parametrize("dt", list(ref.DTYPES))
def test_gradient_with_strides(qmm, dt):
    dtype, gen = ref.DTYPES[dt], gen_of(1)
    h, dy, dh = (rows(40, 200, dtype, gen, 1, 211, 3) for _ in range(3))
    w = rows(1, 200, dtype, gen)[0]
    out = rows(40, 200, dtype, gen, 1, 211, 3)
    dx, dw = qmm.rms_norm_grad(dy, h, w, dh=dh, dx=out)
    check_grad(dx, dw, dy, h, w, 1e-6, dh)


def test_gradient_against_differences(qmm):
    gen = gen_of(4)
    h, dy, w = rows(3, 40, torch.float32, gen), rows(3, 40, torch.float32, gen), rows(1, 40, torch.float32, gen)[0]
    dx, dw = qmm.rms_norm_grad(dy, h, w, 1e-5)
    f = lambda h64, w64: float((ref.norm(h64, w64, 1e-5)[1] * dy.double()).sum())  # noqa: E731
    e = 2.0**-12
    for t, k in ((0, 0), (1, 17), (2, 39)):
        up, down = h.double().clone(), h.double().clone()
        up[t, k] += e
        down[t, k] -= e
        assert abs((f(up, w) - f(down, w)) / (2 * e) - float(dx[t, k])) < 1e-4
        wu, wd = w.double().clone(), w.double().clone()
        wu[k] += e
        wd[k] -= e
        assert abs((f(h, wu) - f(h, wd)) / (2 * e) - float(dw[k])) < 1e-4


def test_gradient_of_no_rows(qmm):
    e = torch.empty(0, 64, device="cuda")
    dx, dw = qmm.rms_norm_grad(e, e, torch.ones(64, device="cuda"))
    assert dx.shape == (0, 64) and not dw.any()
    assert qmm.rms_norm(e)[0].shape == (0, 64) and qmm.rows_quantize(e)[0].shape == (0, 64)


def bits(codes):
    return codes.view(torch.uint8)


@pytest.mark.parametrize("kind", list(ref.ROW8))
@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_rows_of_8_bits(qmm, kind, dt, M, K, residual):
    dtype, gen, k8 = ref.DTYPES[dt], gen_of(M + K), ref.ROW8[kind]
    x, w = rows(M, K, dtype, gen), rows(1, K, dtype, gen)[0]
    r = rows(M, K, dtype, gen) if residual else None
    if M > 2:
        x[1] = 0
        if residual:
            r[1] = 0
    y = torch.empty_like(x)
    codes, scales, h = qmm.rms_norm_rows(x, w, 1e-5, residual=r, dtype=k8, y=y)
    assert torch.equal(h, ref.add(x, r))
    check_y(y, h, w, 1e-5)
    rstd, _ = ref.norm(h, w, 1e-5)
    want, want_s = ref.rows8(h.float() * w.float(), k8, rstd)
    assert torch.equal(bits(codes), bits(want))
    assert bool(((scales.double() - want_s).abs() <= (STAT + 4 * 2.0**-24) * want_s).all())
    for out in ref.DTYPES.values():
        v = qmm.rows_dequantize(codes, scales, dtype=out)
        assert torch.equal(v, (codes.float() * scales[:, None]).to(out))


@pytest.mark.parametrize("kind", list(ref.ROW8))
@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("M,K,pitch,off", [(7, 2048, None, 0), (40, 72, 80, 8), (40, 72, 75, 3), (31, 1003, None, 0)])
def test_quantise_rows_and_back(qmm, kind, dt, M, K, pitch, off):
    dtype, gen, k8 = ref.DTYPES[dt], gen_of(M), ref.ROW8[kind]
    x = rows(M, K, dtype, gen, 1, pitch, off)
    codes = None
    if pitch:
        codes = torch.zeros(M * pitch + off, dtype=torch.uint8, device="cuda").view(k8)[off:].view(M, pitch)[:, :K]
    codes, scales = qmm.rows_quantize(x, codes=codes, dtype=k8)
    want, want_s = ref.rows8(x.float(), k8, 1.0)
    assert torch.equal(bits(codes.contiguous()), bits(want)) and torch.equal(scales.double(), want_s.float().double())
    out = rows(M, K, dtype, gen, 1, pitch, off)
    v = qmm.rows_dequantize(codes, scales, out=out)
    assert torch.equal(v, (codes.float() * scales[:, None]).to(dtype))


@pytest.mark.parametrize("kind", list(ref.ROW8))
def test_codes_at_halves_and_ends(qmm, kind):
    """Every half-way point of the codes, the smallest and largest rows."""
    k8, top = ref.ROW8[kind], ref.TOP[ref.ROW8[kind]]
    if kind == "int8":
        grid = torch.arange(-127, 128).float()
    else:
        grid = torch.arange(0, 127, dtype=torch.uint8).view(k8).float()
    half = (grid[1:] + grid[:-1]) / 2
    t = torch.cat([half, -half, grid, torch.tensor([top])])[None]
    x = torch.cat([t, t * 2.0**-100, t * 2.0**100, t * 2.0**-126, torch.zeros_like(t)]).cuda()
    codes, scales = qmm.rows_quantize(x, dtype=k8)
    want, want_s = ref.rows8(x, k8, 1.0)
    assert torch.equal(bits(codes), bits(want)) and torch.equal(scales.double(), want_s.float().double())
    zero = x.abs().amax(1) < 2.0**-118
    assert zero[4] and not bits(codes)[zero].any() and not scales[zero].any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 300, 4096, 8191, 32768])
@pytest.mark.parametrize("residual", [False, True])
def test_largest_rows(qmm, dt, K, residual):
    """Rows up to the end of the type's range: y, the 8-bit rows' scale and the gradients are numbers of ordinary size, or as small as rstd makes them."""
    dtype, gen = ref.DTYPES[dt], gen_of(K)
    x = rows(7, K, dtype, gen, 5e37)
    top = torch.finfo(dtype).max
    x[0] = top
    x[1] = -top
    x[2, : K // 2] = 0
    x[3] = rows(1, K, dtype, gen, 5e36)[0]
    x[4] = rows(1, K, dtype, gen, 1e20)[0]
    x[5] = rows(1, K, dtype, gen, 1.0)[0]
    r = None
    if residual:
        r = (x.double() * -0.25).to(dtype)
    w = (0.2 + 0.5 * torch.rand(K, generator=gen, device="cuda")).to(dtype)
    eps = float(torch.tensor(1e-6))
    y, h = qmm.rms_norm(x, w, eps, residual=r)
    assert torch.equal(h, ref.add(x, r))
    check_y(y, h, w, eps)
    assert bool((y.double().square().mean(1) > 0.03).all())
    for kind in ref.ROW8.values():
        codes, scales, h8 = qmm.rms_norm_rows(x, w, eps, residual=r, dtype=kind)
        want, scale = ref.rows8(h8.float() * w.float(), kind, ref.norm(h, w, eps)[0])
        assert torch.equal(codes.view(torch.uint8), want.view(torch.uint8))
        assert bool(((scales.double() - scale).abs() <= (STAT + 2.0**-22) * scale + 2.0**-149).all())
    for size in (1.0, 1e18, 1e30):                         # (larger dy: dx itself comes back to ordinary size)
        dy = rows(7, K, dtype, gen, size)
        dh = rows(7, K, dtype, gen, size * 1e-38) if residual else None
        dx, dw = qmm.rms_norm_grad(dy, h, w, eps, dh=dh)
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
        check_grad(dx, dw, dy, h, w, eps, dh)


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("M,K", [(3, 64), (700, 1000), (700, 1001), (40, 16384), (5, 32768)])
def test_gradient_in_the_place_of_what_comes_in(qmm, dt, M, K):
    """dx over dh, and over dy."""
    dtype, gen = ref.DTYPES[dt], gen_of(M + K)
    h, dy, dh, w = rows(M, K, dtype, gen), rows(M, K, dtype, gen), rows(M, K, dtype, gen), rows(1, K, dtype, gen)[0]
    want, dweight = qmm.rms_norm_grad(dy, h, w, dh=dh)
    for place in (0, 1):
        args = [dy.clone(), dh.clone()]
        dx, dw = qmm.rms_norm_grad(args[0], h, w, dh=args[1], dx=args[place])
        assert dx is args[place] and torch.equal(dx, want) and torch.equal(dw, dweight)
        assert torch.equal(args[1 - place], (dy, dh)[1 - place])
