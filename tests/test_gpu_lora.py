"""GPU parity: low-rank adapters of any mixture of rows beside a projection, forward and backward, on 16-bit and 8-bit rows."""
import itertools

import pytest
import torch

from tests import layerref as ref

pytestmark = pytest.mark.gpu

HALVES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def adapters_of(T, n, kind, seed):
    gen = torch.Generator().manual_seed(seed)
    idx = torch.randint(0, n, (T,), generator=gen)
    if kind == "dropped":
        odd = torch.tensor([-1, n, 2**31 - 1, -2**31])[torch.randint(0, 4, (T,), generator=gen)]
        idx = torch.where(torch.rand(T, generator=gen) < 0.3, odd, idx)
    elif kind == "one":
        idx[:] = n - 1
    elif kind == "none":
        idx[:] = -1
    elif kind == "skewed":
        idx = torch.where(torch.rand(T, generator=gen) < 0.7, 0, idx)
    return idx.int().cuda()


def matrix(M, K, dtype, gen, std=1.0, pitch=0, off=0):
    x = (torch.randn(M, K, generator=gen, device="cuda") * std).to(dtype)
    if not pitch:
        return x
    buf = torch.full((M * (K + pitch) + off + 8,), 7.0, dtype=dtype, device="cuda")
    v = buf[off: off + M * (K + pitch)].view(M, K + pitch)[:, :K]
    v.copy_(x)
    return v


class Problem:
    def __init__(self, qmm, dt, T, K, N, n, r, kind, x8=None, scaled=True, pitch=0, off=0, seed=None, std=1.0):
        self.qmm, self.dtype = qmm, HALVES[dt]
        gen = torch.Generator(device="cuda").manual_seed(T + K + N + n + r if seed is None else seed)
        self.T, self.K, self.N, self.n, self.r = T, K, N, n, r
        self.idx = adapters_of(T, n, kind, T + n)
        self.a = (torch.randn(n, r, K, generator=gen, device="cuda") * K**-0.5).to(self.dtype)
        self.b = (torch.randn(n, N, r, generator=gen, device="cuda") * 0.2).to(self.dtype)
        self.scale = torch.rand(n, generator=gen, device="cuda") * 2 - 0.3 if scaled else None
        self.x, self.x_scale = matrix(T, K, self.dtype, gen, std, pitch, off), None
        self.x64 = self.x.double()
        if x8:
            codes = None
            if pitch:
                codes = torch.zeros(T * (K + pitch) + off, dtype=torch.uint8, device="cuda").view(ref.ROW8[x8])[off:].view(T, K + pitch)[:, :K]
            self.x, self.x_scale = qmm.rows_quantize(self.x, codes=codes, dtype=ref.ROW8[x8])
            self.x64 = self.x.double() * self.x_scale.double()[:, None]
        self.y0, self.dy = (matrix(T, N, self.dtype, gen, 1.0, pitch, off) for _ in range(2))
        self.dx0 = matrix(T, K, self.dtype, gen, 1.0, pitch, off)
        self.out = matrix(T, N, self.dtype, gen, 1.0, pitch, off)
        self.dx = matrix(T, K, self.dtype, gen, 1.0, pitch, off)
        self.live = (self.idx >= 0) & (self.idx < n)

    def forward(self, **kw):
        self.s = torch.full((self.T, self.r), 5.0, device="cuda")
        args = dict(scale=self.scale, x_scale=self.x_scale, s=self.s, out=self.out)
        args.update(kw)
        return self.qmm.lora(self.x, self.idx, self.a, self.b, kw.pop("y0", self.y0), **{k: v for k, v in args.items() if k != "y0"})

    def check_forward(self, y, y0, s=True):
        s64, d, mag_s, mag_d, mag_ds = ref.lora(self.x64, self.idx, self.a.double(), self.b.double(), self.scale)
        e1, e2 = ref.sum_error(self.K), ref.sum_error(self.r)
        if s:
            got = torch.where(self.live[:, None], self.s.double(), 0.0)
            assert bool(((got - s64).abs() <= (e1 + 4 * 2.0**-24) * mag_s + 2.0**-126).all())
            assert bool((self.s[~self.live] == 5.0).all())
        want = d + (0 if y0 is None else y0.double())
        # s off by e1, its two halves by 2^-16 of the row's largest, the second sum, the addition, the rounding
        tol = (e1 + 8 * 2.0**-24) * mag_ds + (e2 + 2.0**-16) * (mag_d + mag_ds * e1) + 2.0**-23 * want.abs() + ref.rounding(want, self.dtype) * (1 + 2.0**-10)
        assert bool(((y.double() - want).abs() <= tol).all())
        if y0 is not None:
            assert torch.equal(y[~self.live], y0[~self.live])
        else:
            assert not y[~self.live].any()

    def backward(self, **kw):
        args = dict(dx0=self.dx0, scale=self.scale, x_scale=self.x_scale, dx=self.dx)
        args.update(kw)
        return self.qmm.lora_grad(self.dy, self.x, self.s, self.idx, self.a, self.b, **args)

    def check_backward(self, dx, da, db, dx0):
        n, T = self.n, self.T
        ds, d, mag_s, mag_d, mag_ds = ref.lora(self.dy.double(), self.idx, self.b.double().transpose(1, 2), self.a.double().transpose(1, 2), None)
        c = torch.ones(n, device="cuda", dtype=torch.float64) if self.scale is None else self.scale.double()
        row_c = torch.where(self.live, c[self.idx.clamp(0, n - 1).long()], 0.0)[:, None]
        ds, d, mag_s, mag_d, mag_ds = ds * row_c, d * row_c, mag_s * row_c.abs(), mag_d * row_c.abs(), mag_ds * row_c.abs()
        e1, e2 = ref.sum_error(self.N), ref.sum_error(self.r)
        want = d + (0 if dx0 is None else dx0.double())
        tol = (e1 + 8 * 2.0**-24) * mag_ds + (e2 + 2.0**-16) * (mag_d + mag_ds * e1) + 2.0**-23 * want.abs() + ref.rounding(want, self.dtype) * (1 + 2.0**-10)
        assert bool(((dx.double() - want).abs() <= tol).all())
        if dx0 is not None:
            assert torch.equal(dx[~self.live], dx0[~self.live])
        s = torch.where(self.live[:, None], self.s.double(), 0.0)
        x, dy = self.x64.abs(), self.dy.double()
        for e in range(n):
            t = torch.nonzero(self.idx == e)[:, 0]
            e3 = ref.sum_error(max(1, t.numel())) + 2.0**-15
            want = ds[t].T @ self.x64[t]
            tol = (e1 + 8 * 2.0**-24) * (mag_s[t].T @ x[t]) + e3 * (ds[t].abs().T @ x[t]) + 2.0**-126
            assert bool(((da[e].double() - want).abs() <= tol).all()), e
            want = c[e] * (dy[t].T @ s[t])
            assert bool(((db[e].double() - want).abs() <= e3 * c[e].abs() * (dy[t].abs().T @ s[t].abs()) + 2.0**-126).all()), e


SHAPES = [(1, 64, 32, 1, 8), (1, 2048, 2048, 4, 16), (3, 300, 100, 2, 16), (16, 1024, 512, 9, 64), (17, 257, 131, 3, 32), (100, 2048, 640, 1, 128), (200, 520, 1000, 7, 8),
          (256, 96, 72, 40, 16), (257, 256, 256, 2, 16), (300, 1000, 700, 3, 64), (700, 333, 1111, 5, 32), (1500, 2048, 264, 33, 8), (2100, 640, 1000, 1000, 16), (900, 72, 4096, 4, 128)]


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("kind", ["uniform", "dropped", "one", "none", "skewed"])
@pytest.mark.parametrize("T,K,N,n,r", SHAPES)
def test_forward_and_backward(qmm, dt, kind, T, K, N, n, r):
    p = Problem(qmm, dt, T, K, N, n, r, kind)
    y = p.forward()
    p.check_forward(y, p.y0)
    grads = p.backward()
    p.check_backward(*grads, p.dx0)
    first = [g.clone() for g in (y, p.s, *grads)]
    for g, h in zip(first, (p.forward(), p.s, *p.backward())):                     # the same bits again
        assert torch.equal(g, h) or g is p.s
    del first


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("x8", list(ref.ROW8))
@pytest.mark.parametrize("T,K,N,n,r", [(1, 64, 32, 1, 8), (20, 2048, 512, 6, 16), (100, 333, 200, 3, 32), (400, 1000, 304, 4, 64), (600, 515, 130, 2, 128), (300, 2048, 64, 5, 8)])
def test_rows_of_8_bits(qmm, dt, x8, T, K, N, n, r):
    p = Problem(qmm, dt, T, K, N, n, r, "dropped", x8=x8)
    p.check_forward(p.forward(), p.y0)
    p.check_backward(*p.backward(), p.dx0)


@pytest.mark.parametrize("x8", [None, "e4m3", "int8"])
@pytest.mark.parametrize("T", [40, 400])
@pytest.mark.parametrize("K,N,pitch,off", [(256, 512, 8, 8), (256, 512, 16, 16), (256, 512, 3, 1), (200, 333, 8, 8), (101, 104, 7, 5)])
def test_strides(qmm, x8, T, K, N, pitch, off):
    p = Problem(qmm, "bf16", T, K, N, 3, 16, "dropped", x8=x8, pitch=pitch, off=off)
    p.check_forward(p.forward(), p.y0)
    p.check_backward(*p.backward(), p.dx0)
    for v in (p.out, p.dx):
        gap = v.as_strided((v.shape[0] - 1, pitch), (v.stride(0), 1), v.storage_offset() + v.shape[1])
        assert bool((gap == 7.0).all())


@pytest.mark.parametrize("T", [30, 500])
def test_in_place_and_without_a_base(qmm, T):
    p = Problem(qmm, "f16", T, 300, 520, 4, 16, "dropped", scaled=False)
    y0, dx0 = p.y0.clone(), p.dx0.clone()
    y = p.forward(out=p.y0)
    assert y is p.y0
    p.check_forward(y, y0)
    dx, da, db = p.backward(dx=p.dx0)
    assert dx is p.dx0
    p.check_backward(dx, da, db, dx0)
    y = p.forward(y0=None)
    p.check_forward(y, None)
    p.check_backward(*p.backward(dx0=None), None)
    p.check_forward(p.forward(s=None, y0=y0), y0, s=False)


@pytest.mark.parametrize("T", [50, 600])
def test_one_sort_for_many(qmm, T):
    p = Problem(qmm, "bf16", T, 256, 320, 6, 32, "dropped")
    plan = qmm.expert_sort(p.idx.view(-1, 1), p.n)
    a = [g.clone() for g in (p.forward(plan=plan), p.s, *p.backward(plan=plan))]
    for g, h in zip(a, (p.forward(), p.s, *p.backward())):
        assert torch.equal(g, h)


@pytest.mark.parametrize("T", [64, 640])
def test_parts_alone(qmm, T):
    """Each gradient by itself gives the bits that all together give."""
    p = Problem(qmm, "bf16", T, 256, 320, 3, 16, "uniform")
    p.forward()
    dx, da, db = (g.clone() for g in p.backward())
    L, ws = qmm.lib(), torch.empty(qmm.lora_workspace_bytes(T, p.n, p.r), dtype=torch.uint8, device="cuda")
    for want, which in ((dx, "dX"), (da, "dA"), (db, "dB")):
        out = torch.full_like(want, 3.0)
        q = qmm.LoraArgs(T=T, n=p.n, r=p.r, dtype=1, K=p.K, N=p.N, X=p.x.data_ptr(), ldx=p.K, idx=p.idx.data_ptr(), A=p.a.data_ptr(), B=p.b.data_ptr(),
                         scale=p.scale.data_ptr(), S=p.s.data_ptr(), dY=p.dy.data_ptr(), lddy=p.N, dX0=p.dx0.data_ptr(), lddx0=p.K, lddx=p.K)
        setattr(q, which, out.data_ptr())
        import ctypes
        assert L.qmm_lora_grad(ctypes.byref(q), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0, qmm.last_error()
        assert torch.equal(out, want), which


def test_what_is_not_wanted(qmm):
    """False in place of a gradient: the others come alone, and what they do not need may be missing."""
    p = Problem(qmm, "f16", 90, 128, 160, 3, 16, "dropped")
    p.forward()
    dx, da, db = (g.clone() for g in p.backward())
    got = p.backward(dx=False, da=False)
    assert got[:2] == (None, None) and torch.equal(got[2], db)
    got = qmm.lora_grad(p.dy, None, None, p.idx, p.a, p.b, p.dx0, scale=p.scale, da=False, db=False)
    assert got[1:] == (None, None) and torch.equal(got[0], dx)
    got = qmm.lora_grad(p.dy, p.x, None, p.idx, p.a, p.b, scale=p.scale, dx=False, db=False)
    assert torch.equal(got[1], da)
    with pytest.raises(qmm.QmmError):
        qmm.lora_grad(p.dy, p.x, None, p.idx, p.a, p.b)
    with pytest.raises(AssertionError):
        qmm.lora_grad(p.dy, None, p.s, p.idx, p.a, p.b)


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("T,K,N,n,r", [(1, 160, 96, 1, 8), (70, 333, 263, 3, 16), (90, 512, 768, 4, 32), (300, 512, 520, 3, 64), (330, 257, 100, 2, 128), (1000, 128, 128, 20, 8),
                                       (40, 128, 64, 2, 128), (600, 96, 640, 2, 16)])
def test_integers_are_exact(qmm, dt, T, K, N, n, r):
    """Small integers: every product and sum is exact, so the results are the exact ones, rounded once."""
    p = Problem(qmm, dt, T, K, N, n, r, "dropped")
    gen = torch.Generator(device="cuda").manual_seed(1)

    def ints(t, lo, hi):
        return torch.randint(lo, hi + 1, t.shape, generator=gen, device="cuda").to(t.dtype)
    p.x, p.a, p.b, p.y0, p.dy, p.dx0 = ints(p.x, -2, 2), ints(p.a, -1, 1), ints(p.b, -1, 1), ints(p.y0, -50, 50), ints(p.dy, -2, 2), ints(p.dx0, -50, 50)
    p.scale = torch.tensor([0.5, 2.0, 1.0], device="cuda")[torch.arange(n, device="cuda") % 3]
    p.x64 = p.x.double()
    y = p.forward()
    s, d, *_ = ref.lora(p.x64, p.idx, p.a.double(), p.b.double(), p.scale)
    assert torch.equal(p.s[p.live].double(), s[p.live])
    assert torch.equal(y, (d + p.y0.double()).to(p.dtype))
    dx, da, db = p.backward()
    ds, d, *_ = ref.lora(p.dy.double(), p.idx, p.b.double().transpose(1, 2), p.a.double().transpose(1, 2), None)
    c = torch.where(p.live, p.scale.double()[p.idx.clamp(0, n - 1).long()], 0.0)[:, None]
    assert torch.equal(dx, (d * c + p.dx0.double()).to(p.dtype))
    for e in range(n):
        t = torch.nonzero(p.idx == e)[:, 0]
        assert torch.equal(da[e].double(), (ds * c)[t].T @ p.x64[t]) and torch.equal(db[e].double(), p.scale[e].double() * (p.dy.double()[t].T @ s[t])), e


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("T,K,N,n,r,kind", [(513, 64, 8, 1, 8, "one"), (4097, 136, 264, 5, 16, "skewed"), (2000, 72, 200, 1024, 8, "uniform"), (700, 130, 77, 1024, 16, "one"),
                                            (3000, 256, 128, 3, 32, "none"), (20000, 2056, 136, 3, 32, "skewed"), (1500, 300, 133, 4, 128, "dropped"), (900, 101, 520, 6, 64, "uniform"),
                                            (6000, 128, 1300, 40, 64, "skewed")])
def test_rows_shared_by_blocks(qmm, dt, x8, T, K, N, n, r, kind):
    """Many rows: the blocks of a weight gradient share all adapters' rows.  Integers, so that every sum is exact whoever adds what; a workspace of exactly the size asked for,
    full of NaN, with other memory behind it."""
    p = Problem(qmm, dt, T, K, N, n, r, kind)
    gen = torch.Generator(device="cuda").manual_seed(3)

    def ints(shape, lo, hi, dtype):
        return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda").to(dtype)
    ds_of = ints((T, r), -9, 9, torch.float32)
    x = ints((T, K), -2, 2, torch.int8 if x8 else p.dtype)
    xs = torch.tensor([0.5, 1.0, 2.0], device="cuda")[torch.arange(T, device="cuda") % 3] if x8 else None
    dy, b = ints((T, N), -2, 2, p.dtype), torch.zeros_like(p.b)
    b[:, : min(N, r)] = torch.eye(r, device="cuda", dtype=p.dtype)[: min(N, r)]             # ds = scale * the first elements of dy
    scale = torch.tensor([0.5, 2.0, 1.0], device="cuda")[torch.arange(n, device="cuda") % 3]
    need = qmm.lora_workspace_bytes(T, n, r)
    buf = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    args = dict(scale=scale, x_scale=xs, ws=buf[:need])
    _, da, db = qmm.lora_grad(dy, x, ds_of, p.idx, p.a, b, dx=False, **args)
    one_a = qmm.lora_grad(dy, x, None, p.idx, p.a, b, dx=False, db=False, **args)[1]
    one_b = qmm.lora_grad(dy, None, ds_of, p.idx, p.a, b, dx=False, da=False, scale=scale, ws=buf[:need])[2]
    assert bool((buf[need:] == 255).all())
    ds = torch.zeros(T, r, device="cuda", dtype=torch.float64)
    ds[:, : min(N, r)] = dy[:, : min(N, r)].double()
    xd = x.double() * (xs.double()[:, None] if x8 else 1.0)
    for e in range(n):
        t = torch.nonzero(p.idx == e)[:, 0]
        want_a, want_b = scale[e].double() * ds[t].T @ xd[t], scale[e].double() * dy[t].double().T @ ds_of[t].double()
        for got, want in ((da[e], want_a), (one_a[e], want_a), (db[e], want_b), (one_b[e], want_b)):
            assert torch.equal(got.double(), want), "adapter %d of %d" % (e, n)


@pytest.mark.parametrize("dt,std", [("f16", 2.0**-20), ("f16", 3e4), ("bf16", 1e-30), ("bf16", 1e30)])
@pytest.mark.parametrize("T", [20, 300])
def test_rows_far_from_one(qmm, dt, std, T):
    """s beyond fp16's range and far below it: B of the other size brings the result back."""
    p = Problem(qmm, dt, T, 512, 256, 2, 16, "uniform", scaled=False)
    p.x = (p.x.double() * std).clamp(-6e4 if dt == "f16" else -1e38, 6e4 if dt == "f16" else 1e38).to(p.dtype)
    p.x64 = p.x.double()
    p.b = (p.b.double() * max(1e-3, min(1e3, 1 / std))).to(p.dtype)
    if dt == "f16":
        p.a *= 8
    p.check_forward(p.forward(), p.y0)
    p.dy = (p.dy.double() * max(2.0**-12, min(1.0, std))).to(p.dtype)
    p.check_backward(*p.backward(), p.dx0)


def test_a_mixed_row_does_not_touch_the_others(qmm):
    """A row of infinities and NaN changes its own outputs alone, and its adapter's gradients."""
    for T in (30, 400):
        p = Problem(qmm, "bf16", T, 256, 320, 3, 16, "uniform")
        y = p.forward().clone()
        dx, da, db = (g.clone() for g in p.backward())
        p.x[5, 7], p.x[9, 8] = float("inf"), float("nan")
        p.dy[9, 3] = float("nan")
        y2 = p.forward()
        dx2, da2, db2 = p.backward()
        others = torch.arange(T, device="cuda")
        others = others[(others != 5) & (others != 9)]
        assert torch.equal(y[others], y2[others]) and torch.equal(dx[others], dx2[others])
        assert not torch.isfinite(y2[5]).any() and torch.isnan(y2[9]).all() and torch.isnan(dx2[9]).all()
        hit = {int(p.idx[5]), int(p.idx[9])}
        for e in set(range(3)) - hit:
            assert torch.equal(da[e], da2[e]) and torch.equal(db[e], db2[e])


def test_gradients_against_differences(qmm):
    p = Problem(qmm, "bf16", 12, 40, 24, 2, 8, "uniform")
    p.forward()
    dx, da, db = p.backward(dx0=None)

    def f(x, a, b):
        return float((ref.lora(x, p.idx, a, b, p.scale)[1] * p.dy.double()).sum())
    x, a, b = p.x64, p.a.double(), p.b.double()
    h = 2.0**-6                                            # the function is linear in each argument: differences are exact up to rounding
    for name, got, t in (("x", dx, x), ("a", da, a), ("b", db, b)):
        flat = list(itertools.islice(itertools.product(*(range(0, n, max(1, n // 3)) for n in t.shape)), 20))
        for at in flat:
            args = {"x": x, "a": a, "b": b}
            vals = []
            for sign in (1, -1):
                m = t.clone()
                m[at] += sign * h
                vals.append(f(**{**args, name: m}))
            want = (vals[0] - vals[1]) / (2 * h)
            assert abs(want - float(got[at])) <= 2.0**-8 * abs(want) + 1e-3, (name, at)


def test_no_rows(qmm):
    a, b = torch.ones(2, 8, 32, dtype=torch.float16, device="cuda"), torch.ones(2, 16, 8, dtype=torch.float16, device="cuda")
    x, y = torch.empty(0, 32, dtype=torch.float16, device="cuda"), torch.empty(0, 16, dtype=torch.float16, device="cuda")
    idx = torch.empty(0, dtype=torch.int32, device="cuda")
    assert qmm.lora(x, idx, a, b, y).shape == (0, 16)
    dx, da, db = qmm.lora_grad(y, x, None, idx, a, b)
    assert dx.shape == (0, 32) and not da.any() and not db.any()


@pytest.mark.parametrize("dt,x8", [("f16", None), ("bf16", None), ("bf16", "e4m3")])
@pytest.mark.parametrize("T,K,N", [(300, 256, 136), (300, 131, 136), (300, 256, 77), (900, 256, 136), (900, 131, 136), (900, 256, 77)])
def test_one_workspace_for_call_after_call(qmm, dt, x8, T, K, N):
    """Calls on one workspace right behind one another, each with other rows of other adapters: both weight gradients read the sort and the dS of their own call.  Small integers: every
    sum is exact, whoever adds what."""
    n, r, calls = 5, 16, 12
    p = Problem(qmm, dt, T, K, N, n, r, "uniform", x8=x8)
    gen = torch.Generator(device="cuda").manual_seed(7)

    def ints(shape, lo, hi, dtype):
        return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda").to(dtype)
    b = ints(p.b.shape, -1, 1, p.dtype)
    ws = torch.full((qmm.lora_workspace_bytes(T, n, r),), 255, dtype=torch.uint8, device="cuda")
    each = []
    for _ in range(calls):
        x = ints((T, K), -2, 2, torch.float32).to(ref.ROW8[x8] if x8 else p.dtype)
        each.append((ints((T,), -1, n - 1, torch.int32), x, ints((T, N), -2, 2, p.dtype), ints((T, r), -9, 9, torch.float32)))
    ones = torch.ones(T, device="cuda") if x8 else None
    torch.cuda.synchronize()
    got = [qmm.lora_grad(dy, x, s, idx, p.a, b, x_scale=ones, dx=False, ws=ws)[1:] for idx, x, dy, s in each]
    for (idx, x, dy, s), (da, db) in zip(each, got):
        for e in range(n):
            t = torch.nonzero(idx == e)[:, 0]
            ds = dy[t].double() @ b[e].double()
            assert torch.equal(da[e].double(), ds.T @ x[t].double()) and torch.equal(db[e].double(), dy[t].double().T @ s[t].double())


# ---- the form for more than 512 rows, against the formulas

@pytest.mark.parametrize("x8", [None, "e4m3", "int8"])
@pytest.mark.parametrize("dt,K,N,r,pitch,off", [("bf16", 256, 512, 16, 8, 8), ("f16", 264, 136, 32, 16, 16), ("bf16", 256, 512, 64, 3, 1), ("f16", 200, 333, 8, 8, 8), ("bf16", 101, 104, 16, 7, 5),
                                                ("bf16", 130, 258, 128, 2, 2), ("f16", 257, 131, 64, 4, 4)])
def test_many_rows_with_gaps(qmm, dt, x8, K, N, r, pitch, off):
    p = Problem(qmm, dt, 700, K, N, 3, r, "dropped", x8=x8, pitch=pitch, off=off)
    p.check_forward(p.forward(), p.y0)
    p.check_backward(*p.backward(), p.dx0)
    for v in (p.out, p.dx):
        gap = v.as_strided((v.shape[0] - 1, pitch), (v.stride(0), 1), v.storage_offset() + v.shape[1])
        assert bool((gap == 7.0).all())


@pytest.mark.parametrize("dt,r", [("f16", 16), ("bf16", 64)])
@pytest.mark.parametrize("K,N", [(300, 520), (264, 1111), (1024, 256)])
def test_many_rows_in_place_and_without_a_base(qmm, dt, r, K, N):
    p = Problem(qmm, dt, 1100, K, N, 4, r, "dropped", scaled=False)
    y0, dx0 = p.y0.clone(), p.dx0.clone()
    y = p.forward(out=p.y0)
    assert y is p.y0
    p.check_forward(y, y0)
    dx, da, db = p.backward(dx=p.dx0)
    assert dx is p.dx0
    p.check_backward(dx, da, db, dx0)
    y = p.forward(y0=None)
    p.check_forward(y, None)
    p.check_backward(*p.backward(dx0=None), None)
    p.check_forward(p.forward(s=None, y0=y0), y0, s=False)


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("kind", ["dropped", "skewed"])
@pytest.mark.parametrize("T,K,N,n,r", [(600, 512, 768, 4, 8), (700, 1024, 640, 5, 32), (1030, 640, 1024, 3, 64), (800, 1000, 2056, 6, 64), (513, 2048, 128, 2, 128), (2500, 136, 264, 70, 32)])
def test_many_aligned_rows(qmm, dt, kind, T, K, N, n, r):
    p = Problem(qmm, dt, T, K, N, n, r, kind)
    p.check_forward(p.forward(), p.y0)
    p.check_backward(*p.backward(), p.dx0)


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("x8", list(ref.ROW8))
@pytest.mark.parametrize("T,K,N,n,r", [(600, 264, 136, 3, 8), (900, 1024, 520, 5, 16), (1500, 1000, 304, 4, 32), (700, 2048, 256, 2, 64), (640, 260, 200, 3, 16), (520, 515, 130, 2, 64), (800, 72, 1000, 9, 128)])
def test_many_rows_of_8_bits(qmm, dt, x8, T, K, N, n, r):
    p = Problem(qmm, dt, T, K, N, n, r, "dropped", x8=x8)
    p.check_forward(p.forward(), p.y0)
    p.check_backward(*p.backward(), p.dx0)


@pytest.mark.parametrize("dt,std", [("f16", 2.0**-20), ("f16", 3e4), ("bf16", 1e-30), ("bf16", 1e30)])
@pytest.mark.parametrize("K,N,r", [(512, 256, 16), (333, 131, 64)])
def test_many_rows_far_from_one(qmm, dt, std, K, N, r):
    p = Problem(qmm, dt, 900, K, N, 2, r, "uniform", scaled=False)
    p.x = (p.x.double() * std).clamp(-6e4 if dt == "f16" else -1e38, 6e4 if dt == "f16" else 1e38).to(p.dtype)
    p.x64 = p.x.double()
    p.b = (p.b.double() * max(1e-3, min(1e3, 1 / std))).to(p.dtype)
    if dt == "f16":
        p.a *= 8
    p.check_forward(p.forward(), p.y0)
    p.dy = (p.dy.double() * max(2.0**-12, min(1.0, std))).to(p.dtype)
    p.check_backward(*p.backward(), p.dx0)


@pytest.mark.parametrize("K,N,r", [(256, 320, 16), (256, 320, 64), (131, 77, 32)])
def test_a_mixed_row_among_many_does_not_touch_the_others(qmm, K, N, r):
    T = 900
    p = Problem(qmm, "bf16", T, K, N, 3, r, "uniform")
    y = p.forward().clone()
    dx, da, db = (g.clone() for g in p.backward())
    p.x[5, 7], p.x[9, 8] = float("inf"), float("nan")
    p.dy[9, 3] = float("nan")
    y2 = p.forward()
    dx2, da2, db2 = p.backward()
    others = torch.arange(T, device="cuda")
    others = others[(others != 5) & (others != 9)]
    assert torch.equal(y[others], y2[others]) and torch.equal(dx[others], dx2[others])
    assert not torch.isfinite(y2[5]).any() and torch.isnan(y2[9]).all() and torch.isnan(dx2[9]).all()
    for e in set(range(3)) - {int(p.idx[5]), int(p.idx[9])}:
        assert torch.equal(da[e], da2[e]) and torch.equal(db[e], db2[e])


# ---- the bits that the weight gradients keep

@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("T", [40, 600])
@pytest.mark.parametrize("K,N,r", [(136, 136, 8), (131, 77, 16), (128, 264, 32), (264, 128, 64), (136, 200, 128)])
def test_all_bits_of_s_reach_the_weight_gradients(qmm, dt, T, K, N, r):
    """A row for each adapter, ones for x and dy: dB is s, dA is dS, with all their 24 bits (three bf16 parts) or 22 of them (two tf32 parts).  A sum of parts is cut 25 bits below
    its largest one, which is 2^-24 for each of the three or four; 2^-22 covers both."""
    dtype, gen = HALVES[dt], torch.Generator(device="cuda").manual_seed(T + K)
    idx = torch.randperm(T, generator=gen, device="cuda").int()
    s = (1 + torch.rand(T, r, generator=gen, device="cuda")) * torch.where(torch.rand(T, r, generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    x, a = torch.ones(T, K, dtype=dtype, device="cuda"), torch.zeros(T, r, K, dtype=dtype, device="cuda")
    dy = torch.ones(T, N, dtype=dtype, device="cuda")
    _, _, db = qmm.lora_grad(dy, x, s, idx, a, torch.zeros(T, N, r, dtype=dtype, device="cuda"), dx=False)
    want = s[torch.argsort(idx.long())][:, None, :].double().expand(T, N, r)
    assert bool(((db.double() - want).abs() <= 2.0**-22 * want.abs()).all())
    # dS = b[0] + b[1] + ... of powers of two that add up to 24 bits without a rounding
    b = torch.zeros(T, N, r, dtype=dtype, device="cuda")
    bits = torch.randint(0, 2, (T, 23, r), generator=gen, device="cuda")
    b[:, 0] = 1
    b[:, 1:24] = (bits * 2.0 ** -torch.arange(1, 24, device="cuda")[None, :, None]).to(dtype)
    want = b.double().sum(1)
    _, da, _ = qmm.lora_grad(dy, x, s, idx, a, b, dx=False, db=False)
    want = want[:, :, None].expand(T, r, K)
    # the sum of dS on the tensor cores: at most two products of 32 elements, cut 25 bits below the largest
    assert bool(((da.double() - want).abs() <= (2.0**-22 + 2.0**-23) * want.abs()).all())


@pytest.mark.parametrize("dt", list(HALVES))
@pytest.mark.parametrize("K,N,r", [(136, 136, 16), (131, 77, 32), (264, 264, 64), (128, 200, 128)])
def test_sums_over_many_rows_are_rounded_to_nearest(qmm, dt, K, N, r):
    """8192 rows of one adapter: a weight gradient is the sum of T / 16 = 512 short products at most, each addition rounded to nearest.  Partial sums of random signs grow with the
    root of their length, so the roundings add up to 2^-24 / sqrt(3) sqrt(512 / 2) = 5.5e-7 of the result's norm; the products' own cuts (2^-24 for each of four, of a
    part's size) add less than 2e-7.  Sums that are cut instead, all to one side, are off by 2e-6."""
    T, dtype, gen = 8192, HALVES[dt], torch.Generator(device="cuda").manual_seed(K)
    idx = torch.zeros(T, dtype=torch.int32, device="cuda")
    x, dy = (torch.randn(T, w, generator=gen, device="cuda").to(dtype) for w in (K, N))
    s = torch.randn(T, r, generator=gen, device="cuda")
    b = torch.zeros(1, N, r, dtype=dtype, device="cuda")
    b[0, : min(N, r)] = torch.eye(r, device="cuda", dtype=dtype)[: min(N, r)]               # dS: the first elements of dy, exactly
    _, da, db = qmm.lora_grad(dy, x, s, idx, torch.zeros(1, r, K, dtype=dtype, device="cuda"), b, dx=False)
    ds = torch.zeros(T, r, dtype=torch.float64, device="cuda")
    ds[:, : min(N, r)] = dy[:, : min(N, r)].double()
    for got, want in ((da[0], ds.T @ x.double()), (db[0], dy.double().T @ s.double())):
        assert (got.double() - want).norm() <= 7.5e-7 * want.norm()


@pytest.mark.parametrize("dt,x8", [("f16", None), ("bf16", None), ("bf16", "int8")])
@pytest.mark.parametrize("T", [40, 700])
@pytest.mark.parametrize("K,N,r,off_a,off_b", [(256, 136, 16, 1, 1), (256, 136, 64, 2, 1), (130, 258, 8, 1, 2), (131, 77, 32, 3, 5), (264, 264, 128, 8, 1), (256, 512, 32, 1, 8)])
def test_adapters_that_begin_at_any_element(qmm, dt, x8, T, K, N, r, off_a, off_b):
    """A and B as contiguous pieces of larger tensors, beside rows that are aligned, rows of whole words, and no base at all."""
    p = Problem(qmm, dt, T, K, N, 3, r, "dropped", x8=x8)

    def at(t, off):
        buf = torch.full((t.numel() + 16,), 7.0, dtype=t.dtype, device="cuda")
        v = buf[off: off + t.numel()].view(t.shape)
        v.copy_(t)
        return v
    p.a, p.b = at(p.a, off_a), at(p.b, off_b)
    p.check_forward(p.forward(), p.y0)
    p.check_backward(*p.backward(), p.dx0)
    p.check_forward(p.forward(y0=None), None)
    p.check_backward(*p.backward(dx0=None), None)
