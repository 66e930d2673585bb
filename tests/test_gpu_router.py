"""GPU parity: a router's choice and its gradient, and its way into the experts' operators."""
import itertools
import math

import pytest
import torch

from tests import layerref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qmm():
    from paper_2607_00501_b200 import qmm as _qmm
    assert torch.cuda.is_available()
    _qmm.lib()
    return _qmm


def logits_of(T, E, dt, kind, seed):
    gen = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=gen) * 1.5
    if kind == "ties":
        l = (l * 2).round() / 2
    elif kind == "wide":
        l = l * 60
    elif kind == "masked":
        l[torch.rand(T, E, generator=gen) < 0.4] = -math.inf
        l[::5] = -math.inf                                 # nothing left
        l[1::7, E // 2:] = -math.inf
    elif kind == "ends":                                   # the type's ends, NaN and infinities
        ends = torch.tensor([torch.finfo(ref.DTYPES[dt]).min, torch.finfo(ref.DTYPES[dt]).max, math.inf, -math.inf, math.nan, -100.0, -200.0, 0.0])
        l = torch.where(torch.rand(T, E, generator=gen) < 0.5, ends[torch.randint(0, 8, (T, E), generator=gen)], l)
        l[0] = torch.finfo(ref.DTYPES[dt]).min
        l[1] = math.nan
    elif kind == "low":                                    # every score underflows in 32 bits
        l = l - 150
    return l.to(ref.DTYPES[dt])


def check(qmm, l, topk, sigmoid, bias, G, top, group_top, renorm, scale=1.5, pitch=None, off=0):
    T, E = l.shape
    x = l.cuda()
    if pitch:
        buf = torch.full((T * pitch + off + 8,), 9.0, dtype=l.dtype, device="cuda")
        x = buf[off: off + T * pitch].view(T, pitch)[:, :E]
        x.copy_(l)
    idx, w = qmm.expert_route(x, topk, qmm.SIGMOID if sigmoid else qmm.SOFTMAX, None if bias is None else bias.cuda(), G, top, group_top, renorm, scale)
    want_idx, want = ref.route(l, topk, sigmoid, bias, G, top, group_top, renorm, scale)
    assert torch.equal(idx.cpu().long(), want_idx)
    # expf: 2 ulp and the rounding of its argument (|l - m| 2^-24 relative), a sum of up to 1024 parts in at most 32 + 5 additions, a division, the scale
    lc = ref.clean(l)
    far = torch.where(lc > -math.inf, (lc.amax(1, keepdim=True) - lc).clamp(max=200), 0.0)
    tol = (far.gather(1, want_idx.clamp(min=0)) + 64) * 2.0**-24 * want + 2.0**-126
    assert bool(((w.cpu().double() - want).abs() <= tol).all())
    return x, idx, w


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("sigmoid,renorm", list(itertools.product((False, True), repeat=2)))
@pytest.mark.parametrize("T,E,topk,G,top,group_top", [(1, 1, 1, 1, 1, 1), (1, 128, 8, 1, 1, 1), (33, 46, 7, 1, 1, 1), (70, 256, 8, 8, 4, 2), (40, 160, 6, 8, 3, 1),
                                                      (21, 96, 32, 3, 2, 2), (5, 1024, 32, 32, 5, 2), (9, 1023, 8, 1, 1, 1), (18, 64, 4, 32, 9, 2), (50, 31, 31, 1, 1, 1)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_choice_and_weights(qmm, dt, sigmoid, renorm, T, E, topk, G, top, group_top, with_bias):
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)) * 0.1 if with_bias else None
    check(qmm, logits_of(T, E, dt, "plain", T * E), topk, sigmoid, bias, G, top, group_top, renorm)


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("kind", ["ties", "wide", "masked", "ends", "low"])
@pytest.mark.parametrize("sigmoid,renorm", list(itertools.product((False, True), repeat=2)))
@pytest.mark.parametrize("E,topk,G,top,group_top,with_bias", [(64, 6, 1, 1, 1, False), (64, 6, 1, 1, 1, True), (48, 8, 4, 2, 2, False), (48, 8, 4, 2, 2, True), (40, 5, 8, 3, 1, False)])
def test_ties_masks_and_ends(qmm, dt, kind, sigmoid, renorm, E, topk, G, top, group_top, with_bias):
    bias = (torch.randn(E, generator=torch.Generator().manual_seed(3)) * 0.1).round(decimals=1) if with_bias else None
    check(qmm, logits_of(60, E, dt, kind, E), topk, sigmoid, bias, G, top, group_top, renorm)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_neighbours_nearer_than_32_bits_tell(qmm, sigmoid):
    """Biases that undo the scores to within 1e-9: the order is that of the 64-bit sums."""
    T, E = 200, 64
    gen = torch.Generator().manual_seed(1)
    l = torch.randn(1, E, generator=gen)
    s = ref.scores(l.double(), sigmoid)
    bias = (0.75 - s[0]).float()
    check(qmm, l.expand(T, E).contiguous(), 8, sigmoid, bias, 1, 1, 1, True)
    check(qmm, l.expand(T, E).contiguous(), 8, sigmoid, bias, 8, 4, 2, True)
    check(qmm, (l + torch.randn(T, 1, generator=gen) * 1e-7).contiguous(), 8, sigmoid, bias, 8, 4, 2, False)


def test_biases_that_switch_experts_off(qmm):
    l = logits_of(30, 32, "f32", "plain", 4)
    bias = torch.zeros(32)
    bias[3::4] = -math.inf
    bias[2] = math.nan
    idx = check(qmm, l, 30, True, bias, 1, 1, 1, True)[1].cpu()
    assert not ((idx >= 0) & (idx % 4 == 3)).any() and not (idx == 2).any() and (idx[:, 23:] == -1).all()
    bias[5] = math.inf
    assert (check(qmm, l, 4, True, bias, 4, 2, 1, True)[1].cpu()[:, 0] == 5).all()


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("pitch,off", [(131, 1), (136, 8), (130, 2)])
def test_strides(qmm, dt, pitch, off):
    check(qmm, logits_of(40, 128, dt, "plain", 9), 8, False, None, 1, 1, 1, True, pitch=pitch, off=off)


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("kind", ["plain", "masked", "wide", "low"])
@pytest.mark.parametrize("sigmoid,renorm", list(itertools.product((False, True), repeat=2)))
@pytest.mark.parametrize("T,E,topk,pitch", [(1, 1, 1, None), (40, 128, 8, None), (33, 46, 7, None), (12, 1024, 32, None), (20, 64, 1, None), (25, 64, 6, 67)])
def test_gradient(qmm, dt, kind, sigmoid, renorm, T, E, topk, pitch):
    if E == 1 and kind == "masked":
        kind = "plain"
    l = logits_of(T, E, dt, kind, T + E)
    x, idx, w = check(qmm, l, topk, sigmoid, None, 1, 1, 1, renorm, pitch=pitch)
    dw = torch.randn(T, topk, generator=torch.Generator().manual_seed(2))
    dw[w.cpu() == 0] = math.nan if not (kind in ("wide", "low") and not renorm) else 1.0         # nothing is read at dropped slots
    dw = torch.where(idx.cpu() >= 0, torch.nan_to_num(dw, nan=1.0), dw)
    out = torch.full_like(x, 7.0) if pitch is None else None
    got = qmm.expert_route_grad(dw.cuda(), x, idx, qmm.SIGMOID if sigmoid else qmm.SOFTMAX, renorm, 1.5, out=out).cpu().double()
    full = ref.clean(l).requires_grad_()
    i = idx.cpu().long()
    g = torch.where(i >= 0, dw.double(), 0.0)
    live = (full > -math.inf).any(1)                       # (rows without an expert have no softmax)
    want = torch.zeros_like(full)
    if live.any():
        sub = full[live]
        want[live] = torch.autograd.grad((ref.route_weights(sub, i[live], sigmoid, renorm, 1.5) * g[live]).sum(), sub)[0]
    want = torch.nan_to_num(want, nan=0.0)
    # p (|g_i| + |g|.p) bounds what cancels; its factors are off like the weights
    s = ref.scores(full.detach(), sigmoid)
    p = torch.zeros_like(s).scatter_add_(1, i.clamp(min=0), torch.where(i >= 0, w.cpu().double() / 1.5, 0.0))
    p = torch.maximum(p, torch.zeros_like(p) if sigmoid or renorm else s)
    gg = 1.5 * torch.zeros_like(s).scatter_add_(1, i.clamp(min=0), g.abs())
    far = torch.where(full > -math.inf, (full.amax(1, keepdim=True) - full).clamp(max=200), 0.0).detach()
    tol = (far + far.amax(1, keepdim=True).clamp(max=30) + 160) * 2.0**-24 * p * (gg + (gg * p).sum(1, keepdim=True)) + ref.rounding(want, l.dtype) + 2.0**-126
    assert bool(((got - want).abs() <= tol).all())


def test_gradient_against_differences(qmm):
    T, E, topk = 6, 24, 5
    l = logits_of(T, E, "f32", "plain", 8)
    dw = torch.randn(T, topk, generator=torch.Generator().manual_seed(3))
    for sigmoid, renorm in itertools.product((False, True), repeat=2):
        idx, _ = qmm.expert_route(l.cuda(), topk, int(sigmoid), renormalize=renorm)
        got = qmm.expert_route_grad(dw.cuda(), l.cuda(), idx, int(sigmoid), renorm).cpu().double()
        i = idx.cpu().long()
        for t, e in itertools.product(range(T), range(0, E, 3)):
            h = 2.0**-10
            d = []
            for sign in (1, -1):
                m = l.double().clone()
                m[t, e] += sign * h
                d.append(float((ref.route_weights(m, i, sigmoid, renorm, 1.0) * dw.double()).sum()))
            # third derivatives of the weights are below 1 in magnitude per |dw|, so the difference is off by h^2 / 6 of sum |dw| at most
            assert abs((d[0] - d[1]) / (2 * h) - float(got[t, e])) <= h * h * float(dw.abs().sum()) + 1e-5


def test_gradient_of_the_same_expert_twice(qmm):
    l = logits_of(3, 40, "f32", "plain", 2)
    idx = torch.tensor([[4, 4, 9], [7, -1, 7], [1, 2, 3]], dtype=torch.int32)
    dw = torch.randn(3, 3, generator=torch.Generator().manual_seed(2))
    got = qmm.expert_route_grad(dw.cuda(), l.cuda(), idx.cuda(), renormalize=False).cpu()
    full = l.double().requires_grad_()
    want = torch.autograd.grad((ref.route_weights(full, idx.long(), False, False, 1.0) * torch.where(idx >= 0, dw, 0.0).double()).sum(), full)[0]
    assert torch.allclose(got.double(), want, atol=1e-6)


def test_route_into_the_experts(qmm):
    """logits -> choice -> sort, gather, combine and back: gradients of x and of the logits against torch's own; a masked token gets nothing."""
    T, H, E, topk = 50, 64, 16, 3
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(T, H, generator=gen, device="cuda")
    l = torch.randn(T, E, generator=gen, device="cuda")
    l[7] = -math.inf
    l[9, 2:] = -math.inf
    target = torch.randn(T, H, generator=gen, device="cuda")
    idx, w = qmm.expert_route(l, topk, qmm.SIGMOID, scale=2.0)
    assert (idx[7] == -1).all() and (idx[9] == -1).sum() == 1 and abs(float(w[9].sum()) - 2.0) < 1e-5
    plan = qmm.expert_sort(idx, E)
    xs = qmm.expert_gather(x, plan)
    y = qmm.expert_combine(xs, plan, w)
    dy = 2 * (y - target)
    dxs, dw = qmm.expert_combine_grad(dy, xs, plan, w)
    dx = qmm.expert_gather_grad(dxs, plan)
    dl = qmm.expert_route_grad(dw, l, idx, qmm.SIGMOID, scale=2.0)
    x64, l64 = x.double().requires_grad_(), l.double().requires_grad_()
    y64 = ref.route_weights(l64, idx.long(), True, True, 2.0).sum(1, keepdim=True) * x64
    gx, gl = torch.autograd.grad(((y64 - target.double()) ** 2).sum(), (x64, l64))
    assert not y[7].any() and not dl[7].any()
    # the weights of a token add up to 2 whatever its logits, so the exact gradient of the logits is zero up to dy . x summed in 32 bits
    assert (dx.double() - gx).norm() / gx.norm() < 1e-5
    assert (dl.double() - gl).abs().max() < 64 * 2.0**-23 * (dy.abs() * x.abs()).sum(1).max() * 2


def bucketed(E, sigmoid, T, topk, targets, seed):
    """Logits and biases that bring the scores of `targets` (expert -> value) there, to within the roundings of the logits, topk - 1 others above and the rest far below."""
    gen = torch.Generator().manual_seed(seed)
    l = torch.randn(1, E, generator=gen)
    want = 0.2 + 0.2 * torch.rand(E, generator=gen, dtype=torch.float64)
    want[E - topk + 1:] = 0.8 + 0.01 * torch.arange(topk - 1)
    for e, v in targets.items():
        want[e] = v
    bias = (want - ref.scores(l.double(), sigmoid)[0]).float()
    noise = torch.zeros(T, E)
    noise[:, list(targets)] = torch.randn(T, len(targets), generator=gen) * (1e-7 if sigmoid else 2e-8 * E)
    return l + noise, bias


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,G", [(64, 1), (256, 1), (256, 8), (1024, 1)])
@pytest.mark.parametrize("topk", [1, 5])
def test_a_better_expert_behind_the_first_not_chosen(qmm, sigmoid, E, G, topk):
    """The comparison's keys hold a score's upper bits alone.  Of one key's experts the lower index comes first: expert 20 stands before expert 40, whose score is the larger one and
    within 1e-8 of expert 50's, across the border of two keys at 0.75."""
    width = 2.0**-24 * 32 * max(1, E // 32)
    l, bias = bucketed(E, sigmoid, 300 if E == 1024 else 1500, topk, {50: 0.75 + 1e-8, 20: 0.75 - 0.6 * width, 40: 0.75 - 1e-8}, E + topk)
    check(qmm, l, topk, sigmoid, bias, G, min(G, 6), 2 if G > 1 else 1, True)
    check(qmm, l.flip(1).contiguous(), topk, sigmoid, bias.flip(0).contiguous(), G, G, 1, False)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E", [64, 256, 1024])
@pytest.mark.parametrize("topk", [1, 2, 5])
def test_equal_experts_before_a_better_one_of_the_same_key(qmm, sigmoid, E, topk):
    """Experts 20 and 30 are equal to the last bit; expert 40 is better by a third of a key's width."""
    width = 2.0**-24 * 32 * max(1, E // 32)
    l, bias = bucketed(E, sigmoid, 50, topk, {40: 0.75 + 0.6 * width, 20: 0.75 + 0.3 * width}, E + topk)
    l[:, 30], bias[30] = l[:, 20], bias[20]
    if not sigmoid:                                        # (expert 30's share of the denominator is no longer what the biases were made for: the scores of the three move alike)
        s = ref.scores(l[:1].double(), False)[0]
        bias[40] = (0.75 + 0.6 * width - s[40]).float()
        bias[[20, 30]] = (0.75 + 0.3 * width - s[20]).float()
    idx = check(qmm, l, topk, sigmoid, bias, 1, 1, 1, True)[1].cpu()
    assert (idx[:, topk - 1] == 40).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,topk,G", [(64, 6, 1), (256, 8, 8), (1024, 32, 1)])
def test_all_experts_equal_but_few(qmm, sigmoid, E, topk, G):
    l, bias = torch.zeros(40, E), torch.full((E,), 0.125)
    assert (check(qmm, l, topk, sigmoid, bias, G, G, 1, True)[1].cpu() == torch.arange(topk)).all()
    l[20:, E - 3] = 1e-6                                   # one score is better by a few roundings, one by none
    l[30:, E - 2] = 1e-9
    check(qmm, l, topk, sigmoid, bias, G, G, 1, True)


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("sigmoid,renorm", list(itertools.product((False, True), repeat=2)))
@pytest.mark.parametrize("T,E,topk,pitch", [(1, 1, 1, 1), (50, 128, 8, 128), (50, 128, 8, 131), (33, 46, 7, 48), (40, 1024, 32, 1024), (40, 1023, 32, 1023)])
def test_gradient_in_the_logits_place(qmm, dt, sigmoid, renorm, T, E, topk, pitch):
    l = torch.full((T, pitch), 9.0, dtype=ref.DTYPES[dt], device="cuda")[:, :E]
    l.copy_(logits_of(T, E, dt, "masked" if E > 1 else "plain", E))
    scores = qmm.SIGMOID if sigmoid else qmm.SOFTMAX
    idx, _ = qmm.expert_route(l, topk, scores, renormalize=renorm)
    dw = torch.randn(T, topk, generator=torch.Generator().manual_seed(2)).cuda()
    want = qmm.expert_route_grad(dw, l, idx, scores, renorm)
    got = qmm.expert_route_grad(dw, l, idx, scores, renorm, out=l)
    assert got is l and torch.equal(got, want)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("E", [12, 256])
def test_weights_of_chosen_scores_far_from_one_another(qmm, dt, E):
    """Biases choose experts whose scores lie many orders below one: the weights are ratios of the scores, ordinary numbers where the smaller scores are none."""
    sets = [(-44, -102, -60), (-75, -131, -110), (-1, -85, -70), (5, -86, -30), (-79, -81, -150), (-81, -85, -160), (-20, -87, -104), (0, -84, -80), (-10, -10, -95)]
    l, bias = torch.full((len(sets), E), 3.0), torch.full((E,), -3.0)
    bias[1:10:4] = torch.tensor([4.0, 3.0, 2.0])
    for t, s in enumerate(sets):
        l[t, 1:10:4] = torch.tensor(s, dtype=torch.float32) + (0.37 if dt == "f32" else 0.0)
    l = l.to(ref.DTYPES[dt])
    for scale in (1.5, -2.0):
        idx, w = qmm.expert_route(l.cuda(), 3, qmm.SIGMOID, bias.cuda(), renormalize=True, scale=scale)
        want_idx, want = ref.route(l, 3, True, bias, 1, 1, 1, True, scale)
        assert torch.equal(idx.cpu().long(), want_idx) and torch.equal(want_idx, torch.tensor([[1, 5, 9]] * len(sets)))
        # expf: 2 ulp, its argument's rounding of up to 2^-24 of 150, twice; half a dozen roundings; below fp32's normal numbers one of 2^-149, twice
        tol = (2 * 150 + 32) * 2.0**-24 * want.abs() + 2.0**-147
        assert bool(((w.cpu().double() - want).abs() <= tol).all())
        dw = torch.tensor([[1.0, -2.0, 0.5]]).expand(len(sets), 3).contiguous()
        got = qmm.expert_route_grad(dw.cuda(), l.cuda(), idx, qmm.SIGMOID, True, scale, out=torch.empty_like(l, device="cuda")).cpu().double()
        p, g = want.abs() / abs(scale), scale * dw.double()
        d = p * (p[:, None, :] * (g[:, :, None] - g[:, None, :])).sum(2) * torch.sigmoid(-l.double()[:, 1:10:4])
        size = p * (p[:, None, :] * (g[:, :, None] - g[:, None, :]).abs()).sum(2)
        assert bool(((got[:, 1:10:4] - d).abs() <= (4 * 150 + 64) * 2.0**-24 * size + ref.rounding(d, l.dtype) + 2.0**-146).all())


@pytest.mark.parametrize("dt", list(ref.DTYPES))
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,G,top,topk", [(21, 7, 6, 9), (64, 8, 5, 6), (256, 8, 4, 8), (96, 3, 2, 20)])
def test_groups_by_logits_whose_scores_are_all_alike(qmm, dt, sigmoid, E, G, top, topk):
    """Without a bias groups are valued by their largest logit: softmax scores beside one of 2000 are zero in 64 bits too, sigmoids of 45 are one.  Many equal logits, so that the
    choice's end lies among them."""
    gen = torch.Generator().manual_seed(E)
    l = (torch.randn(80, E, generator=gen) * 3).round()
    l[:, : E // 2] = torch.where(torch.rand(80, E // 2, generator=gen) < 0.7, 0.0, l[:, : E // 2])
    if sigmoid:
        l += 45
    else:
        l[torch.arange(80), torch.randint(0, E, (80,), generator=gen)] = 2000.0
    l = l.to(ref.DTYPES[dt])
    for renorm in (False, True):
        check(qmm, l, topk, sigmoid, None, G, top, 1, renorm)
