"""Rows that choose their experts: choice, weights, order and gradient against evaluations row by row in 64 bits.

Tolerances.  u = 2^-24.  The choice and the order are whole numbers and have to be equal.  A weight may be held in fp32 on its way: the
argument l - top of its exponential is off by |l - top| u, the exponential by 2 u, the sum of up to 1024 positive terms by 16 + 6
additions' u and what its terms are off by on their average (at most 8 u: terms that count have arguments of a few units), the division and the
factor by 2 u: (|l - top| + 40) u of the weight.  Gradients of logits are sums of two such products, held to twice that of the sum of
their magnitudes, and one rounding to the logits' type."""
import ctypes
import itertools
import math

import numpy as np
import pytest
import torch

from test_gpu_experts import BF16, F32, HALF, U, g, gen, strided, within  # noqa: F401 (g: the fixture)

pytestmark = pytest.mark.gpu
INF = math.inf


def reference(logits, k, score="softmax", bias=None, groups=1, groups_kept=1, group_best=1, renormalise=True, scale=1.0, n=None):
    """expert, weight, place, off by the definition, a row at a time (numpy, fp64); also each weight's |l - top|."""
    v = logits.detach().double().cpu().numpy()
    rows, experts = v.shape
    b = None if bias is None else bias.double().cpu().numpy()
    used = rows if n is None else min(rows, max(0, int(n)))
    expert, weight, far = np.full((rows, k), -1, np.int64), np.zeros((rows, k)), np.zeros((rows, k))
    per = experts // groups
    for r in range(used):
        l = v[r]
        if np.isnan(l).any() or (score == "softmax" and (l == INF).any()):
            weight[r] = np.nan
            continue
        top = l.max()
        if top == -INF:
            continue
        with np.errstate(over="ignore"):
            s = np.exp(l - top) / np.exp(l - top).sum() if score == "softmax" else 1 / (1 + np.exp(-l))
        ok = (l > -INF) & (True if b is None else (b > -INF))
        value = s if b is None else s + b
        order = l if b is None else value
        if groups > 1:
            worth = []
            for q in range(groups):
                inside = sorted((value[i] for i in range(q * per, (q + 1) * per) if ok[i]), reverse=True)[:group_best]
                worth.append(sum(inside) if inside else -INF)
            kept = [q for q in sorted(range(groups), key=lambda q: (-worth[q], q)) if worth[q] > -INF][:groups_kept]
            ok = ok & np.isin(np.arange(experts) // per, kept)
        chosen = sorted((i for i in range(experts) if ok[i]), key=lambda i: (-order[i], i))[:k]
        total = 1.0
        if renormalise and chosen:
            total = sum(s[i] for i in chosen)
            if total < 1e-290 or score == "softmax":   # the same quotient where the scores themselves vanish
                m = max(l[i] for i in chosen)
                s = np.where(np.isin(np.arange(experts), chosen), np.exp(np.minimum(l - m, 0)), 0)
                total = sum(s[i] for i in chosen)
        for j, i in enumerate(chosen):
            expert[r, j], weight[r, j], far[r, j] = i, scale * s[i] / total, min(abs(l[i] - top), 800.0) if score == "softmax" else min(abs(l[i]), 800.0)
    pairs = sorted((e, i) for i, e in enumerate(expert.ravel()) if e >= 0)
    place = np.full(rows * k, -1, np.int64)
    for at, (_, i) in enumerate(pairs):
        place[i] = at
    off = np.searchsorted([e for e, _ in pairs], np.arange(experts + 1)) if pairs else np.zeros(experts + 1, np.int64)
    put = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return put(expert), put(weight), put(place.reshape(rows, k)), put(off), put(far)


def check(r, want):
    expert, weight, place, off, far = want
    assert torch.equal(r.expert.long(), expert)
    within(r.weight, weight, (far + 40) * U * weight.nan_to_num().abs() + 2.0 ** -149)
    assert torch.equal(r.off.long(), off) and torch.equal(r.place.long(), place)


SIZES = [(1, 1, 1), (1, 64, 8), (3, 5, 5), (17, 72, 4), (130, 256, 8), (70, 257, 3), (40, 512, 16), (9, 1000, 32), (33, 1024, 32), (2, 65, 32),
         (200, 23, 2), (64, 128, 1)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows,experts,k", SIZES)
def test_choice_weights_and_order(g, rows, experts, k, score, dtype):
    r = gen(rows + experts)
    logits = (2 * torch.randn(rows, experts, device="cuda", generator=r)).to(dtype)
    bias = 0.3 * torch.randn(experts, device="cuda", generator=r)
    for b, renormalise, scale in ((None, True, 1.0), (bias, False, 2.5), (bias, True, 0.5), (None, False, 1.0)):
        want = reference(logits, k, score, b, renormalise=renormalise, scale=scale)
        check(g.gear_route(logits, k, score, bias=b, renormalise=renormalise, scale=scale), want)
        for x in (strided(logits, 3), strided(logits, 8), strided(torch.cat([logits[:, :1], logits], 1), 2)[:, 1:]):
            check(g.gear_route(x, k, score, bias=b, renormalise=renormalise, scale=scale), want)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,k", [(6, 3), (64, 8), (200, 5), (700, 9)])
def test_ties_go_to_the_lowest_expert(g, experts, k, score):
    r = gen(experts)
    logits = torch.randint(-1, 2, (40, experts), device="cuda", generator=r).float()
    logits[3], logits[4] = 0.0, -300.0
    steps = 0.25 * torch.randint(-1, 2, (experts,), device="cuda", generator=r).float()
    for bias in (None, torch.zeros(experts, device="cuda"), steps):
        check(g.gear_route(logits, k, score, bias=bias), reference(logits, k, score, bias))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,k", [(16, 4), (160, 8), (300, 6)])
def test_sums_that_fp32_cannot_tell_apart(g, experts, k, score):
    """Biases that undo the scores but for their own rounding: all experts' sums lie within 2^-24 of each other, in an order that only 64 bits show."""
    r = gen(experts)
    row = torch.randn(experts, device="cuda", generator=r)
    s = torch.softmax(row.double(), 0) if score == "softmax" else torch.sigmoid(row.double())
    bias = (0.75 - s).float()
    logits = row.repeat(50, 1)
    logits[1::2] += 0.001 * torch.randn(25, 1, device="cuda", generator=r)
    check(g.gear_route(logits, k, score, bias=bias), reference(logits, k, score, bias))


GROUPS = [(12, 3, 2, 1, 4), (12, 3, 2, 2, 4), (160, 8, 3, 2, 6), (256, 8, 4, 2, 8), (64, 64, 5, 2, 5), (512, 16, 1, 1, 20), (1024, 4, 3, 2, 32),
          (36, 12, 12, 2, 7), (100, 2, 1, 2, 1)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,kept,best,k", GROUPS)
def test_groups(g, experts, groups, kept, best, k, score, dtype):
    r = gen(experts + groups)
    logits = torch.randn(45, experts, device="cuda", generator=r).to(dtype)
    logits[7], logits[8, experts // groups:] = 0.0, -INF                 # a row of ties; one with a single group left
    logits[9, ::2], logits[10, 1:] = -INF, -INF
    bias = 0.2 * torch.randn(experts, device="cuda", generator=r)
    bias[: experts // groups] = -INF
    for b in (None, bias):
        kw = dict(bias=b, groups=groups, groups_kept=kept, group_best=best, renormalise=True, scale=2.5)
        check(g.gear_route(logits, k, score, **kw), reference(logits, k, score, **kw))
        check(g.gear_route(strided(logits, 5), k, score, **kw), reference(logits, k, score, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,k", [(5, 4), (64, 8), (300, 7), (1024, 3)])
def test_masks_infinities_and_nan(g, experts, k, score):
    r = gen(experts)
    logits = torch.randn(30, experts, device="cuda", generator=r)
    logits[0] = -INF                                         # no expert
    logits[1, 1:] = -INF                                     # one
    logits[2, 0] = math.nan                                  # broken
    logits[3, 1] = INF
    logits[4, :2] = INF
    logits[5] = torch.finfo(F32).min                         # a mask of the type's lowest value
    logits[6, 2:] = torch.finfo(F32).min
    logits[7] = 3e38
    logits[8] = -200.0 - torch.arange(experts, device="cuda") / 8     # sigmoids that vanish in fp32
    logits[9] = -1000.0 - torch.arange(experts, device="cuda")        # and in fp64
    logits[10] = math.nan
    bias = 0.1 * torch.randn(experts, device="cuda", generator=r)
    masked = bias.clone()
    masked[0], masked[3] = -INF, math.nan
    for b, renormalise in itertools.product((None, bias, masked, torch.full_like(bias, -INF)), (True, False)):
        check(g.gear_route(logits, k, score, bias=b, renormalise=renormalise), reference(logits, k, score, b, renormalise=renormalise))
    forced = bias.clone()
    forced[-2:] = INF
    check(g.gear_route(logits, k, score, bias=forced), reference(logits, k, score, forced))


@pytest.mark.parametrize("n", [-5, 0, 1, 33, 64, 99, 100, 5000])
def test_padding(g, n):
    """Rows behind the batch's end go nowhere, whatever they hold."""
    logits = torch.randn(100, 40, device="cuda", generator=gen(n + 9))
    logits[max(0, min(n, 100)):] = math.nan
    word = torch.tensor([n], dtype=torch.int32, device="cuda")
    want = reference(logits, 3, n=n)
    r = g.gear_route(logits, 3, n=word)
    check(r, want)
    d = g.gear_route_backward(logits, r, torch.ones(100, 3, device="cuda"), renormalise=False)
    assert torch.equal(d[max(0, min(n, 100)):], torch.zeros_like(d[max(0, min(n, 100)):])) and torch.isfinite(d).all()


@pytest.mark.parametrize("rows,groups", [(1, 1), (40, 1), (3000, 1), (40, 4), (3000, 4), (40_000, 1)])
def test_the_choice_alone(g, rows, groups):
    """From C, without an order of the pairs: no workspace is needed."""
    from paper_1806_03925_amd import binding as b
    logits = torch.randn(rows, 64, device="cuda", generator=gen(rows))
    want = g.gear_route(logits, 5, groups=groups, groups_kept=max(1, groups // 2))
    expert, weight = torch.empty_like(want.expert), torch.empty_like(want.weight)
    a = b.gear_route_args(rows, 64, 5, b.GEAR_F32, b.GEAR_SCORE_SOFTMAX, groups, max(1, groups // 2), 1, 1, 1.0, logits.data_ptr(), 64, None, None,
                          expert.data_ptr(), weight.data_ptr(), None, None)
    assert b.lib.gear_route(ctypes.byref(a), None, 0, torch.cuda.current_stream().cuda_stream) == b.GEAR_OK
    assert torch.equal(expert, want.expert) and torch.equal(weight, want.weight)


@pytest.mark.parametrize("experts,k,dtype", [(24, 8, F32), (24, 3, BF16), (64, 8, F32), (63, 8, F32), (200, 8, F32), (256, 5, BF16), (130, 1, F32), (256, 8, F32)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_many_rows(g, experts, k, dtype, score):
    """Long batches have kernels of their own: the same rows as in short ones, and some of them by the definition."""
    rows = 33_001
    r = gen(experts)
    logits = (1.5 * torch.randn(rows, experts, device="cuda", generator=r)).to(dtype)
    logits[5::7, experts // 3:] = -INF
    logits[6::11] = 0.25
    logits[12::13] = -INF
    logits[100, 3], logits[200, 0] = math.nan, INF
    bias = (0.2 / experts) * torch.randn(experts, device="cuda", generator=r)
    for b in (None, bias):
        for x in (logits, strided(logits, 1)):
            long = g.gear_route(x, k, score, bias=b, renormalise=False, scale=2.5)
            for first in (0, 1000, 20_000, rows - 700):
                short = g.gear_route(x[first:first + 700], k, score, bias=b, renormalise=False, scale=2.5)
                assert torch.equal(long.expert[first:first + 700], short.expert)
                within(long.weight[first:first + 700], short.weight, 80 * U * short.weight.nan_to_num().abs())   # (d + 40) u of each; chosen logits are within 20 of the top here, masked rows too
        part = slice(90, 210)
        expert, weight, _, _, far = reference(logits[part], k, score, b, renormalise=False, scale=2.5)
        assert torch.equal(long.expert[part].long(), expert)
        within(long.weight[part], weight, (far + 40) * U * weight.nan_to_num().abs() + 2.0 ** -149)


def test_no_rows(g):
    r = g.gear_route(torch.empty(0, 24, device="cuda"), 3)
    assert r.expert.shape == (0, 3) and torch.equal(r.off, torch.zeros(25, dtype=torch.int32, device="cuda"))
    assert g.gear_route_backward(torch.empty(0, 24, device="cuda"), r, torch.empty(0, 3, device="cuda")).shape == (0, 24)


@pytest.mark.parametrize("rows,experts,k", [(1025, 7, 3), (5000, 1024, 4), (20_001, 40, 3), (70_000, 256, 1), (300_000, 3, 2), (16_385, 300, 8), (65_536, 64, 2), (17_000_000, 3, 1)])
def test_order_of_many_runs(g, rows, experts, k):
    """The order from the choice, by torch's stable sort."""
    r = gen(rows)
    logits = torch.randn(rows, experts, device="cuda", generator=r)
    logits[::5, : experts // 2 + 1] = -INF
    n = torch.tensor([rows - rows // 9], dtype=torch.int32, device="cuda")
    route = g.gear_route(logits, k, n=n)
    order = torch.sort(torch.where(torch.arange(rows, device="cuda")[:, None] < n, logits, -INF), dim=1, descending=True, stable=True)
    expert = torch.where(order.values[:, :k] > -INF, order.indices[:, :k], -1)
    assert torch.equal(route.expert.long(), expert)
    line, at = torch.sort(torch.where(expert >= 0, expert, experts).flatten(), stable=True)
    place = torch.empty_like(at).scatter_(0, at, torch.arange(at.numel(), device="cuda")).view(rows, k)
    assert torch.equal(route.place.long(), torch.where(expert >= 0, place, -1))
    assert torch.equal(route.off.long(), torch.searchsorted(line, torch.arange(experts + 1, device="cuda")))


def test_rows_far_apart(g):
    """Rows whose distance takes the last ones past 2^31 elements."""
    apart = (1 << 20) - 1
    rows = 2100
    wide = torch.empty(rows * apart, dtype=BF16, device="cuda")
    logits = wide.as_strided((rows, 9), (apart, 1))
    logits.copy_(torch.randn(rows, 9, device="cuda", generator=gen(1)))
    got = g.gear_route(logits, 2)
    want = g.gear_route(logits.contiguous(), 2)
    assert torch.equal(got.expert, want.expert) and torch.equal(got.weight, want.weight) and torch.equal(got.place, want.place)
    dw = torch.randn(rows, 2, device="cuda", generator=gen(2))
    assert torch.equal(g.gear_route_backward(logits, got, dw), g.gear_route_backward(logits.contiguous(), got, dw))


# ---- gradient -------------------------------------------------------------------------------------------------------
def weights64(v, expert, score, renormalise, scale):
    """The weights as a function of the logits (64 bits), the choice held fixed."""
    s = torch.sigmoid(v) if score == "sigmoid" else torch.softmax(v, 1)
    w = torch.where(expert >= 0, s.gather(1, expert.clamp(min=0).long()), 0.0)
    if renormalise:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    return scale * w


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows,experts,k", SIZES)
def test_gradient(g, rows, experts, k, score, renormalise, dtype):
    r = gen(rows * 3 + experts)
    scale = 2.5
    logits = (2 * torch.randn(rows, experts, device="cuda", generator=r)).to(dtype)
    if rows > 2 and experts > 2:
        logits[1, 1:] = -INF                              # fewer experts than slots
        logits[2] = -INF
    dw = torch.randn(rows, k, device="cuda", generator=r)
    route = g.gear_route(logits, k, score, renormalise=renormalise, scale=scale)
    dw_there = torch.where(route.expert >= 0, dw, math.nan)   # what flows into an empty slot is nothing, whatever it is
    v = logits.double().nan_to_num(neginf=-1e4).requires_grad_()   # exp(-1e4) is 0
    w = weights64(v, route.expert, score, renormalise, scale)
    want = torch.autograd.grad(w, v, dw.double())[0]
    want = torch.where((route.expert >= 0).any(1, keepdim=True), want, 0.0)
    # magnitudes that cancel: of chosen experts, and (softmax over all) of the scores
    flow = (scale * dw.abs().double() * (route.expert >= 0))
    w64 = (w / scale).detach()
    inner = (w64 * flow).sum(1, keepdim=True)
    size = torch.zeros_like(want).scatter_add_(1, route.expert.clamp(min=0).long(), w64 * flow)
    size += torch.zeros_like(want).scatter_add_(1, route.expert.clamp(min=0).long(), w64 * inner * (route.expert >= 0))
    if score == "softmax" and not renormalise:
        size += torch.softmax(v, 1).detach() * inner
    far = torch.where(torch.isfinite(logits), (logits.double() - (logits.double().amax(1, keepdim=True) if score == "softmax" else 0)).abs(), 0.0)
    # the reference is not exact either: where a gradient is zero because two sums are equal (softmax, divided: every logit that was not chosen), 64 bits
    # leave up to 2^-53 of each of their up to 1024 terms, 2^-43 of the row's magnitudes
    bound = 2 * (far + 40) * U * size + HALF[dtype] * want.abs() + 2.0 ** -43 * inner + 1e-37
    for x, out in ((logits, None), (strided(logits, 3), strided(torch.zeros_like(logits), 5))):
        got = g.gear_route_backward(x, route, dw_there, score, renormalise, scale, out=out)
        within(got, want, bound)
        assert out is None or got is out


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient_against_differences(g, score, renormalise):
    """Central differences of the forward pass itself in 64 bits: off by h^2 / 6 of the third derivative (below 1, h = 1e-4: 2e-9) and 2^-52 / h."""
    r = gen(5)
    logits, dw = torch.randn(6, 9, device="cuda", generator=r), torch.randn(6, 3, device="cuda", generator=r)
    route = g.gear_route(logits, 3, score, renormalise=renormalise, scale=1.5)
    got = g.gear_route_backward(logits, route, dw, score, renormalise, 1.5)
    h, want = 1e-4, torch.zeros(6, 9, dtype=torch.float64, device="cuda")
    for i in range(9):
        step = torch.zeros(6, 9, dtype=torch.float64, device="cuda")
        step[:, i] = h
        up, down = (weights64(logits.double() + d, route.expert, score, renormalise, 1.5) for d in (step, -step))
        want[:, i] = ((up - down) * dw).sum(1) / (2 * h)
    within(got, want, 1e-8 + 2 * 48 * U * 1.5 * 2 * dw.abs().sum(1, keepdim=True))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient_of_an_only_expert(g, score):
    """Divided by itself a weight is `scale` whatever its logit is: exactly zero, from one slot or from several of which one was filled."""
    r = gen(8)
    logits, dw = 4 * torch.randn(700, 24, device="cuda", generator=r), 100 * torch.randn(700, 20, device="cuda", generator=r)
    for x, k in ((logits, 1), (torch.where(torch.arange(24, device="cuda") == 7, logits, -INF), 3), (torch.where(torch.arange(24, device="cuda") == 7, logits, -INF), 20)):
        route = g.gear_route(x, k, score, scale=1.7)
        assert int((route.expert >= 0).sum()) == 700
        assert (g.gear_route_backward(x, route, dw[:, :k].contiguous(), score, True, 1.7) == 0).all()


def test_gradient_of_broken_rows(g):
    logits = torch.randn(5, 20, device="cuda", generator=gen(6))
    logits[1, 3], logits[3, 0] = math.nan, INF
    for score, renormalise in itertools.product(("softmax", "sigmoid"), (True, False)):
        route = g.gear_route(logits, 4, score, renormalise=renormalise)
        d = g.gear_route_backward(logits, route, torch.ones(5, 4, device="cuda"), score, renormalise)
        bad = [1, 3] if score == "softmax" else [1]
        assert d[bad].isnan().all() and torch.isfinite(d[[r for r in range(5) if r not in bad]]).all()


# ---- refusals, streams, graphs --------------------------------------------------------------------------------------
def test_refusals(g):
    x = torch.randn(4, 12, device="cuda")
    r = g.gear_route(x, 2)
    for call in (lambda: g.gear_route(x.cpu(), 2), lambda: g.gear_route(x.double(), 2), lambda: g.gear_route(x[0], 2), lambda: g.gear_route(x.t(), 2),
                 lambda: g.gear_route(x, 0), lambda: g.gear_route(x, 13), lambda: g.gear_route(x, 2, "tanh"), lambda: g.gear_route(x, 2, groups=5),
                 lambda: g.gear_route(x, 5, groups=3, groups_kept=1), lambda: g.gear_route(x, 2, group_best=3), lambda: g.gear_route(x, 2, scale=0.0),
                 lambda: g.gear_route(x, 2, bias=torch.zeros(11, device="cuda")), lambda: g.gear_route(x, 2, bias=torch.zeros(12, device="cuda").to(BF16)),
                 lambda: g.gear_route(x, 2, n=torch.zeros(1, device="cuda")), lambda: g.gear_route(x, 2, n=torch.zeros(1, dtype=torch.int32)),
                 lambda: g.gear_route_backward(x[:3], r, torch.ones(3, 2, device="cuda")), lambda: g.gear_route_backward(x, r, torch.ones(4, 3, device="cuda")),
                 lambda: g.gear_route_backward(x, r, torch.ones(4, 2, device="cuda").to(BF16)), lambda: g.gear_route_backward(x, r, torch.ones(4, 2, device="cuda"), out=x),
                 lambda: g.gear_route_backward(x, r, torch.ones(4, 2, device="cuda"), "none"), lambda: g.Route(r.expert, r.weight, r.place[:3], r.off),
                 lambda: g.Route(r.expert, r.weight.double(), r.place, r.off), lambda: g.Route(r.expert.long(), r.weight, r.place, r.off),
                 lambda: g.Route(r.expert, r.weight, r.place, r.off[:1]), lambda: g.Route(r.expert[0], r.weight[0], r.place[0], r.off)):
        with pytest.raises(g.GearError):
            call()


def test_captured_and_replayed_beside_eager_calls(g):
    rows, experts, k = 3000, 96, 4
    r = gen(3)
    logits, dw = torch.randn(rows, experts, device="cuda", generator=r), torch.randn(rows, k, device="cuda", generator=r)
    n = torch.tensor([rows], dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g.gear_route_backward(logits, g.gear_route(logits, k, n=n), dw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        route = g.gear_route(logits, k, n=n)
        d = g.gear_route_backward(logits, route, dw, renormalise=True)
    for i in range(4):
        logits.copy_(torch.randn(rows, experts, device="cuda", generator=r))
        n.fill_(rows - 500 * i)
        graph.replay()
        eager = g.gear_route(logits, k, n=n)
        d_eager = g.gear_route_backward(logits, eager, dw)
        torch.cuda.synchronize()
        for a, b in ((route.expert, eager.expert), (route.weight, eager.weight), (route.place, eager.place), (route.off, eager.off), (d, d_eager)):
            assert torch.equal(a, b)


def test_two_streams_at_once(g):
    x = [torch.randn(8000, 128, device="cuda", generator=gen(i)) for i in range(2)]
    want = [g.gear_route(t, 6, "sigmoid") for t in x]
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(g.gear_route(x[i], 6, "sigmoid"))
    torch.cuda.synchronize()
    for w, rs in zip(want, got):
        for r in rs:
            assert torch.equal(r.expert, w.expert) and torch.equal(r.place, w.place) and torch.equal(r.off, w.off) and torch.equal(r.weight, w.weight)


def reference_many(logits, k, score="softmax", bias=None, groups=1, groups_kept=1, group_best=1, renormalise=True, scale=1.0, n=None):
    """What reference() gives, for long batches without NaN or +inf: sorts of whole columns in 64 bits."""
    v = logits.double()
    rows, experts = v.shape
    there = torch.ones(rows, 1, dtype=torch.bool, device="cuda") if n is None else torch.arange(rows, device="cuda")[:, None] < n
    top = torch.where(v.amax(1, keepdim=True) > -INF, v.amax(1, keepdim=True), 0.0)
    s = torch.exp(v - top) if score == "softmax" else 1 / (1 + torch.exp(-v))
    if score == "softmax":
        s = s / s.sum(1, keepdim=True).clamp(min=1.0)
    ok = (v > -INF) & there if bias is None else (v > -INF) & (bias > -INF) & there
    value = torch.where(ok, s if bias is None else s + bias.double(), -INF)
    order = torch.where(ok, v, -INF) if bias is None else value
    if groups > 1:
        best = torch.sort(value.view(rows, groups, -1), dim=2, descending=True).values[:, :, :group_best]
        worth = torch.where((best > -INF).any(2), torch.where(best > -INF, best, 0.0).sum(2), -INF)
        keep = torch.zeros(rows, groups, dtype=torch.bool, device="cuda")
        keep.scatter_(1, torch.sort(worth, dim=1, descending=True, stable=True).indices[:, :groups_kept], True)
        order = torch.where(keep.repeat_interleave(experts // groups, 1), order, -INF)
    by = torch.sort(order, dim=1, descending=True, stable=True)
    expert = torch.where(by.values[:, :k] > -INF, by.indices[:, :k], -1)
    at = expert.clamp(min=0)
    chosen = torch.where(expert >= 0, v.gather(1, at), -INF)
    weight = torch.where(expert >= 0, s.gather(1, at), 0.0)
    if renormalise:
        if score == "softmax":
            high = chosen.amax(1, keepdim=True)
            weight = torch.where(expert >= 0, torch.exp(chosen - torch.where(high > -INF, high, 0.0)), 0.0)
        total = weight.sum(1, keepdim=True)
        weight = weight / torch.where(total > 0, total, 1.0)
    far = torch.where(expert >= 0, (chosen - (top if score == "softmax" else 0.0)).abs(), 0.0)
    line, pair = torch.sort(torch.where(expert >= 0, expert, experts).flatten(), stable=True)
    place = torch.empty_like(pair).scatter_(0, pair, torch.arange(pair.numel(), device="cuda")).view(rows, k)
    off = torch.searchsorted(line, torch.arange(experts + 1, device="cuda"))
    return expert, scale * weight, torch.where(expert >= 0, place, -1), off, far


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows,experts,k,groups", [(40, 64, 8, 1), (40, 300, 5, 1), (40, 1000, 12, 1), (33_001, 64, 8, 1), (33_001, 256, 8, 1), (200, 160, 6, 8)])
def test_logits_next_to_nothing(g, rows, experts, k, groups, score):
    """bf16 logits down to the smallest denormal, one step of their type from each other: without a bias it is they that are compared, however close."""
    r = gen(experts)
    step = torch.arange(experts, device="cuda", dtype=torch.int16)
    for low, high in ((0, 128), (0, 700), (128, 300), (0x300, 0x380), (0x600, 0x700), (0xb00, 0xc80), (0xd00, 0xe80)):
        bits = torch.randint(low, high, (rows, experts), device="cuda", generator=r).to(torch.int16)
        bits[::3] = (low + step % (high - low)).to(torch.int16)
        bits[1::3] |= (torch.randint(0, 2, bits[1::3].shape, device="cuda", generator=r) * -32768).to(torch.int16)
        for logits in (bits.view(BF16), bits.view(BF16).float()):
            kw = dict(groups=groups, groups_kept=max(1, groups // 2), group_best=1)
            check(g.gear_route(logits, k, score, **kw), reference_many(logits, k, score, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups", [(64, 8), (512, 16), (1024, 32)])
@pytest.mark.parametrize("large", [64.0, 1e3, 2.0 ** 20])
def test_groups_whose_largest_two_cancel(g, experts, groups, large, score):
    """Two experts of each group are left, their biases large and opposite: what their sums in fp32 lose is a part of the biases, not of the sums."""
    r = gen(experts)
    per = experts // groups
    logits = 2 * torch.randn(3000, experts, device="cuda", generator=r)
    bias = torch.full((groups, per), -INF, device="cuda")
    each = large * (1 + torch.arange(groups, device="cuda") / groups)       # apart, so that the choice within the groups kept is clear
    bias[:, 1], bias[:, per - 1] = each, -each
    kw = dict(bias=bias.flatten(), groups=groups, groups_kept=groups // 4, group_best=2)
    check(g.gear_route(logits, 4, score, **kw), reference_many(logits, 4, score, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,kept,k", [(12, 3, 2, 6), (160, 8, 5, 16), (1024, 32, 12, 32)])
def test_groups_parked_by_the_lowest_bias(g, experts, groups, kept, k, score):
    """The type's lowest value for all of a group's experts: two of them are beyond fp32, but the group is still there to be chosen after the others."""
    r = gen(experts)
    logits = 2 * torch.randn(400, experts, device="cuda", generator=r)
    logits[5::9, experts // 2:] = -INF
    for value in (torch.finfo(F32).min, -2e38):
        bias = 0.1 * torch.randn(groups, experts // groups, device="cuda", generator=r)
        bias[::2] = value
        bias[0, 1:] = 0.0 if groups > 3 else value
        for best in (1, 2):
            kw = dict(bias=bias.flatten(), groups=groups, groups_kept=kept, group_best=best)
            check(g.gear_route(logits, k, score, **kw), reference_many(logits, k, score, **kw))
            check(g.gear_route(logits[:9], k, score, **kw), reference(logits[:9], k, score, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,k,groups", [(64, 8, 1), (256, 8, 1), (160, 6, 8), (700, 12, 1)])
def test_experts_parked_by_large_biases(g, experts, k, groups, score):
    """A bias far beyond all scores, as a finite mask, changes nothing for the others: neither their order, also where fp32 cannot tell their sums apart, nor their weights."""
    r = gen(experts)
    logits = 1.5 * torch.randn(4000, experts, device="cuda", generator=r)
    row = torch.randn(experts, device="cuda", generator=r)
    s = torch.softmax(row.double(), 0) if score == "softmax" else torch.sigmoid(row.double())
    for close, park in itertools.product((False, True), (-1e4, -100.0, 1e4, -3e38)):
        bias = (0.75 - s).float() if close else 0.1 / experts * torch.randn(experts, device="cuda", generator=r)
        logits[::50] = row
        bias[experts // 2] = park
        if park < 0:
            bias[experts // 2 + 1] = park
        kw = dict(bias=bias, groups=groups, groups_kept=max(1, groups // 2), group_best=min(2, groups))
        check(g.gear_route(logits, k, score, **kw), reference_many(logits, k, score, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows", [1, 3, 16])
@pytest.mark.parametrize("experts,groups,kept,best,k", GROUPS)
def test_groups_in_one_workgroup(g, experts, groups, kept, best, k, rows, score):
    """Choice and order in one launch, which takes the most LDS of all."""
    r = gen(experts + rows)
    logits = torch.randn(rows, experts, device="cuda", generator=r)
    logits[rows // 2, ::3] = -INF
    bias = 0.2 * torch.randn(experts, device="cuda", generator=r)
    for b in (None, bias):
        for x in (logits, logits.to(BF16), strided(logits, 3)):
            kw = dict(bias=b, groups=groups, groups_kept=kept, group_best=best)
            check(g.gear_route(x, k, score, **kw), reference(x, k, score, **kw))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("rows,experts,groups,kept,best,k", [(10_001, 160, 8, 3, 2, 6), (9_000, 12, 3, 2, 2, 4), (33_001, 64, 16, 4, 1, 8), (5_000, 512, 16, 4, 2, 20), (3_000, 1024, 4, 3, 2, 32)])
def test_groups_of_long_batches(g, rows, experts, groups, kept, best, k, score, dtype):
    """Workgroups that take several passes over rows, the next one's logits on their way while LDS holds this one's."""
    r = gen(rows)
    logits = (1.5 * torch.randn(rows, experts, device="cuda", generator=r)).to(dtype)
    logits[5::11, experts // 3:] = -INF
    logits[6::97] = 0.25
    logits[12::101] = -INF
    bias = 0.05 * torch.randn(experts, device="cuda", generator=r)
    bias[1::7] = -INF
    n = torch.tensor([rows - rows // 20], dtype=torch.int32, device="cuda")
    for b in (None, bias):
        kw = dict(bias=b, groups=groups, groups_kept=kept, group_best=best, scale=2.5, n=n)
        check(g.gear_route(logits, k, score, **kw), reference_many(logits, k, score, **kw))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,k,dtype", [(24, 3, BF16), (64, 8, F32), (63, 8, BF16), (160, 8, F32), (256, 8, BF16), (256, 16, F32), (300, 4, F32), (1024, 8, BF16)])
def test_divided_weights_of_long_batches(g, experts, k, dtype, score):
    rows = 33_001
    r = gen(experts)
    logits = (1.5 * torch.randn(rows, experts, device="cuda", generator=r)).to(dtype)
    logits[5::7, experts // 3:] = -INF
    logits[12::13] = -INF
    bias = (0.2 / experts) * torch.randn(experts, device="cuda", generator=r)
    for b in (None, bias):
        check(g.gear_route(logits, k, score, bias=b, scale=2.5), reference_many(logits, k, score, b, scale=2.5))


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("scale", [3.3e38, 1e-30])
def test_scales_at_the_ends_of_fp32(g, scale, score, renormalise):
    """Nothing on the way to a weight or to its gradient is larger than these are themselves."""
    r = gen(21)
    scale = float(np.float32(scale))
    logits, dw = torch.randn(300, 40, device="cuda", generator=r) - 1, torch.rand(300, 6, device="cuda", generator=r) * 2 - 1
    route = g.gear_route(logits, 6, score, renormalise=renormalise, scale=scale)
    check(route, reference(logits, 6, score, renormalise=renormalise, scale=scale))
    v = logits.double().requires_grad_()
    w = weights64(v, route.expert, score, renormalise, scale)
    want = torch.autograd.grad(w, v, dw.double())[0]
    # as in test_gradient: twice what the two products' factors are off by, of the sum of their magnitudes; 24 bits of a scale's and a weight's quotient are among the 40
    p = w.detach() / scale
    inner = (p * dw.abs().double()).sum(1, keepdim=True)
    size = torch.zeros_like(want).scatter_add_(1, route.expert.long(), p * (dw.abs().double() + inner))
    if score == "softmax" and not renormalise:
        size += torch.softmax(v, 1).detach() * inner
    far = (logits.double() - (logits.double().amax(1, keepdim=True) if score == "softmax" else 0)).abs()
    within(g.gear_route_backward(logits, route, dw, score, renormalise, scale), want, scale * (2 * (far + 40) * U * size + 2.0 ** -43 * inner))
