"""The operators of a Dense Part whose rows choose their experts, as a program calls them: the routing of rows by their
scores and its gradient, the rows' way to their experts and back and its gradients, and products in 8-bit integers with a
scale for every row and every output.

Five kinds of case: "route" (choice, weights and order of the experts), "route_back" (the scores' gradient), "rows" (a
training step's four passes over rows: copied to their experts, weighted sums on their way back, and the gradients of both),
"product_i8" (rows to 8-bit integers, product) and "serve" (routing, rows to their experts in 8-bit integers, their products,
weighted sums).  Widths are those of `gear_inputs/configs.py` and of the tests (1152, 1024, 576, 72, ...) or powers of two.

The definitions.  Scores of a row: softmax or sigmoid of its logits.  An expert is eligible where neither its logit nor its
bias is -inf.  Experts are ordered by score + bias (without a bias: by logit), ties by the lowest index; where experts come
in groups, a group's value is the sum of its `best` best (of as many as are eligible), and only experts of the groups_kept
best groups can be chosen (ties by the lowest index).  The k best are chosen; a place that no expert is left for holds -1 and
weighs 0, as do all of a row behind the batch's `used` rows.  Weights are the chosen experts' scores, divided by their sum if
`renormalise`, times scale.  Chosen pairs (row, slot) are lined up by expert, row and slot: `place`, and `off`, where each expert begins.
8 bits: q = the integer nearest to 127 v / max|v| (ties to even), the scale max|v| / 127, over a row or over an output's weights.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one image that has just arrived chooses its experts: latency
        dict(name="route_one_row", kind="route", rows=1, used=1, experts=64, k=8, score="softmax", bias=False, groups=1, kept=1, best=1,
             renormalise=True, scale=1.0, masked=False, dtype="f32"),
        # a padded batch: experts in groups, some switched off, a bias that balances them
        dict(name="route_groups", kind="route", rows=10_001, used=9_500, experts=160, k=6, score="sigmoid", bias=True, groups=8, kept=3, best=2,
             renormalise=True, scale=2.5, masked=True, dtype="bf16"),
        # a production batch over many experts
        dict(name="route_large", kind="route", rows=65_536, used=65_536, experts=256, k=8, score="softmax", bias=True, groups=1, kept=1, best=1,
             renormalise=False, scale=1.0, masked=False, dtype="f32"),
        # an ordinary training batch's way back through the routing
        dict(name="route_back", kind="route_back", rows=4_097, used=4_097, experts=72, k=4, score="sigmoid", renormalise=True, scale=2.5, dtype="bf16"),
        # the same for a production batch, every expert's score touched by the softmax
        dict(name="route_back_large", kind="route_back", rows=65_536, used=65_536, experts=256, k=8, score="softmax", renormalise=False, scale=1.0,
             dtype="f32"),
        # a first trial of a model in full precision: few narrow rows, some of them padding
        dict(name="rows_small", kind="rows", rows=1_000, used=960, dim=72, experts=5, k=3, dtype="f32"),
        # an ordinary training batch
        dict(name="rows", kind="rows", rows=16_384, used=16_384, dim=1152, experts=8, k=2, dtype="bf16"),
        # production: wide rows, many experts
        dict(name="rows_large", kind="rows", rows=65_536, used=65_536, dim=2048, experts=64, k=4, dtype="bf16"),
        # one row through a layer in 8-bit integers: latency
        dict(name="i8_one_row", kind="product_i8", rows=1, dim=1152, out=1024, experts=0, dtype="bf16"),
        # the whole cache refreshed: the largest product in 8-bit integers
        dict(name="i8_large", kind="product_i8", rows=65_536, dim=4096, out=4096, experts=0, dtype="bf16"),
        # a handful of images served: every launch counts
        dict(name="serve_small", kind="serve", rows=33, used=33, dim=576, out=520, experts=16, k=4, dtype="bf16"),
        # a part of the cache refreshed by routed experts
        dict(name="serve", kind="serve", rows=16_384, used=16_000, dim=1152, out=1024, experts=64, k=4, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = 8 * _log_int(rng, lo // 8, hi // 8)
    return n // 128 * 128 if n >= 256 and rng.random() < 0.3 else n      # whole tiles, as configured models mostly have


def draw(rng):
    """One more case: sizes spread over the range between the smallest and the largest listed one."""
    kind = rng.choice(["route", "route", "route_back", "rows", "rows", "product_i8", "serve"])
    rows = _log_int(rng, 1, 65_536)
    used = rows if rng.random() < 0.6 else rng.randint(0, rows)
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("route", "route_back"):
        experts = _log_int(rng, 2, 512)
        while rows * experts > 65_536 * 256:
            rows //= 2
        used = min(used, rows)
        case = dict(kind=kind, rows=rows, used=used, experts=experts, k=min(experts, _log_int(rng, 1, 16)), score=rng.choice(["softmax", "sigmoid"]),
                    renormalise=rng.random() < 0.6, scale=rng.choice([1.0, 1.0, 2.5, 0.5]), dtype=dtype)
        if kind == "route_back":
            return case
        fits = [g for g in (2, 3, 4, 5, 6, 7, 8, 12, 16) if experts % g == 0 and experts // g >= 2]
        groups = rng.choice(fits) if fits and rng.random() < 0.4 else 1
        kept = rng.randint(1, groups)
        case["k"] = min(case["k"], experts // groups * kept)
        return dict(case, bias=rng.random() < 0.6, groups=groups, kept=kept, best=rng.choice([1, 2]) if groups > 1 else 1, masked=rng.random() < 0.3)
    dim = _width(rng, 64, 8192)
    if kind == "rows":
        experts = _log_int(rng, 2, 64)
        k = min(experts, _log_int(rng, 1, 8))
        while rows * (k + 1) * dim * SIZE[dtype] > 65_536 * 5 * 2048 * 2:
            rows //= 2
        return dict(kind=kind, rows=rows, used=min(used, rows), dim=dim, experts=experts, k=k, dtype=dtype)
    out = _width(rng, 64, 8192)
    if kind == "product_i8":
        experts = rng.choice([0, 0, _log_int(rng, 2, 64)])
        while 2.0 * rows * dim * out > 2e12:
            rows //= 2
        while max(1, experts) * dim * out > 64 * 2048 * 1024:
            experts //= 2
        return dict(kind=kind, rows=max(1, rows), dim=dim, out=out, experts=experts, dtype=dtype)
    experts = _log_int(rng, 2, 64)
    while experts > 2 and experts * dim * out > 64 * 2048 * 1024:
        experts //= 2
    k = min(experts, _log_int(rng, 1, 8))
    while rows > 1 and (2.0 * rows * k * dim * out > 5e11 or rows * k * (dim + out) > 65_536 * 5 * 2048):
        rows //= 2
    return dict(kind=kind, rows=rows, used=min(used, rows), dim=dim, out=out, experts=experts, k=k, dtype="bf16")


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _features(rows, dim, dtype, gen, scale=1.0):
    """Rows of features: every row a size of its own, every 50th column large, every 97th row empty (a missing image)."""
    x = torch.randn(rows, dim, device="cuda", generator=gen)
    x *= scale * torch.exp(torch.randn(rows, 1, device="cuda", generator=gen))
    x[:, ::50] *= 8.0
    x[96::97] = 0.0
    return x.to(dtype)


def _logits(rows, experts, dtype, gen):
    """Scores before their squashing: popular experts and rare ones, every 97th row undecided (the missing image's)."""
    v = 1.5 * torch.randn(rows, experts, device="cuda", generator=gen) + 0.7 * torch.randn(experts, device="cuda", generator=gen)
    v[96::97] = 0.0
    return v.to(dtype)


def _sizes(rows, experts, seed):
    """Rows of each expert: popular ones and rare ones, some without a row."""
    rng = random.Random(seed)
    if experts == 0:
        return [rows]
    weights = [0.0 if experts > 2 and rng.random() < 0.1 else 1.0 / (1 + i) ** 0.7 for i in range(experts)]
    if not any(weights):
        weights[0] = 1.0
    rng.shuffle(weights)
    total, left, sizes = sum(weights), rows, []
    for w in weights:
        n = min(left, int(rows * w / total + rng.random()))
        sizes.append(n)
        left -= n
    sizes[max(range(experts), key=weights.__getitem__)] += left
    return sizes


class _State:
    pass


def _inputs(case, seed):
    """The data of a case, made from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.kind = kind = case["kind"]
    s.case = case
    rows, dtype = case["rows"], DTYPE[case["dtype"]]
    if kind != "product_i8":
        experts, k = case["experts"], case["k"]
        s.logits = _logits(rows, experts, torch.float32 if kind in ("rows", "serve") else dtype, gen)
        s.bias, s.n = None, None
        if case.get("bias"):
            s.bias = (0.05 if case["score"] == "sigmoid" else 0.5 / experts) * torch.randn(experts, device="cuda", generator=gen)
        if case.get("masked"):       # some experts switched off, and in some rows all but a few not allowed
            if s.bias is not None:
                s.bias[1::7] = -math.inf
            s.logits[5::11, experts // 8:] = -math.inf
        if case["used"] < rows:
            s.n = torch.tensor([case["used"]], dtype=torch.int32, device="cuda")
    if kind == "route_back":
        s.dweight = 1e-3 * torch.randn(rows, k, device="cuda", generator=gen)
    if kind == "rows":
        dim = case["dim"]
        s.x = _features(rows, dim, dtype, gen)
        s.y = _features(rows * k, dim, dtype, gen)
        s.dout = _features(rows, dim, dtype, gen, 1e-3)
        s.dxs = _features(rows * k, dim, dtype, gen, 1e-3)
    if kind in ("product_i8", "serve"):
        dim, out = case["dim"], case["out"]
        s.x = _features(rows, dim, dtype, gen)
        s.w = (torch.randn(max(1, case["experts"]), out, dim, device="cuda", generator=gen) * dim ** -0.5).to(dtype)
        s.w *= torch.exp(0.5 * torch.randn(out, 1, device="cuda", generator=gen)).to(dtype)
    if kind == "product_i8":
        s.sizes = _sizes(rows, case["experts"], seed)
        ends = torch.tensor([0] + s.sizes).cumsum(0)
        s.bounds = ends.tolist()
        s.off = ends.to(torch.int32).cuda() if case["experts"] else None
    if kind == "serve":
        s.residual = _features(rows, out, dtype, gen)
    return s


ROUTING = dict(score="softmax", groups=1, kept=1, best=1, renormalise=True, scale=1.0)     # of the kinds whose cases do not say


def _options(case):
    return {name: case.get(name, usual) for name, usual in ROUTING.items()}


def prepare(case, seed):
    """What a program has before the call: its inputs; the weights in 8 bits, laid out once; in a training step's passes over
    rows and in the routing's gradient, the routing of the forward pass."""
    s = _inputs(case, seed)
    if s.kind in ("rows", "route_back"):
        s.expert, s.weight, s.place, s.off = _route(s.logits, case["k"], s.bias, s.n, **_options(case))
        if s.kind == "rows":         # rows that belong to no expert are nobody's to write
            s.xs, s.dy = torch.zeros_like(s.y), torch.zeros_like(s.y)
    if s.kind in ("product_i8", "serve") and not own:
        s.wq, s.wscale = _quantise(s.w.float())
        s.w = None
    if own:
        import paper_1806_03925_amd as g
        if s.kind in ("rows", "route_back"):
            s.route = g.Route(s.expert, s.weight, s.place, s.off)
        if s.kind in ("product_i8", "serve"):
            s.weights = g.gear_weights_i8(s.w)
            s.w = None
    return s


# ---- the plain form ---------------------------------------------------------------------------------------------------
def _scores(logits, score):
    """In 64 bits: the order of experts hangs on differences that 32 bits lose."""
    v = logits.double()
    if score == "sigmoid":
        return torch.sigmoid(v)
    e = torch.exp(v - v.amax(1, keepdim=True))
    return torch.nan_to_num(e / e.sum(1, keepdim=True), nan=0.0)       # a row without an eligible expert


def _route(logits, k, bias, n, score, groups, kept, best, renormalise, scale):
    rows, experts = logits.shape
    minus = torch.tensor(-math.inf, dtype=torch.float64, device=logits.device)
    scores = _scores(logits, score)
    eligible = logits > -math.inf
    value = scores
    if bias is not None:
        value = scores + bias.double()
        eligible = eligible & (bias > -math.inf)
    if n is not None:
        eligible = eligible & (torch.arange(rows, device=logits.device)[:, None] < n)
    value = torch.where(eligible, value, minus)
    order = value if bias is not None else torch.where(eligible, logits.double(), minus)
    if groups > 1:
        top = torch.sort(value.view(rows, groups, -1), dim=2, descending=True).values[:, :, :best]
        group = torch.where(top[:, :, 0] > minus, torch.where(top > minus, top, torch.zeros_like(top)).sum(2), minus)
        first = torch.sort(group, dim=1, descending=True, stable=True).indices[:, :kept]
        keep = torch.zeros(rows, groups, dtype=torch.bool, device=logits.device).scatter_(1, first, True)
        order = torch.where(keep.repeat_interleave(experts // groups, 1), order, minus)
    by = torch.sort(order, dim=1, descending=True, stable=True)
    chosen, there = by.indices[:, :k], by.values[:, :k] > minus
    weight = torch.where(there, scores.gather(1, chosen), torch.zeros_like(minus))
    if renormalise:
        total = weight.sum(1, keepdim=True)
        weight = weight / torch.where(total > 0, total, torch.ones_like(total))
    expert = torch.where(there, chosen, torch.full_like(chosen, -1))
    line = torch.where(there, chosen, torch.full_like(chosen, experts)).flatten()
    line, at = torch.sort(line, stable=True)
    place = torch.empty_like(at).scatter_(0, at, torch.arange(at.numel(), device=at.device)).view(rows, k)
    place = torch.where(there, place, torch.full_like(place, -1))
    off = torch.searchsorted(line, torch.arange(experts + 1, device=line.device))
    return expert.int(), (scale * weight).float(), place.int(), off.int()


def _route_back(logits, expert, dweight, score, renormalise, scale):
    there, at = expert >= 0, expert.clamp(min=0).long()
    picked = torch.zeros(logits.shape, device=logits.device).scatter_add_(1, at, there.float())
    flow = torch.zeros(logits.shape, device=logits.device).scatter_add_(1, at, torch.where(there, scale * dweight, torch.zeros_like(dweight)))
    s = _scores(logits, score).float()
    if renormalise:                  # weights p = s / sum of the chosen: dp / ds = (1 - p) / sum, -p / sum
        total = (s * picked).sum(1, keepdim=True)
        total = torch.where(total > 0, total, torch.ones_like(total))
        flow = picked * (flow - (flow * s).sum(1, keepdim=True) / total) / total
    if score == "sigmoid":
        d = s * (1 - s) * flow
    else:
        d = s * (flow - (flow * s).sum(1, keepdim=True))
    return d.to(logits.dtype)


def _spread(x, place, k, dtype):
    """Rows [rows x dim], or [rows x k x dim], where they belong in the order of experts; zeros where nobody's are."""
    rows, dim = place.shape[0], x.shape[-1]
    v = (x[:, None, :].expand(rows, k, dim) if x.dim() == 2 else x).reshape(rows * k, dim)
    to = torch.where(place >= 0, place, torch.full_like(place, rows * k)).flatten().long()
    return torch.zeros(rows * k + 1, dim, dtype=v.dtype, device=v.device).index_copy_(0, to, v)[:rows * k].to(dtype)   # those of no expert end up in the last


def _collect(y, place):
    """[rows x k x dim] in 32 bits; zeros for a place that no expert was left for."""
    v = y.float()[place.clamp(min=0).flatten().long()].view(*place.shape, y.shape[1])
    return torch.where((place >= 0)[:, :, None], v, torch.zeros_like(v))


def _quantise(v):
    """Integers and scales over the last dimension; the quotient in 64 bits, as it decides a whole step next to a tie."""
    top = v.abs().amax(-1, keepdim=True).double()
    q = torch.round(127.0 * v.double() / torch.where(top > 0, top, torch.ones_like(top)))
    return q.to(torch.int8), (top / 127.0).float()


def _grouped(q, scale, wq, wscale, bounds):
    """Rows in 8-bit integers times the transposed weights of each expert."""
    return torch.cat([q[a:b].float() @ wq[e].float().t() * scale[a:b] * wscale[e].t() for e, (a, b) in enumerate(zip(bounds, bounds[1:]))])


def _plain(s):
    c = s.case
    if s.kind == "route":
        return _route(s.logits, c["k"], s.bias, s.n, **_options(c))
    if s.kind == "route_back":
        return _route_back(s.logits, s.expert, s.dweight, c["score"], c["renormalise"], c["scale"])
    if s.kind == "rows":
        dtype, k = s.x.dtype, c["k"]
        xs = _spread(s.x, s.place, k, dtype)
        back, dout = _collect(s.y, s.place), s.dout.float()
        out = s.x.float() + (s.weight[:, :, None] * back).sum(1)
        dy = _spread(s.weight[:, :, None] * dout[:, None, :], s.place, k, dtype)
        dweight = (back * dout[:, None, :]).sum(2)
        dx = dout + _collect(s.dxs, s.place).sum(1)
        return xs, out.to(dtype), dy, dweight, dx.to(dtype)
    if s.kind == "product_i8":
        return _grouped(*_quantise(s.x.float()), s.wq, s.wscale, s.bounds).to(torch.bfloat16)
    expert, weight, place, off = _route(s.logits, c["k"], None, s.n, **_options(c))
    q, scale = _quantise(s.x.float())
    q, scale = _spread(q, place, c["k"], q.dtype), _spread(scale, place, c["k"], scale.dtype)
    y = _grouped(q, scale, s.wq, s.wscale, off.tolist())
    y = torch.cat([y, y.new_zeros(place.numel() - y.shape[0], y.shape[1])])
    out = s.residual.float() + (weight[:, :, None] * _collect(y, place)).sum(1)
    return expert, weight, out.to(s.residual.dtype)


# ---- the framework's calls --------------------------------------------------------------------------------------------
def _called(s):
    import paper_1806_03925_amd as g
    c = s.case
    if s.kind == "route":
        r = g.gear_route(s.logits, c["k"], score=c["score"], bias=s.bias, groups=c["groups"], groups_kept=c["kept"], group_best=c["best"],
                         renormalise=c["renormalise"], scale=c["scale"], n=s.n)
        return r.expert, r.weight, r.place, r.off
    if s.kind == "route_back":
        return g.gear_route_backward(s.logits, s.route, s.dweight, score=c["score"], renormalise=c["renormalise"], scale=c["scale"])
    if s.kind == "rows":
        xs = g.gear_expert_gather(s.x, s.route, out=s.xs)
        out = g.gear_expert_combine(s.y, s.route, residual=s.x)
        dy, dweight = g.gear_expert_combine_backward(s.dout, s.y, s.route, dy=s.dy)
        dx = g.gear_expert_combine(s.dxs, s.route, weighted=False, residual=s.dout)
        return xs, out, dy, dweight, dx
    if s.kind == "product_i8":
        return g.gear_matmul_i8(g.gear_rows_i8(s.x), s.weights, s.off)
    r = g.gear_route(s.logits, c["k"], n=s.n)
    y = g.gear_matmul_i8(g.gear_expert_gather_i8(s.x, r), s.weights, r.off, out_dtype=torch.float32)     # what is added up is not rounded before
    return r.expert, r.weight, g.gear_expert_combine(y, r, residual=s.residual, out_dtype=s.residual.dtype)


def run(s):
    return _called(s) if own else _plain(s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    """Inputs read once, outputs written once, the products' operations."""
    kind, rows, size, experts = case["kind"], float(case["rows"]), SIZE[case["dtype"]], case["experts"]
    if kind == "route":
        return {"bytes": rows * experts * size + 12.0 * rows * case["k"] + 8.0 * experts, "flops": rows * experts * 5.0}
    if kind == "route_back":         # weights divided by their sum hang on the chosen scores alone
        few = case["renormalise"] or case["score"] == "sigmoid"
        read = min(rows * case["k"], rows * experts) if few else rows * experts
        return {"bytes": (read + rows * experts) * size + 8.0 * rows * case["k"], "flops": rows * experts * 4.0}
    if kind == "product_i8":
        n, out = rows * case["dim"], case["out"]
        return {"bytes": n * size + max(1, experts) * case["dim"] * out + 2 * rows * out, "flops": 2.0 * n * out}
    used, k = float(case["used"]), case["k"]
    if kind == "rows":
        return {"bytes": (6 * rows + 5 * used * k) * case["dim"] * size + 16.0 * rows * k, "flops": 7.0 * used * k * case["dim"]}
    dim, out = case["dim"], case["out"]
    return {"bytes": rows * experts * 4 + rows * dim * size + experts * dim * out + 2 * rows * out * size + 8.0 * rows * k,
            "flops": 2.0 * used * k * dim * out}


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------------
def _exact_choice(case, s):
    """[rows x k] chosen experts (-1: none) and the scores; ranks counted pair by pair instead of sorted."""
    rows, experts, k, o = case["rows"], case["experts"], case["k"], _options(case)
    v = s.logits.double()
    scores = 1 / (1 + torch.exp(-v)) if o["score"] == "sigmoid" else torch.softmax(v, 1)
    bias = torch.zeros(experts, dtype=torch.float64, device="cuda") if s.bias is None else s.bias.double()
    expert = torch.full((rows, k), -1, dtype=torch.long, device="cuda")
    part = max(1, 60_000_000 // (experts * experts))
    index = torch.arange(experts, device="cuda")

    def rank(x):       # how many of a row come before each
        ahead = (x[:, None, :] > x[:, :, None]) | ((x[:, None, :] == x[:, :, None]) & (torch.arange(x.shape[1], device="cuda")[None, None, :]
                                                                                    < torch.arange(x.shape[1], device="cuda")[None, :, None]))
        return ahead.sum(2)

    for a in range(0, case["used"], part):
        b = min(case["used"], a + part)
        ok = ~torch.isinf(v[a:b]) & ~torch.isinf(bias)
        value = (scores[a:b] + bias).masked_fill(~ok, -math.inf)
        order = value if s.bias is not None else v[a:b].masked_fill(~ok, -math.inf)
        if o["groups"] > 1:
            per = experts // o["groups"]
            inside = value.view(b - a, o["groups"], per)
            best = inside.masked_fill(rank(inside.reshape(-1, per)).view(inside.shape) >= o["best"], -math.inf)
            total = torch.where(torch.isinf(best), 0.0, best).sum(2).masked_fill(torch.isinf(best).all(2), -math.inf)
            order = order.masked_fill((rank(total) >= o["kept"])[:, index // per], -math.inf)
        at = rank(order)
        for j in range(k):
            hit = (at == j) & ~torch.isinf(order)
            expert[a:b, j] = torch.where(hit.any(1), (hit * index).sum(1), -1)
    return expert, scores


def _exact_weights(case, expert, scores):
    o = _options(case)
    w = torch.where(expert >= 0, scores.gather(1, expert.clamp(min=0)), 0.0)
    if o["renormalise"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return o["scale"] * w


def _exact_i8(v):
    """What the nearest integers of 127 v / max stand for."""
    v = v.double()
    unit = v.abs().amax(-1, keepdim=True) / 127
    z = v / torch.where(unit > 0, unit, 1.0)
    low = torch.floor(z)
    up = (z - low > 0.5) | ((z - low == 0.5) & (low % 2 != 0))
    return (low + up) * unit


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "product_i8":
        rows = _exact_i8(s.x)
        out = torch.empty(case["rows"], case["out"], dtype=torch.float64, device="cuda")
        for e, n in enumerate(s.sizes):
            part = slice(s.bounds[e], s.bounds[e] + n)
            out[part] = rows[part].matmul(_exact_i8(s.w[e]).t().contiguous())
        return out
    expert, scores = _exact_choice(case, s)
    weight = _exact_weights(case, expert, scores)
    if kind == "route":
        return None, weight, None, None
    if kind == "route_back":
        with torch.enable_grad():
            v = s.logits.double().requires_grad_()
            fresh = torch.sigmoid(v) if case["score"] == "sigmoid" else torch.softmax(v, 1)
            return torch.autograd.grad(_exact_weights(case, expert, fresh), v, s.dweight.double())[0]
    rows, k = case["rows"], case["k"]
    pairs = (expert >= 0).flatten().nonzero().flatten()
    pairs = pairs[torch.sort(expert.flatten()[pairs], stable=True).indices]        # (row, slot) in the order of experts
    source = pairs // k
    if kind == "rows":
        w = weight.flatten()[pairs][:, None]
        xs, dy = (torch.zeros(rows * k, case["dim"], dtype=torch.float64, device="cuda") for _ in range(2))
        xs[:pairs.numel()] = s.x.double()[source]
        dy[:pairs.numel()] = w * s.dout.double()[source]
        out = s.x.double().index_add_(0, source, w * s.y[:pairs.numel()].double())
        dx = s.dout.double().index_add_(0, source, s.dxs[:pairs.numel()].double())
        dweight = torch.zeros(rows * k, dtype=torch.float64, device="cuda")
        dweight[pairs] = (s.dout.double()[source] * s.y[:pairs.numel()].double()).sum(1)
        return xs, out, dy, dweight.view(rows, k), dx
    out, x = s.residual.double(), _exact_i8(s.x)
    of = expert.flatten()[pairs]
    for e in range(case["experts"]):
        mine = pairs[of == e]
        if mine.numel():
            out.index_add_(0, mine // k, weight.flatten()[mine][:, None] * x[mine // k].matmul(_exact_i8(s.w[e]).t().contiguous()))
    return None, weight, out
