"""Rows on their way to their experts and back, and products in 8-bit integers, against evaluations in 64 bits.

Tolerances.  u = 2^-24.  A weighted sum of k rows in fp32: (k + 2) u of the sum of its terms' magnitudes, and one rounding of the result.  A dot product of
dim terms, added up by at least 16 threads (32 above 128 columns, 64 above 256, 256 above 4096) and then in a tree: at most (dim / 16 + 16) u of its magnitudes.
Integers and copies are equal.  A product in integers is exact up to its conversion and two factors: 3 u, and one rounding to bf16."""
import itertools
import math

import pytest
import torch

from test_gpu_experts import BF16, F32, HALF, U, g, gen, strided, within  # noqa: F401 (g: the fixture)

pytestmark = pytest.mark.gpu


def routed(g, rows, k, experts, seed, empty=True):
    """A route of random choices; some slots, and some whole rows, without an expert."""
    r = gen(seed)
    logits = torch.randn(rows, experts, device="cuda", generator=r)
    if empty:
        logits[1::3, : experts - max(1, k // 2)] = -math.inf
        logits[2::5] = -math.inf
    return g.gear_route(logits, k, renormalise=False)


def pairs_of(route):
    there = (route.place >= 0).flatten()
    row = torch.arange(route.rows, device="cuda").repeat_interleave(route.k)[there]
    return there, row, route.place.flatten()[there].long()


SHAPES = [(1, 8, 1, 1), (1, 1152, 4, 8), (7, 72, 3, 5), (65, 128, 2, 9), (33, 136, 8, 16), (50, 520, 5, 6), (40, 1152, 2, 8), (9, 2056, 32, 40), (3, 8200, 3, 4),
          (2, 65536, 2, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim,k,experts", SHAPES)
def test_gather(g, rows, dim, k, experts, dtype):
    x = torch.randn(rows, dim, device="cuda", generator=gen(dim)).to(dtype)
    route = routed(g, rows, k, experts, rows)
    there, row, place = pairs_of(route)
    want = torch.full((rows * k, dim), -7.0, dtype=dtype, device="cuda")
    want[place] = x[row]
    assert int(route.off[-1]) == place.numel()
    for xx, out in ((x, torch.full_like(want, -7.0)), (strided(x, 8), strided(torch.full_like(want, -7.0), 16))):
        assert g.gear_expert_gather(xx, route, out=out) is out and torch.equal(out, want)
    assert torch.equal(g.gear_expert_gather(x, route)[:place.numel()], want[:place.numel()])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim,k,experts", SHAPES)
def test_combine(g, rows, dim, k, experts, dtype):
    r = gen(dim + k)
    y = torch.randn(rows * k, dim, device="cuda", generator=r).to(dtype)
    res = torch.randn(rows, dim, device="cuda", generator=r).to(dtype)
    route = routed(g, rows, k, experts, rows)
    there, row, place = pairs_of(route)
    y[int(route.off[-1]):] = math.nan                        # nobody's
    for weighted, residual in itertools.product((True, False), (None, res)):
        w = route.weight.flatten()[there].double()[:, None] if weighted else 1.0
        want = torch.zeros(rows, dim, dtype=torch.float64, device="cuda") if residual is None else residual.double()
        size = want.abs().index_add_(0, row, (w * y[place].double()).abs())
        want = want.index_add_(0, row, w * y[place].double())
        bound = (k + 2) * U * size + HALF[dtype] * want.abs()
        got = g.gear_expert_combine(y, route, weighted=weighted, residual=residual)
        within(got, want, bound)
        out = strided(torch.zeros_like(res), 8) if residual is None else strided(residual, 24)
        assert g.gear_expert_combine(strided(y, 16), route, weighted=weighted, residual=out if residual is not None else None, out=out) is out
        assert torch.equal(out, got)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim,k,experts", SHAPES)
def test_combine_backward(g, rows, dim, k, experts, dtype):
    r = gen(dim + k)
    y = torch.randn(rows * k, dim, device="cuda", generator=r).to(dtype)
    dout = torch.randn(rows, dim, device="cuda", generator=r).to(dtype)
    route = routed(g, rows, k, experts, rows)
    there, row, place = pairs_of(route)
    y[int(route.off[-1]):] = math.nan
    w = route.weight.flatten()[there].double()[:, None]
    dy = torch.full((rows * k, dim), -7.0, dtype=torch.float64, device="cuda")
    dy[place] = w * dout.double()[row]
    terms = dout.double()[row] * y[place].double()
    dweight, size = (torch.zeros(rows * k, dtype=torch.float64, device="cuda") for _ in range(2))
    dweight[there], size[there] = terms.sum(1), terms.abs().sum(1)
    for d, yy, out in ((dout, y, torch.full_like(y, -7.0)), (strided(dout, 8), strided(y, 16), strided(torch.full_like(y, -7.0), 24))):
        got, got_w = g.gear_expert_combine_backward(d, yy, route, dy=out)
        assert got is out
        within(got, dy, (U + HALF[dtype]) * dy.abs())
        within(got_w.flatten(), dweight, (dim / 16 + 16) * U * size)
    again = y.clone()                                        # dy in y's place
    _, w_again = g.gear_expert_combine_backward(dout, again, route, dy=again)
    total = place.numel()
    assert torch.equal(again[:total], got[:total]) and torch.equal(w_again, got_w) and again[total:].isnan().all()


def test_empty_slots_and_nan(g):
    """A slot without a place is a row of zeros: NaN weights reach the sum, other numbers do not, and nothing comes back through it."""
    x = torch.randn(4, 64, device="cuda", generator=gen(1))
    logits = torch.full((4, 6), -math.inf, device="cuda")
    logits[0, 2], logits[1, :3], logits[3, 0] = 1.0, 0.5, math.nan
    route = g.gear_route(logits, 2)
    assert route.expert.tolist() == [[2, -1], [0, 1], [-1, -1], [-1, -1]] and route.weight[3].isnan().all() and route.weight[2].tolist() == [0, 0]
    y = torch.full((8, 64), math.inf, device="cuda")
    y[:3] = x[:3]
    out = g.gear_expert_combine(y, route, residual=x)
    assert torch.isfinite(out[:3]).all() and torch.equal(out[2], x[2]) and out[3].isnan().all()
    assert torch.equal(g.gear_expert_combine(y, route, weighted=False, residual=x)[2:], x[2:])
    _, dweight = g.gear_expert_combine_backward(torch.full_like(x, math.nan), y, route)
    assert dweight[0, 0].isnan() and dweight[0, 1] == 0 and torch.equal(dweight[2:], torch.zeros(2, 2, device="cuda"))


def test_places_out_of_range_are_none(g):
    x = torch.randn(3, 64, device="cuda", generator=gen(1))
    place = torch.tensor([[0, 6], [-9, 2], [2 ** 31 - 1, 5]], dtype=torch.int32, device="cuda")
    route = g.Route(torch.zeros_like(place), torch.ones(3, 2, device="cuda"), place, torch.tensor([0, 6], dtype=torch.int32, device="cuda"))
    room = torch.full((6, 64), 5.0, device="cuda")
    g.gear_expert_gather(x, route, out=room)
    assert torch.equal(room, torch.stack([x[0], room[1] * 0 + 5, x[1], room[1] * 0 + 5, room[1] * 0 + 5, x[2]]))
    assert torch.equal(g.gear_expert_combine(room, route), x)
    dy, dw = g.gear_expert_combine_backward(x, room, route, dy=torch.zeros_like(room))
    assert torch.equal(dy, torch.where((room == 5).all(1, keepdim=True), 0.0, room)) and dw[0, 1] == 0 and dw[1, 0] == 0 and dw[2, 0] == 0
    q = g.RowsI8(torch.full((6, 128), 9, dtype=torch.int8, device="cuda"), torch.full((6,), 3.0, device="cuda"), 64)
    g.gear_expert_gather_i8(x, route, out=q)
    assert (q.q[[1, 3, 4]] == 9).all() and q.scale[[1, 3, 4]].tolist() == [3.0] * 3


def test_offsets_past_32_bits(g):
    """Places whose bytes and elements lie beyond 2^31."""
    rows, k, dim = 70_000, 1, 32_768
    x = torch.randn(rows, 1, device="cuda", generator=gen(4)).to(BF16).expand(rows, dim).contiguous()
    place = torch.randperm(rows, device="cuda", generator=gen(5)).to(torch.int32)[:, None].contiguous()
    route = g.Route(torch.zeros_like(place), torch.full((rows, k), 2.0, device="cuda"), place, torch.tensor([0, rows], dtype=torch.int32, device="cuda"))
    xs = g.gear_expert_gather(x, route)
    assert torch.equal(xs[place[:, 0].long(), 0], x[:, 0]) and torch.equal(xs[place[:, 0].long(), dim - 1], x[:, 0])
    back = g.gear_expert_combine(xs, route)
    assert torch.equal(back[:, 0], 2 * x[:, 0]) and torch.equal(back[:, dim - 1], 2 * x[:, 0])
    del back
    q = g.gear_expert_gather_i8(x, route)
    assert torch.equal(q.q[place[:, 0].long(), dim - 1].int(), 127 * torch.sign(x[:, 0]).int())
    dy, dw = g.gear_expert_combine_backward(x, xs, route, dy=xs)
    assert torch.equal(dy[place[:, 0].long(), dim - 1], 2 * x[:, 0])
    within(dw[:, 0], dim * x[:, 0].double() ** 2, (dim / 16 + 16) * U * dim * x[:, 0].double() ** 2)


def test_no_rows(g):
    route = g.gear_route(torch.empty(0, 8, device="cuda"), 2)
    x = torch.empty(0, 64, device="cuda")
    assert g.gear_expert_gather(x, route).shape == (0, 64) and g.gear_expert_combine(x, route, residual=x).shape == (0, 64)
    dy, dw = g.gear_expert_combine_backward(x, x, route)
    assert dy.shape == (0, 64) and dw.shape == (0, 2) and g.gear_expert_gather_i8(x, route).q.shape == (0, 128)
    w = g.gear_weights_i8(torch.randn(8, 24, 64, device="cuda"))
    assert g.gear_matmul_i8(g.gear_expert_gather_i8(x, route), w, route.off).shape == (0, 24)


def test_results_in_the_place_of_rows_still_to_be_read_are_refused(g):
    """With one expert a row the sizes would allow it."""
    x = torch.randn(6, 64, device="cuda")
    route = g.gear_route(torch.randn(6, 3, device="cuda"), 1)
    for call in (lambda: g.gear_expert_gather(x, route, out=x), lambda: g.gear_expert_combine(x, route, out=x),
                 lambda: g.gear_expert_combine_backward(x, x.clone(), route, dy=x)):
        with pytest.raises(g.GearError):
            call()


def test_results_that_share_a_part_of_what_is_read_are_refused(g):
    room = torch.randn(9, 64, device="cuda")
    a, b, c = room[:6], room[1:7], room.view(-1)[16:16 + 6 * 64].view(6, 64)
    logits = torch.randn(6, 3, device="cuda")
    route = g.gear_route(logits, 1)
    wide = torch.randn(6, 192, device="cuda")
    dense = g.gear_route(logits, 3)
    dw = torch.randn(6, 3, device="cuda")
    for call in (lambda: g.gear_expert_gather(a, route, out=b), lambda: g.gear_expert_gather(a, route, out=c), lambda: g.gear_expert_combine(b, route, out=a),
                 lambda: g.gear_expert_combine(a.clone(), route, residual=a, out=b), lambda: g.gear_expert_combine(a.clone(), route, residual=c, out=a),
                 lambda: g.gear_expert_combine_backward(a, a.clone(), route, dy=b), lambda: g.gear_expert_combine_backward(a.clone(), a, route, dy=c),
                 lambda: g.gear_expert_combine_backward(a, a.clone(), route, dweight=room.view(-1)[:6].view(6, 1)),
                 lambda: g.gear_expert_combine_backward(a, a.clone(), route, dweight=route.weight),
                 lambda: g.gear_expert_gather(wide[:, :64], route, out=wide[:, 32:96]),
                 lambda: g.gear_route_backward(logits, dense, dw, out=dw), lambda: g.gear_route_backward(logits, dense, dw, out=dense.weight),
                 lambda: g.gear_rows_i8(a, out=g.RowsI8(room.view(-1)[64:64 + 6 * 32].view(torch.int8).view(6, 128), torch.empty(6, device="cuda"), 64)),
                 lambda: g.gear_rows_i8(a, out=g.RowsI8(torch.empty(6, 128, dtype=torch.int8, device="cuda"), room.view(-1)[:6], 64))):
        with pytest.raises(g.GearError):
            call()
    # columns of one matrix, and parts of one allocation one behind the other
    x = wide[:, :64].clone()
    want = g.gear_expert_gather(x, route)
    assert torch.equal(g.gear_expert_gather(wide[:, :64], route, out=wide[:, 64:128]), want)
    assert torch.equal(g.gear_expert_combine(wide[:, 64:128], route, weighted=False, out=wide[:, 128:]), x)
    both = torch.cat([x, x])
    assert torch.equal(g.gear_expert_gather(both[:6], route, out=both[6:]), want)


# ---- 8-bit integers -------------------------------------------------------------------------------------------------
def integers(v):
    """q and scale from the definition, 64 bits: floor, remainder and parity instead of a rounding."""
    v = v.double()
    broken = ~torch.isfinite(v).all(-1, keepdim=True)
    v = torch.where(broken, 0.0, v)
    top = v.abs().amax(-1, keepdim=True)
    z = 127 * v / torch.where(top > 0, top, 1.0)
    low = torch.floor(z)
    q = low + ((z - low > 0.5) | ((z - low == 0.5) & (low % 2 != 0)))
    return q, torch.where(broken, math.nan, top / 127)[..., 0]


def check_rows(rows8, v):
    q, scale = integers(v)
    dim = v.shape[1]
    assert torch.equal(rows8.q[:, :dim].double(), q) and (rows8.q[:, dim:] == 0).all()
    within(rows8.scale, scale, U * scale.nan_to_num().abs() + 2.0 ** -149)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(1, 8), (3, 72), (5, 128), (70, 136), (33, 520), (9, 1152), (4, 2056), (300, 4096), (3, 8200), (2, 65536)])
def test_rows_in_integers(g, rows, dim, dtype):
    r = gen(rows + dim)
    x = (torch.randn(rows, dim, device="cuda", generator=r) * torch.exp(2 * torch.randn(rows, dim, device="cuda", generator=r))).to(dtype)
    check_rows(g.gear_rows_i8(x), x)
    check_rows(g.gear_rows_i8(strided(x, 8)), x)
    route = routed(g, rows, 3, 5, dim)
    there, row, place = pairs_of(route)
    out = g.gear_expert_gather_i8(x, route, out=g.RowsI8(torch.full((rows * 3, (dim + 127) // 128 * 128), 55, dtype=torch.int8, device="cuda"),
                                                         torch.full((rows * 3,), 0.5, device="cuda"), dim))
    q, scale = integers(x)
    assert torch.equal(out.q[place, :dim].double(), q[row]) and (out.q[place, dim:] == 0).all()
    assert torch.equal(out.scale[place], g.gear_rows_i8(x).scale[row])
    assert (out.q[place.numel():] == 55).all() and (out.scale[place.numel():] == 0.5).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_integers_next_to_ties(g, dtype):
    """Quotients on a half (top = 127 2^e) and one unit in the last place beside it, of either sign; other largest values, too."""
    half = torch.arange(-126.5, 127.0, 0.5, device="cuda", dtype=torch.float64)
    rows = []
    for scale in (1.0, 2.0 ** -3, 2.0 ** 40, 2.0 ** -120, 2.0 ** -140, 3.0, 1.7, 2.0 ** 120):
        v = (half * scale).to(dtype)
        up, down = torch.nextafter(v, torch.full_like(v, math.inf)), torch.nextafter(v, torch.full_like(v, -math.inf))
        top = torch.tensor([127.0 * scale], device="cuda").to(dtype)
        for w in (v, up, down):
            rows.append(torch.nn.functional.pad(torch.cat([torch.where(w.abs() > top, 0, w), top]), (0, 512 - half.numel() - 1)))
    x = torch.stack(rows)
    check_rows(g.gear_rows_i8(x), x)


def test_rows_of_zeros_infinities_and_denormals(g):
    x = torch.randn(8, 200, device="cuda", generator=gen(3))
    x[0], x[1, 3], x[2, 7], x[3, 199] = 0.0, math.inf, math.nan, -math.inf
    x[4] *= 2.0 ** -140
    x[5], x[5, 0] = 0.0, -(2.0 ** -149)
    x[6] *= 2.0 ** 125
    x[7, :] = -0.0
    check_rows(g.gear_rows_i8(x), x)
    w = g.gear_weights_i8(x)
    assert w.scale.shape == (1, 8)
    _, scale = integers(x)
    within(w.scale[0], scale, U * scale.nan_to_num().abs() + 2.0 ** -149)
    rows = g.gear_rows_i8(torch.randn(3, 200, device="cuda"))
    out = g.gear_matmul_i8(rows, w, out_dtype=F32)
    assert out[:, 1:4].isnan().all() and torch.equal(out[:, [0, 7]], torch.zeros(3, 2, device="cuda"))
    want = (rows.q[:, :200].double() @ integers(x)[0].t().contiguous()) * rows.scale[:, None].double() * w.scale.double()
    want = torch.where(want.abs() > torch.finfo(F32).max, want.sign() * math.inf, want)      # rows of 2^125 reach beyond fp32
    within(out[:, 4:7], want[:, 4:7], 3.01 * U * want[:, 4:7].abs().nan_to_num(posinf=0) + 2.0 ** -149)
    out = g.gear_matmul_i8(g.gear_rows_i8(x), g.gear_weights_i8(torch.randn(16, 200, device="cuda")), out_dtype=F32)
    assert out[1:4].isnan().all() and torch.equal(out[0], torch.zeros(16, device="cuda"))


PRODUCTS = [(1, 8, 8, 0), (1, 1024, 1152, 0), (5, 72, 136, 0), (33, 520, 576, 16), (300, 1024, 1152, 0), (535, 816, 6208, 0), (1024, 1024, 512, 0),
            (700, 1024, 264, 9), (2000, 2048, 256, 0), (4097, 72, 320, 0), (9000, 264, 200, 4), (4096, 2048, 128, 7), (17408, 1024, 136, 8), (40, 24, 65536, 0), (300, 200, 3200, 0)]


@pytest.mark.parametrize("rows,n,k,experts", PRODUCTS)
def test_product(g, rows, n, k, experts):
    r = gen(rows + n + k)
    e = max(1, experts)
    x = torch.randn(rows, k, device="cuda", generator=r)
    w = torch.randn(e, n, k, device="cuda", generator=r)
    sizes = torch.rand(e, device="cuda", generator=r)
    sizes[1::3] = 0
    ends = torch.cat([torch.zeros(1, device="cuda"), (sizes.cumsum(0) / sizes.sum() * (rows - rows // 9)).round()])
    off = ends.to(torch.int32) if experts else None
    q = g.gear_rows_i8(x)
    wq, ws = integers(w)
    weights = g.gear_weights_i8(w)
    within(weights.scale, ws, U * ws)
    want = torch.full((rows, n), -7.0, dtype=torch.float64, device="cuda")
    bounds = off.tolist() if experts else [0, rows]
    for i in range(e):
        a, b = bounds[i], bounds[i + 1]
        want[a:b] = (q.q[a:b, :k].double() @ wq[i].t().contiguous()) * q.scale[a:b, None].double() * weights.scale[i].double()
    for dtype, pad in ((F32, 0), (BF16, 0), (BF16, 8), (F32, 16)):
        out = strided(torch.full((rows, n), -7.0, dtype=dtype, device="cuda"), pad)
        status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
        assert g.gear_matmul_i8(q, weights, off, out=out, status=status if experts else None) is out
        within(out, want, (3.01 * U + (HALF[dtype] if dtype is BF16 else 0)) * want.abs())
        assert not experts or int(status) == g.GEAR_OK


def test_largest_integers_are_added_up_exactly(g):
    """127^2 65536 = 2^30 - 2^24 + ..., and -128 from weights that were integers before: all 31 bits are used, and one unit shows."""
    k = 65536
    q = torch.full((34, k), 127, dtype=torch.int8, device="cuda")
    q[1::2] = -127
    q[2, 5] = 126
    w = torch.full((40, k), -128, dtype=torch.int8, device="cuda")
    w[3] = 127
    one = torch.ones(34, device="cuda"), torch.ones(40, device="cuda")
    out = g.gear_matmul_i8(g.RowsI8(q, one[0], k), g.gear_weights_i8(w, one[1]), out_dtype=F32)
    want = q.double() @ w.double().t().contiguous()
    within(out, want, U * want.abs())
    assert out[0, 0] == -127 * 128 * k and out[2, 0] == torch.tensor(-127 * 128 * k + 128, dtype=F32)


@pytest.mark.parametrize("experts,n,k", [(1, 8, 8), (3, 72, 136), (2, 136, 520)])
def test_weights_that_are_integers_already(g, experts, n, k):
    r = gen(n)
    w = torch.randint(-128, 128, (experts, n, k), device="cuda", generator=r).to(torch.int8)
    scale = torch.rand(experts, n, device="cuda", generator=r) + 0.1
    x = torch.randn(50, k, device="cuda", generator=r)
    off = torch.linspace(0, 50, experts + 1, device="cuda").to(torch.int32)
    q = g.gear_rows_i8(x)
    weights = g.gear_weights_i8(w, scale)
    assert torch.equal(weights.scale, scale)
    scale.zero_()                                            # the weights keep their own
    out = g.gear_matmul_i8(q, weights, off, out_dtype=F32)
    b = off.tolist()
    want = torch.cat([q.q[b[i]:b[i + 1], :k].double() @ w[i].double().t().contiguous() * weights.scale[i].double() for i in range(experts)])
    want = want * q.scale[:, None].double()
    within(out, want, 3.01 * U * want.abs())


def test_offsets_that_are_no_list(g):
    q = g.gear_rows_i8(torch.randn(20, 64, device="cuda"))
    w = g.gear_weights_i8(torch.randn(3, 24, 64, device="cuda"))
    out = torch.full((20, 24), 5.0, device="cuda")
    g.gear_expert_status().zero_()
    for off in ([0, 5, 4, 20], [1, 5, 8, 20], [0, 5, 8, 21], [0, -1, 8, 20]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        g.gear_matmul_i8(q, w, off, out=out, status=status)
        assert int(status) == g.GEAR_ERR_RANGE and (out == 5).all()
        assert int(g.gear_expert_status()) == g.GEAR_OK
    g.gear_matmul_i8(q, w, off, out=out)
    assert int(g.gear_expert_status()) == g.GEAR_ERR_RANGE and (out == 5).all()
    g.gear_expert_status().zero_()


def test_refusals(g):
    x = torch.randn(4, 64, device="cuda")
    route = g.gear_route(torch.randn(4, 6, device="cuda"), 2)
    y = torch.randn(8, 64, device="cuda")
    w = g.gear_weights_i8(torch.randn(6, 24, 64, device="cuda"))
    one = g.gear_weights_i8(torch.randn(24, 64, device="cuda"))
    q = g.gear_rows_i8(x)
    for call in (lambda: g.gear_expert_gather(x[:3], route), lambda: g.gear_expert_gather(x.cpu(), route), lambda: g.gear_expert_gather(x.double(), route),
                 lambda: g.gear_expert_gather(x[:, :60], route), lambda: g.gear_expert_gather(x, route, out=y[:7]),
                 lambda: g.gear_expert_gather(x, route, out=y.to(BF16)), lambda: g.gear_expert_combine(y[:7], route),
                 lambda: g.gear_expert_combine(y, route, residual=x.to(BF16)), lambda: g.gear_expert_combine(y, route, residual=x[:, :56]),
                 lambda: g.gear_expert_combine(y, route, out=y), lambda: g.gear_expert_combine_backward(x, y[:, :56], route),
                 lambda: g.gear_expert_combine_backward(x, y, route, dweight=torch.zeros(7, device="cuda")),
                 lambda: g.gear_expert_combine_backward(x, y, route, dy=x), lambda: g.gear_rows_i8(x.half()), lambda: g.gear_rows_i8(x[0]),
                 lambda: g.gear_rows_i8(x[:, :60]), lambda: g.gear_rows_i8(x, out=g.gear_rows_i8(x[:2])), lambda: g.gear_expert_gather_i8(x, route, out=q),
                 lambda: g.RowsI8(q.q, q.scale, 200), lambda: g.RowsI8(q.q, q.scale[:2], 64), lambda: g.RowsI8(q.q.cpu(), q.scale, 64),
                 lambda: g.RowsI8(q.q.view(torch.uint8), q.scale, 64), lambda: g.gear_weights_i8(torch.randn(24, 60, device="cuda")),
                 lambda: g.gear_weights_i8(torch.randn(20, 64, device="cuda")), lambda: g.gear_weights_i8(torch.zeros(24, 64, device="cuda"), torch.ones(24, device="cuda")),
                 lambda: g.gear_weights_i8(torch.zeros(24, 64, dtype=torch.int8, device="cuda"), torch.ones(23, device="cuda")),
                 lambda: g.gear_weights_i8(torch.zeros(24, 64, dtype=torch.int8, device="cuda")), lambda: g.gear_matmul_i8(q, w),
                 lambda: g.gear_matmul_i8(g.gear_rows_i8(x[:, :56]), one), lambda: g.gear_matmul_i8(q, w, route.off[:6]),
                 lambda: g.gear_matmul_i8(q, one, out_dtype=torch.float16), lambda: g.gear_matmul_i8(q, one, out=x)):
        with pytest.raises(g.GearError):
            call()


# ---- as they are used together --------------------------------------------------------------------------------------
def layer64(x, wr, w, expert, renormalise=True):
    """x + sum of the chosen experts' products, in 64 bits, the choice held fixed."""
    s = torch.softmax(x @ wr.t(), 1).gather(1, expert)
    s = s / s.sum(1, keepdim=True)
    y = torch.stack([x @ w[e].t() for e in range(w.shape[0])], 1)              # every expert of every row
    return x + (s[:, :, None] * y.gather(1, expert[:, :, None].expand(-1, -1, w.shape[1]))).sum(1)


def test_a_layer_learns_by_its_gradients(g):
    """Router, experts and sums in fp32, forward and back, against autograd in 64 bits."""
    rows, dim, experts, k = 150, 72, 8, 3
    r = gen(11)
    x, dout = (torch.randn(rows, dim, device="cuda", generator=r) for _ in range(2))
    wr, w = torch.randn(experts, dim, device="cuda", generator=r) * 0.3, torch.randn(experts, dim, dim, device="cuda", generator=r) * dim ** -0.5
    router, weights = g.ExpertWeights(wr), g.ExpertWeights(w)
    logits = g.gear_expert_matmul(x, router)
    route = g.gear_route(logits, k)
    xs = g.gear_expert_gather(x, route)
    y = g.gear_expert_matmul(xs, weights, route.off)
    out = g.gear_expert_combine(y, route, residual=x)
    dy, dweight = g.gear_expert_combine_backward(dout, y, route)
    dw = g.gear_expert_wgrad(dy, xs, route.off)
    dxs = g.gear_expert_dgrad(dy, weights, route.off)
    dlogits = g.gear_route_backward(logits, route, dweight)
    dwr = g.gear_expert_wgrad(dlogits, x)[0]
    dx = g.gear_expert_combine(dxs, route, weighted=False, residual=dout)
    dx += g.gear_expert_dgrad(dlogits, router)
    p = [t.double().requires_grad_() for t in (x, wr, w)]
    want = layer64(*p, route.expert.long())
    grads = torch.autograd.grad(want, p, dout.double())
    # no bound of the worst case, which every term rounded one way would reach: a sum of n <= 150 terms of either sign errs by about sqrt(n) u = 7.3e-7 of its typical
    # size, five of them stand in a row (logits, experts, sums, dots, gradients): 3.7e-6, and an error of logits of a typical size of 2.5 is a relative one of the
    # weights: 9e-6.  Six deviations are 5.5e-5 of a typical value, and the largest is larger.  (Each operator by itself is held to its worst case above.)
    for got, ref in ((out, want.detach()), (dx, grads[0]), (dwr, grads[1]), (dw, grads[2])):
        within(got, ref, 1e-4 * ref.abs().max())


def test_a_layer_serves_in_integers(g):
    """Routing, rows in integers, products and sums in one captured graph, replayed for other rows, against the same from 64 bits."""
    rows, dim, out_dim, experts, k = 90, 136, 72, 8, 3
    r = gen(12)
    x, logits = torch.zeros(rows, dim, device="cuda", dtype=BF16), torch.zeros(rows, experts, device="cuda")
    n = torch.tensor([rows], dtype=torch.int32, device="cuda")
    w = torch.randn(experts, out_dim, dim, device="cuda", generator=r) * dim ** -0.5
    weights = g.gear_weights_i8(w)

    def serve():
        route = g.gear_route(logits, k, n=n)
        y = g.gear_matmul_i8(g.gear_expert_gather_i8(x, route), weights, route.off)
        return route, g.gear_expert_combine(y, route)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        serve()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        route, out = serve()
    wq, ws = integers(w)
    w64 = wq * ws[..., None]
    for i in range(3):
        x.copy_(torch.randn(rows, dim, device="cuda", generator=r))
        logits.copy_(torch.randn(rows, experts, device="cuda", generator=r))
        n.fill_(rows - 20 * i)
        graph.replay()
        _, eager = serve()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(out[rows - 20 * i:], torch.zeros_like(out[rows - 20 * i:]))
        xq, xs = integers(x)
        y = torch.stack([(xq * xs[:, None]) @ w64[e].t().contiguous() for e in range(experts)], 1)
        chosen = y.gather(1, route.expert.clamp(min=0).long()[:, :, None].expand(-1, -1, out_dim)) * route.weight.double()[:, :, None]
        # a product in bf16 (half a step and 5 u: the scales are fp32 themselves), the sum, and its rounding
        within(out, chosen.sum(1), HALF[BF16] * chosen.sum(1).abs() + (HALF[BF16] + (k + 8) * U) * 1.01 * chosen.abs().sum(1))
    assert int(g.gear_expert_status()) == g.GEAR_OK


@pytest.mark.parametrize("rows,dim,k,experts", SHAPES)
def test_combine_of_products_in_fp32(g, rows, dim, k, experts):
    """Products that were not rounded on their way to a bf16 sum: one rounding in all, that of the result."""
    r = gen(dim + k)
    y = torch.randn(rows * k, dim, device="cuda", generator=r)
    res = torch.randn(rows, dim, device="cuda", generator=r).to(BF16)
    route = routed(g, rows, k, experts, rows)
    there, row, place = pairs_of(route)
    y[int(route.off[-1]):] = math.nan                        # nobody's
    for weighted, residual in itertools.product((True, False), (None, res)):
        w = route.weight.flatten()[there].double()[:, None] if weighted else 1.0
        want = torch.zeros(rows, dim, dtype=torch.float64, device="cuda") if residual is None else residual.double()
        size = want.abs().index_add_(0, row, (w * y[place].double()).abs())
        want = want.index_add_(0, row, w * y[place].double())
        got = g.gear_expert_combine(y, route, weighted=weighted, residual=residual, out_dtype=BF16)
        assert got.dtype is BF16
        within(got, want, (k + 2) * U * size + HALF[BF16] * want.abs())
        out = strided(torch.zeros_like(res), 8) if residual is None else strided(residual, 24)
        assert g.gear_expert_combine(strided(y, 16), route, weighted=weighted, residual=out if residual is not None else None, out=out, out_dtype=BF16) is out
        assert torch.equal(out, got)
    assert g.gear_expert_combine(y, route).dtype is F32          # said, not taken from the residual's type


def test_combine_refuses_other_types(g):
    x, y = torch.randn(4, 64, device="cuda"), torch.randn(8, 64, device="cuda")
    route = g.gear_route(torch.randn(4, 6, device="cuda"), 2)
    room = torch.zeros(12, 64, device="cuda")
    for call in (lambda: g.gear_expert_combine(y.to(BF16), route, residual=x), lambda: g.gear_expert_combine(y.to(BF16), route, out=x),
                 lambda: g.gear_expert_combine(y.to(BF16), route, out_dtype=F32), lambda: g.gear_expert_combine(y, route, residual=x.to(BF16), out=x),
                 lambda: g.gear_expert_combine(y, route, residual=x.to(BF16)), lambda: g.gear_expert_combine(y, route, out=x.to(BF16)),
                 lambda: g.gear_expert_combine(y, route, residual=x, out_dtype=BF16), lambda: g.gear_expert_combine(y, route, out=x, out_dtype=BF16),
                 lambda: g.gear_expert_combine(y, route, residual=x.to(BF16), out_dtype=F32), lambda: g.gear_expert_combine(y, route, out_dtype=torch.float16),
                 lambda: g.gear_expert_combine(room[:8], route, out=room[7:9].view(BF16).view(4, 64), out_dtype=BF16)):
        with pytest.raises(g.GearError):
            call()


def test_a_layer_serves_with_one_rounding(g):
    """Integers, their products and the sum in 32 bits: the result is off by its own rounding to bf16 and by what fp32 loses."""
    rows, dim, out_dim, experts, k = 300, 136, 72, 16, 4
    r = gen(13)
    x, res = torch.randn(rows, dim, device="cuda", generator=r).to(BF16), torch.randn(rows, out_dim, device="cuda", generator=r).to(BF16)
    w = torch.randn(experts, out_dim, dim, device="cuda", generator=r) * dim ** -0.5
    route = g.gear_route(torch.randn(rows, experts, device="cuda", generator=r), k)
    y = g.gear_matmul_i8(g.gear_expert_gather_i8(x, route), g.gear_weights_i8(w), route.off, out_dtype=F32)
    out = g.gear_expert_combine(y, route, residual=res, out_dtype=BF16)
    (xq, xs), (wq, ws) = integers(x), integers(w)
    every = torch.stack([(xq * xs[:, None]) @ (wq[e] * ws[e][:, None]).t().contiguous() for e in range(experts)], 1)
    chosen = every.gather(1, route.expert.long()[:, :, None].expand(-1, -1, out_dim)) * route.weight.double()[:, :, None]
    want = res.double() + chosen.sum(1)
    # 5 u of a product (its conversion, two factors, and the factors' own roundings), (k + 2) u of the sum
    within(out, want, HALF[BF16] * want.abs() + 1.01 * (k + 7) * U * (res.double().abs() + chosen.abs().sum(1)))


@pytest.mark.parametrize("rows,n,k,experts", [(1, 72, 136, 0), (5, 1024, 4096, 0), (33, 520, 576, 16), (300, 1024, 1152, 0), (1500, 1024, 3200, 3), (4096, 2048, 128, 7)])
@pytest.mark.parametrize("x_power,w_power", [(122, -100), (122, -140), (-140, 110), (-148, 120), (-60, -60), (100, 20), (0, -149)])
def test_products_of_extreme_scales(g, rows, n, k, experts, x_power, w_power):
    """Scales that take sums times one of them out of fp32's range, while the result is an ordinary number (or one beyond the range, or next to nothing)."""
    r = gen(rows + n + k)
    e = max(1, experts)
    q = torch.randint(-127, 128, (rows, (k + 127) // 128 * 128), device="cuda", generator=r).to(torch.int8)
    q[:, k:] = 0
    w = torch.randint(-127, 128, (e, n, k), device="cuda", generator=r).to(torch.int8)
    power = lambda p, *shape: (torch.exp2(torch.rand(*shape, device="cuda", dtype=torch.float64, generator=r)) * 2.0 ** p).float()
    x_scale, w_scale = power(x_power, rows), power(w_power, e, n)
    x_scale[rows // 2], w_scale[0, n // 2] = 0.75, 0.75       # ordinary ones among them
    bounds = [0] + sorted(torch.randint(0, rows + 1, (e - 1,), generator=torch.Generator().manual_seed(rows)).tolist()) + [rows]
    off = torch.tensor(bounds, dtype=torch.int32, device="cuda") if experts else None
    rows8, weights = g.RowsI8(q, x_scale, k), g.gear_weights_i8(w, w_scale)
    for dtype in (F32, BF16):
        out = g.gear_matmul_i8(rows8, weights, off, out_dtype=dtype)
        want = torch.cat([(q[a:b, :k].double() @ w[i].double().t().contiguous()) * (x_scale[a:b, None].double() * w_scale[i].double())
                          for i, (a, b) in enumerate(zip(bounds, bounds[1:]))])
        half, least = (HALF[BF16], 2.0 ** -133) if dtype is BF16 else (0.0, 2.0 ** -149)
        most = torch.finfo(dtype).max
        edge = (want.abs() > most * (1 - 2.0 ** -6))          # may round to infinity or not
        assert torch.where(edge & (want.abs() > most * (1 + 2.0 ** -6)), out.double() == want.sign() * math.inf, True).all()
        within(torch.where(edge, 0.0, out), torch.where(edge, 0.0, want), torch.where(edge, 0.0, (3.01 * U + half) * want.abs() + least))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinite_weights_without_a_place_are_nothing(g, dtype):
    """Only a program's own weights can be infinite; at a slot without a place they add no more than any other number."""
    x = torch.randn(5, 64, device="cuda", generator=gen(2)).to(dtype)
    place = torch.tensor([[0, -1], [-1, 1], [10, 2], [-1, -1], [3, -1]], dtype=torch.int32, device="cuda")
    weight = torch.tensor([[1.0, math.inf], [-math.inf, 2.0], [math.inf, 1.0], [math.inf, -math.inf], [1.0, math.nan]], device="cuda")
    route = g.Route(place.clamp(max=0), weight, place, torch.tensor([0, 4], dtype=torch.int32, device="cuda"))
    y = torch.randn(10, 64, device="cuda", generator=gen(3)).to(dtype)
    out = g.gear_expert_combine(y, route, residual=x)
    factor = torch.tensor([1.0, 2.0, 1.0, 0.0], dtype=torch.float64, device="cuda")[:, None]
    want = x[:4].double() + factor * y[[0, 1, 2, 0]].double()
    within(out[:4], want, 4 * U * (x[:4].double().abs() + (factor * y[[0, 1, 2, 0]].double()).abs()) + HALF[dtype] * want.abs())
    assert torch.equal(out[3], x[3]) and out[4].isnan().all()


def test_results_in_the_memory_of_a_route_or_of_a_products_operands_are_refused(g):
    """Every workgroup reads places, weights and offsets, and none may find a result there."""
    def parts(room, *sizes):       # int32 words, one behind the other, each on 64 bytes
        out, at = [], 0
        for n in sizes:
            out.append(room.view(-1)[at:at + n])
            at += (n + 15) // 16 * 16
        return out
    rows, dim = 8, 64
    source = g.gear_route(torch.randn(rows, 3, device="cuda"), 2)
    x, y = torch.randn(rows, dim, device="cuda"), torch.randn(2 * rows, dim, device="cuda")

    def route_in(room):
        expert, weight, place, off = parts(room, 16, 16, 16, 4)
        for t, v in ((expert, source.expert), (weight, source.weight.view(torch.int32)), (place, source.place), (off, source.off)):
            t.copy_(v.flatten())
        return g.Route(expert.view(rows, 2), weight.view(torch.float32).view(rows, 2), place.view(rows, 2), off)
    few, many = (torch.zeros(n, dim, dtype=torch.int32, device="cuda") for n in (rows, 2 * rows))
    in_few, in_many = route_in(few), route_in(many)
    f32 = lambda t: t.view(torch.float32)
    q = g.gear_rows_i8(torch.randn(8, 64, device="cuda"))
    w = g.gear_weights_i8(torch.randn(3, 256, 64, device="cuda"))
    o = torch.empty(8 * 256, device="cuda")
    off = o[:4].view(torch.int32)
    off.copy_(torch.tensor([0, 2, 5, 8], dtype=torch.int32))
    ordinary, scale = off.clone(), o[16:24].fill_(1.0)
    few8 = g.gear_weights_i8(torch.randn(3, 8, 64, device="cuda"))
    few8.scale, few8.p_scale = o.view(-1)[:24].view(3, 8), o.data_ptr()
    wide = torch.zeros(8 * 256 * 4, dtype=torch.int8, device="cuda")
    for call in (lambda: g.gear_expert_gather(x, in_many, out=f32(many)), lambda: g.gear_expert_combine(y, in_few, out=f32(few)),
                 lambda: g.gear_expert_combine(y, in_few, weighted=False, residual=f32(few), out=f32(few)),
                 lambda: g.gear_expert_combine_backward(x, y, in_many, dy=f32(many)),
                 lambda: g.gear_expert_gather_i8(x, in_many, out=g.RowsI8(many.view(-1)[:512].view(torch.int8).view(16, 128), torch.empty(16, device="cuda"), dim)),
                 lambda: g.gear_expert_gather_i8(x, in_many, out=g.RowsI8(torch.empty(16, 128, dtype=torch.int8, device="cuda"), f32(in_many.place.flatten()), dim)),
                 lambda: g.RowsI8(wide[:1024].view(8, 128), wide[512:544].view(torch.float32), 64),
                 lambda: g.gear_matmul_i8(q, w, off, out=o.view(8, 256)),
                 lambda: g.gear_matmul_i8(g.RowsI8(q.q, scale, 64), w, ordinary, out=o.view(8, 256)),
                 lambda: g.gear_matmul_i8(g.RowsI8(wide[:1024].view(8, 128), q.scale, 64), w, ordinary, out=wide.view(torch.float32).view(8, 256)),
                 lambda: g.gear_matmul_i8(q, w, ordinary, out=o.view(8, 256), status=o[40:41].view(torch.int32)),
                 lambda: g.gear_matmul_i8(q, w, ordinary, out=w.packed.view(torch.float32)[:8 * 256].view(8, 256)),
                 lambda: g.gear_matmul_i8(q, few8, ordinary, out=o[16:80].view(8, 8))):
        with pytest.raises(g.GearError):
            call()
    # beside each other they are fine
    room = torch.zeros(8, 512, device="cuda")
    assert torch.equal(g.gear_matmul_i8(q, w, ordinary, out=room[:, 256:]), g.gear_matmul_i8(q, w, ordinary, out_dtype=F32))
    out = torch.zeros(2 * rows + 2, dim, dtype=torch.int32, device="cuda")
    beside = route_in(out[2 * rows:])
    assert torch.equal(g.gear_expert_gather(x, beside, out=f32(out[:2 * rows])), g.gear_expert_gather(x, source))


@pytest.mark.parametrize("experts,n,k", [(1, 8, 8), (1, 264, 4104), (3, 72, 136), (16, 520, 576)])
def test_weights_in_bf16(g, experts, n, k):
    """Weights of that type are the integers nearest to them, and nothing is rounded twice."""
    r = gen(n + k)
    w = (torch.randn(experts, n, k, device="cuda", generator=r) * torch.exp(torch.randn(experts, n, 1, device="cuda", generator=r))).to(BF16)
    w[0, 1], w[-1, 2, k // 2], w[-1, 3, 0] = 0.0, math.inf, math.nan
    x = torch.randn(70, k, device="cuda", generator=r)
    b = [round(70 * i / experts) for i in range(experts + 1)]
    q, weights = g.gear_rows_i8(x), g.gear_weights_i8(w)
    wq, ws = integers(w)
    within(weights.scale, ws, U * ws.nan_to_num())
    same = g.gear_weights_i8(w.float())
    assert torch.equal(same.scale.nan_to_num(), weights.scale.nan_to_num())
    off = torch.tensor(b, dtype=torch.int32, device="cuda")
    out = g.gear_matmul_i8(q, weights, off, out_dtype=F32)
    want = torch.cat([q.q[b[i]:b[i + 1], :k].double() @ wq[i].t().contiguous() * weights.scale[i].double() for i in range(experts)]) * q.scale[:, None].double()
    within(out, want, 3.01 * U * want.nan_to_num().abs())
    assert torch.equal(out.nan_to_num(), g.gear_matmul_i8(q, same, off, out_dtype=F32).nan_to_num())
