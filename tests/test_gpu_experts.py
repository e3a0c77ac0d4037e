"""The operators of a Dense Part made of experts (norm, 8-bit products, products grouped by expert, clipping) against plain
evaluations in 64 bits, at the sizes and values where they can go wrong.

Tolerances.  u = 2^-24 is the rounding error of fp32 (24 significant bits), 2^-8 of bf16 (8 of them).  A sum of n terms in fp32 is off by at most n u times the sum
of the terms' magnitudes whatever its order, and products of bf16 or 8-bit operands are exact in fp32, so a product over k
is held to (k + 8) 2u sum |a| |b| (twice, as the matrix instruction need not round to nearest inside), plus one rounding of
the result.  In 8 bits the instruction adds eight neighbouring products at once, and keeps of each what is at least 2^-13 of
the largest one's power of two: up to eight units of that for every eight products come on top.  The norm's factor comes from a sum of squares, all positive: (dim + 8) u relative for the sum in the worst
order; rows are summed by at least 64 threads and then in a tree, (dim / 64 + 16) u, halved by the square root."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def g():
    import paper_1806_03925_amd as g
    return g


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(t, pad, fill=math.nan):
    """The same matrix with `pad` columns of `fill` between its rows."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=torch.float32, device="cuda").to(t.dtype)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def within(got, want, bound):
    """Every element within its bound of `want`; NaN and infinities in the same places."""
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)) and torch.equal(torch.isnan(want), torch.isnan(got))
    assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()])
    bound = bound.expand_as(want) if torch.is_tensor(bound) else torch.full_like(want, bound)
    off = ((got - want).abs() - bound)[fine]
    assert off.numel() == 0 or off.max() <= 0, (off.max().item(), int((off > 0).sum()))


# ---- 8 bits, from the definition -----------------------------------------------------------------------------------
def exponents(v):
    """v [rows x dim] (64 bits) -> exponents [rows x blocks], found by search over the definition."""
    b = torch.nn.functional.pad(v, (0, -v.shape[1] % 128)).view(v.shape[0], -1, 128)
    top = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax(-1)
    e = torch.full_like(top, 128)
    for k in range(128, -128, -1):
        e = torch.where(top <= 448.0 * 2.0 ** k, torch.full_like(top, k), e)
    return torch.where(top == 0, torch.zeros_like(e), e).to(torch.int64)


def grid8():
    """All values of e4m3 that are not negative, ascending, from its definition."""
    small = [f * 2.0 ** -9 for f in range(8)]
    return torch.tensor(small + [(8 + f) * 2.0 ** (e - 10) for e in range(1, 16) for f in range(8) if (e, f) != (15, 7)],
                        dtype=torch.float64, device="cuda")


def nearest8(z):
    """The e4m3 values nearest to z (64 bits, |z| <= 448), ties to the even fraction."""
    grid = grid8()
    at = torch.searchsorted(grid, z.abs().contiguous()).clamp(1, len(grid) - 1)
    lo, hi = grid[at - 1], grid[at]
    down = (z.abs() - lo < hi - z.abs()) | ((z.abs() - lo == hi - z.abs()) & ((at - 1) % 2 == 0))
    return torch.where(down, lo, hi) * torch.sign(z)


def values8(rows8):
    rows = rows8.q.shape[0]
    e = rows8.scale[:, :rows8.q.shape[1] // 128].double() - 127
    return (rows8.q.view(torch.float8_e4m3fn).double().view(rows, -1, 128) * torch.exp2(e).unsqueeze(-1)).flatten(1)


def weights8(w):
    """[experts x N x K] -> what its 8-bit form stands for, in 64 bits."""
    experts, n, k = w.shape
    p = torch.nn.functional.pad(w.double(), (0, -k % 128, 0, -n % 128))
    b = p.view(experts, p.shape[1] // 128, 128, p.shape[2] // 128, 128).transpose(2, 3).reshape(-1, 128 * 128)
    top = b.abs().amax(1, keepdim=True)
    unit = torch.exp2(exponents(top).double())
    v = nearest8(b / unit) * unit
    return v.view(experts, p.shape[1] // 128, p.shape[2] // 128, 128, 128).transpose(2, 3).reshape(p.shape)[:, :n, :k]


# ---- norm -----------------------------------------------------------------------------------------------------------
NORM_SHAPES = [(1, 8), (3, 72), (5, 512), (6, 520), (9, 1024), (2, 1152), (65, 2048), (3, 2056), (2, 4104), (2, 8192), (1, 8200),
               (1, 33000), (2, 65536)]


def norm_ref(x, residual, gain, eps):
    h = x.double() + (0 if residual is None else residual.double())
    return h, h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * gain.double()


def norm_bound(dim, dtype):
    return (dim / 64 + 24) * U + HALF[dtype]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
def test_norm(g, dtype, rows, dim):
    r = gen(rows * 7 + dim)
    x = (torch.randn(rows, dim, device="cuda", generator=r) * 3).to(dtype)
    res = torch.randn(rows, dim, device="cuda", generator=r).to(dtype)
    gain = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r)
    if rows > 2:
        x[1], res[1] = 0, 0                                  # a row of zeros stays one
    for residual, xx in ((None, x), (res, x), (res, strided(x, 8))):
        h, y = norm_ref(x, residual, gain, 1e-6)
        out = g.gear_rmsnorm(xx, gain, 1e-6, residual=residual)
        assert out.rows8 is None and (out.sum is None) == (residual is None)
        within(out.y, y, norm_bound(dim, dtype) * y.abs())
        if residual is not None:
            within(out.sum, h, HALF[dtype] * h.abs())
    # the sum in the residual's place, the norm in x's, rows apart
    place, y_place = strided(res, 16), strided(x, 24)
    g.gear_rmsnorm(y_place, gain, 1e-6, residual=place, out=g.NormOutput(place, y_place, None))
    assert torch.equal(place, out.sum) and torch.equal(y_place, out.y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(1, 8), (5, 136), (70, 1152), (3, 2048), (4, 4104), (2, 9000)])
def test_norm_in_8_bits(g, dtype, rows, dim):
    r = gen(rows + dim)
    x = (torch.randn(rows, dim, device="cuda", generator=r) * torch.exp(3 * torch.randn(rows, dim, device="cuda", generator=r))).to(dtype)
    gain = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r)
    _, y = norm_ref(x, None, gain, 1e-6)
    out = g.gear_rmsnorm(x, gain, 1e-6, q8=True)
    q = out.rows8
    wide = torch.nn.functional.pad(y, (0, -dim % 128))
    assert (q.q.view(torch.uint8)[:, dim:] == 0).all()
    e = q.scale[:, :wide.shape[1] // 128].long() - 127
    top = wide.view(rows, -1, 128).abs().amax(-1)
    near = (top / 448 / torch.exp2(torch.round(torch.log2(top.clamp_min(1e-300) / 448))) - 1).abs() < 2 * norm_bound(dim, F32)
    assert (e == exponents(y))[~near].all() and ((e - exponents(y)).abs() <= 1).all()
    unit = torch.exp2(e.double()).repeat_interleave(128, 1)
    # half of the last fraction bit, or of the smallest step, and what the norm itself may be off
    bound = torch.maximum(2.0 ** -4 * wide.abs(), 2.0 ** -10 * unit) * (1 + 2.0 ** -3) + norm_bound(dim, F32) * wide.abs()
    within(values8(q), wide, bound)
    within(out.y, values8(q)[:, :dim], 0.0)                 # y stands for the same values: bf16 and fp32 hold them exactly
    alone = g.gear_rmsnorm(x, gain, 1e-6, y=False, q8=True)
    assert alone.y is None and torch.equal(alone.rows8.q.view(torch.uint8), q.q.view(torch.uint8)) and torch.equal(alone.rows8.scale, q.scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [8, 120, 128, 136, 520, 1152, 4096, 12000])
def test_rows_in_8_bits_are_the_nearest_values(g, dtype, dim):
    """Bit for bit: values of all sizes, ties, blocks at the edge of a scale, the smallest and largest numbers there are."""
    r = gen(dim)
    x = torch.randn(12, dim, device="cuda", generator=r) * torch.exp(2 * torch.randn(12, dim, device="cuda", generator=r))
    x[1] = 0
    x[2] = (torch.randint(0, 1000, (dim,), device="cuda", generator=r).float() - 500) / 2       # ties
    x[3] *= 1e-40                                                                                # below the smallest normal number
    x[4] *= 1e36
    x[5, 0] = 448.0
    x[6, 0] = 449.0 if dtype is F32 else 450.0
    x[7] = 3.0e38
    x[8, 3], x[8, 4], x[8, 5] = math.inf, -math.inf, math.nan
    x[9] = math.nan
    x = x.to(dtype)
    q = g.gear_rows8(strided(x, 8))
    v = torch.nn.functional.pad(x.double(), (0, -dim % 128))
    e = exponents(x.double())
    assert torch.equal(q.scale[:, :e.shape[1]].long() - 127, e)
    unit = torch.exp2(e.double()).repeat_interleave(128, 1)
    fine = torch.isfinite(v)
    want = torch.where(fine, nearest8(torch.where(fine, v / unit, torch.zeros_like(v))), torch.full_like(v, math.nan))
    within(q.q.view(torch.float8_e4m3fn).double(), want, 0.0)


def test_norm_with_infinities_and_nan_stays_in_its_row(g):
    x = torch.randn(4, 1152, device="cuda", generator=gen(1))
    clean = g.gear_rmsnorm(x, torch.ones(1152, device="cuda"), 1e-6, q8=True)
    x[1, 7], x[2, 9] = math.inf, math.nan
    out = g.gear_rmsnorm(x, torch.ones(1152, device="cuda"), 1e-6, q8=True)
    for row in (0, 3):
        assert torch.equal(out.y[row], clean.y[row]) and torch.equal(out.rows8.scale[row], clean.rows8.scale[row])
    assert out.y[1, 7].isnan() and (out.y[1, 128:] == 0).all() and out.y[2].isnan().all()


def norm_back_ref(h, gain, dy, eps, dsum=None):
    h, dy, gain = h.double(), dy.double(), gain.double()
    s = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    a = dy * gain
    dx = s * a - h * s ** 3 * (a * h).mean(1, keepdim=True) + (0 if dsum is None else dsum.double())
    terms = dy * h * s
    scale = (s * a).abs() + h.abs() * s ** 3 * (a * h).abs().mean(1, keepdim=True) + (0 if dsum is None else dsum.double().abs())
    return dx, terms.sum(0), scale, terms.abs().sum(0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", NORM_SHAPES + [(1023, 72), (4100, 512), (5000, 264), (1500, 2056)])
def test_norm_backward(g, dtype, rows, dim):
    r = gen(rows * 3 + dim)
    draw = lambda: torch.randn(rows, dim, device="cuda", generator=r).to(dtype)
    h, dy, dsum = draw() * 2, draw(), draw()
    if rows > 2:
        h[1] = 0
    gain = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r)
    for more in (None, dsum):
        dx, dgain, scale, total = norm_back_ref(h, gain, dy, 1e-5, more)
        got, got_gain = g.gear_rmsnorm_backward(strided(h, 8), gain, strided(dy, 16), 1e-5, dsum=more)
        within(got, dx, 4 * norm_bound(dim, F32) * scale + HALF[dtype] * dx.abs())
        within(got_gain, dgain, (norm_bound(dim, F32) + (rows + 8) * U) * total)
    again, again_gain = g.gear_rmsnorm_backward(h, gain, dy, 1e-5, dsum=dsum)
    assert torch.equal(again, got) and torch.equal(again_gain, got_gain)
    g.gear_rmsnorm_backward(h, gain, dy, 1e-5, dsum=dsum, dx=dsum)     # in the place of what flows in
    assert torch.equal(dsum, got)


def test_norm_backward_against_differences(g):
    """d/dt of sum(y * dy) along a direction, central differences in 64 bits: error t^2 / 6 times a third derivative of
    order one relative, at t = 1e-4, far below the kernel's own bound."""
    r = gen(5)
    h, dy, v = (torch.randn(7, 264, device="cuda", generator=r) for _ in range(3))
    gain, vg = 1 + 0.3 * torch.randn(264, device="cuda", generator=r), torch.randn(264, device="cuda", generator=r)
    dx, dgain = g.gear_rmsnorm_backward(h, gain, dy, 1e-5)
    loss = lambda a, b: (norm_ref(a, None, b, 1e-5)[1] * dy.double()).sum().item()
    t = 1e-4
    along_h = (loss(h.double() + t * v, gain) - loss(h.double() - t * v, gain)) / (2 * t)
    along_gain = (loss(h, gain.double() + t * vg) - loss(h, gain.double() - t * vg)) / (2 * t)
    assert abs((dx.double() * v).sum().item() - along_h) < 1e-5 * (dx.double() * v).abs().sum().item()
    assert abs((dgain.double() * vg).sum().item() - along_gain) < 1e-5 * (dgain.double() * vg).abs().sum().item()


def test_norm_of_no_rows(g):
    x = torch.empty(0, 72, device="cuda")
    out = g.gear_rmsnorm(x, torch.ones(72, device="cuda"), 1e-6, q8=True)
    assert out.y.shape == (0, 72) and out.rows8.q.shape == (0, 128)
    dx, dgain = g.gear_rmsnorm_backward(x, torch.ones(72, device="cuda"), x, 1e-6, dgain=torch.full((72,), 3.0, device="cuda"))
    assert dx.shape == (0, 72) and (dgain == 0).all()


# ---- products grouped by expert ---------------------------------------------------------------------------------------
SIZES = [[1], [0], [130], [5, 0, 1], [0, 0, 0], [127, 1, 128, 0, 129], [300, 3, 64, 65], [0, 33, 0, 0, 700], [40] * 70]


def offsets(sizes):
    return torch.tensor([0] + sizes).cumsum(0).to(torch.int32).cuda()


def operands(dtype, sizes, n, k, extra=0):
    r = gen(sum(sizes) * 13 + n * 5 + k)
    rows = sum(sizes) + extra
    draw = lambda *s: torch.randn(s, device="cuda", generator=r).to(dtype)
    return draw(rows, k), draw(rows, n), draw(len(sizes), n, k)


def grouped(a, w, sizes):
    """a rows times w_e^T and the sums of magnitudes, 64 bits."""
    out = torch.zeros(a.shape[0], w.shape[1], dtype=torch.float64, device="cuda")
    mag, at = out.clone(), 0
    for e, n in enumerate(sizes):
        rows, we = a[at:at + n].double(), w[e].double()
        out[at:at + n], mag[at:at + n] = rows @ we.t().contiguous(), rows.abs() @ we.abs().t().contiguous()
        at += n
    return out, mag


def units8(a, w):
    """8 * 2^-13 times the largest of every eight neighbouring products, summed: what 8-bit products may lose besides."""
    a, w = a.abs(), w.abs()
    total = torch.zeros(a.shape[0], w.shape[0], dtype=torch.float64, device="cuda")
    for at in range(0, a.shape[1], 8):
        total += (a[:, None, at:at + 8] * w[None, :, at:at + 8]).amax(-1)
    return total * 2.0 ** -10


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k", [(8, 8), (72, 320), (136, 40), (264, 72), (520, 136)])
@pytest.mark.parametrize("sizes", SIZES)
def test_expert_products(g, dtype, sizes, n, k):
    x, dy, w = operands(dtype, sizes, n, k, extra=3)       # three rows that are nobody's
    off, used = offsets(sizes), sum(sizes)
    x[used:], dy[used:] = math.nan, math.nan
    weights = g.ExpertWeights(w)
    want, mag = grouped(x[:used], w, sizes)
    out = torch.full((used + 3, n + 8), 7.0, device="cuda").to(dtype)
    g.gear_expert_matmul(strided(x, 8), weights, off, out=out[:, :n])
    within(out[:used, :n], want, (k + 8) * 2 * U * mag + HALF[dtype] * want.abs())
    assert (out[used:] == 7).all() and (out[:, n:] == 7).all()
    if dtype is BF16:
        got = g.gear_expert_matmul(x, weights, off, out_dtype=F32)
        within(got[:used], want, (k + 8) * 2 * U * mag)
    want, mag = grouped(dy[:used], w.transpose(1, 2).contiguous(), sizes)
    within(g.gear_expert_dgrad(strided(dy, 16), weights, off)[:used], want, (n + 8) * 2 * U * mag + HALF[dtype] * want.abs())
    dw = g.gear_expert_wgrad(strided(dy, 8), strided(x, 16), off, dw=torch.full((len(sizes), n, k), math.nan, device="cuda"))
    at = 0
    for e, m in enumerate(sizes):
        a, b = dy[at:at + m].double(), x[at:at + m].double()
        within(dw[e], a.t().contiguous() @ b, (m + 8) * 2 * U * (a.abs().t().contiguous() @ b.abs()))
        at += m


@pytest.mark.parametrize("n,k", [(8, 8), (72, 128), (136, 136), (264, 520), (520, 1152)])
@pytest.mark.parametrize("sizes", SIZES)
def test_products_in_8_bits(g, sizes, n, k):
    x, _, w = operands(BF16, sizes, n, k, extra=3)
    off, used = offsets(sizes), sum(sizes)
    x[used:] = math.nan
    if used > 2:
        x[1] = 0
    rows, weights = g.gear_rows8(x), g.gear_weights8(w)
    a, b = values8(rows)[:used, :k], weights8(w)
    want, mag = grouped(a, b, sizes)
    at = [0, *torch.tensor(sizes).cumsum(0).tolist()]
    lost = torch.cat([units8(a[i:j], b[e]) for e, (i, j) in enumerate(zip(at, at[1:]))])
    out = torch.full((used + 3, n + 8), 7.0, device="cuda", dtype=BF16)
    g.gear_matmul8(rows, weights, off, out=out[:, :n])
    within(out[:used, :n], want, lost + (k + 8) * 2 * U * mag + HALF[BF16] * (want.abs() + lost))
    assert (out[used:] == 7).all() and (out[:, n:] == 7).all()
    got = g.gear_matmul8(rows, weights, off, out_dtype=F32)
    within(got[:used], want, lost + (k + 8) * 2 * U * mag)
    if len(sizes) == 1:
        assert torch.equal(g.gear_matmul8(g.Rows8(rows.q[:used], rows.scale[:used], k), weights), out[:used, :n])


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("rows,n,k", [(1, 1024, 1152), (2, 4096, 4096), (17, 520, 8192), (33, 264, 1024), (257, 1024, 576),
                                      (1025, 2048, 264), (4096, 1152, 1024), (20000, 256, 72)])
def test_products_of_one_layer(g, kind, rows, n, k):
    """One expert without offsets, from a single row to thousands: every shape of tile."""
    r = gen(rows + n + k)
    dtype = F32 if kind == "f32" else BF16
    x, w = torch.randn(rows, k, device="cuda", generator=r).to(dtype), torch.randn(n, k, device="cuda", generator=r).to(dtype)
    if kind == "e4m3":
        x *= torch.exp(torch.randn(rows, 1, device="cuda", generator=r)).to(dtype)
        q = g.gear_rows8(x)
        got = g.gear_matmul8(q, g.gear_weights8(w), out_dtype=F32)
        a, b = values8(q)[:, :k], weights8(w[None])[0]
        lost = units8(a, b)
    else:
        got = g.gear_expert_matmul(x, g.ExpertWeights(w, backward=False), out_dtype=F32)
        a, b, lost = x.double(), w.double(), 0.0
    within(got, a @ b.t().contiguous(), lost + (k + 8) * 2 * U * (a.abs() @ b.abs().t().contiguous()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,k", [(1, 264, 136), (4099, 136, 264), (16385, 320, 72), (9000, 1024, 512)])
def test_weight_gradient_of_one_layer(g, dtype, rows, n, k):
    """Long contractions over the rows; twice the same bits."""
    x, dy, _ = operands(dtype, [rows], n, k)
    got = g.gear_expert_wgrad(dy, x)
    a, b = dy.double(), x.double()
    within(got[0], a.t().contiguous() @ b, (rows + 8) * 2 * U * (a.abs().t().contiguous() @ b.abs()))
    assert torch.equal(got, g.gear_expert_wgrad(dy, x))


@pytest.mark.parametrize("sizes", [[6000, 1, 0, 2500], [0] * 900 + [3] * 100, [1] * 1024])
def test_uneven_and_many_experts(g, sizes):
    x, dy, w = operands(BF16, sizes, 136, 72)
    off = offsets(sizes)
    want, mag = grouped(x, w, sizes)
    within(g.gear_expert_matmul(x, g.ExpertWeights(w), off, out_dtype=F32), want, 80 * 2 * U * mag)
    dw = g.gear_expert_wgrad(dy, x, off)
    at = 0
    for e, m in enumerate(sizes):
        if m and e % 37 in (0, 1, 2):
            a, b = dy[at:at + m].double(), x[at:at + m].double()
            within(dw[e], a.t().contiguous() @ b, (m + 8) * 2 * U * (a.abs().t().contiguous() @ b.abs()))
        elif not m:
            assert (dw[e] == 0).all()
        at += m


def test_nan_stays_in_its_row_and_expert(g):
    sizes = [70, 60]
    x, dy, w = operands(BF16, sizes, 72, 200)
    off = offsets(sizes)
    clean = g.gear_matmul8(g.gear_rows8(x), g.gear_weights8(w), off)
    x[69, 5] = math.inf
    got = g.gear_matmul8(g.gear_rows8(x), g.gear_weights8(w), off)
    assert got[69].isnan().all() and torch.equal(got[:69], clean[:69]) and torch.equal(got[70:], clean[70:])
    dw = g.gear_expert_wgrad(dy, x, off)
    assert not torch.isfinite(dw[0, :, 5]).any() and torch.isfinite(dw[0, :, 6:]).all() and torch.isfinite(dw[1]).all()


def test_large_and_small_scales(g):
    """Scales far from one, on both sides: products of 2^100 and 2^-100 and back."""
    r = gen(3)
    x, w = torch.randn(40, 264, device="cuda", generator=r), torch.randn(1, 72, 264, device="cuda", generator=r)
    base = g.gear_matmul8(g.gear_rows8(x), g.gear_weights8(w), out_dtype=F32)
    for p in (-100.0, 90.0):
        got = g.gear_matmul8(g.gear_rows8(x * 2.0 ** p), g.gear_weights8(w * 2.0 ** -p), out_dtype=F32)
        assert torch.equal(got, base)


@pytest.mark.parametrize("off", [[1, 40, 100], [0, 60, 50], [0, 50, 101], [0, -1, 100], [0, 2 ** 31 - 1, 100]])
def test_offsets_that_are_no_list_of_rows(g, off):
    x, dy, w = operands(BF16, [50, 50], 72, 64)
    off = torch.tensor(off, dtype=torch.int64).to(torch.int32).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = [lambda out: g.gear_expert_matmul(x, g.ExpertWeights(w), off, out=out, status=status),
             lambda out: g.gear_matmul8(g.gear_rows8(x), g.gear_weights8(w), off, out=out, status=status)]
    for call in calls:
        out = torch.full((100, 72), 7.0, device="cuda", dtype=BF16)
        status.zero_()
        call(out)
        assert status.item() == g.GEAR_ERR_RANGE and (out == 7).all()
    dw = torch.full((2, 72, 64), 7.0, device="cuda")
    status.zero_()
    g.gear_expert_wgrad(dy, x, off, dw=dw, status=status)
    assert status.item() == g.GEAR_ERR_RANGE and (dw == 7).all()
    good = offsets([50, 50])
    g.gear_expert_wgrad(dy, x, good, dw=dw, status=status)
    assert status.item() == 0


def test_gradients_against_differences(g):
    """sum(Y * G) is linear in X and in W: differences of any width are exact but for rounding."""
    sizes = [9, 0, 30]
    x, G, w = operands(F32, sizes, 72, 40)
    off = offsets(sizes)
    dx, dw = g.gear_expert_dgrad(G, g.ExpertWeights(w), off), g.gear_expert_wgrad(G, x, off)
    loss = lambda a, b: (grouped(a, b, sizes)[0] * G.double()).sum().item()
    vx, _, vw = operands(F32, sizes, 72, 40)
    vx, vw = vx.flip(0), vw.flip(0)
    along = (loss(x.double() + vx, w) - loss(x.double() - vx, w)) / 2
    assert abs((dx.double() * vx).sum().item() - along) < 80 * 2 * U * (dx.double() * vx).abs().sum().item() * 8
    along = (loss(x, w.double() + vw) - loss(x, w.double() - vw)) / 2
    assert abs((dw.double() * vw).sum().item() - along) < 80 * 2 * U * (dw.double() * vw).abs().sum().item() * 8


def test_master_weights_are_rounded_once(g):
    """fp32 weights laid out as bf16 give the bits of weights rounded to bf16 before; update() replaces them."""
    x, dy, w = operands(F32, [30, 20], 72, 136)
    off = offsets([30, 20])
    a, b = g.ExpertWeights(w, operand=BF16), g.ExpertWeights(w.to(BF16))
    assert torch.equal(g.gear_expert_matmul(x.to(BF16), a, off), g.gear_expert_matmul(x.to(BF16), b, off))
    assert torch.equal(g.gear_expert_dgrad(dy.to(BF16), a, off), g.gear_expert_dgrad(dy.to(BF16), b, off))
    b.update(2 * w.to(BF16))
    assert torch.equal(g.gear_expert_matmul(x.to(BF16), b, off), 2 * g.gear_expert_matmul(x.to(BF16), a, off))


# ---- long lists of rows -------------------------------------------------------------------------------------------------
def test_rows_beyond_32_bits_of_offset(g):
    rows = 2 ** 31 // 2048 + 300                             # more than 2^31 elements, and 2^32 bytes, of 2048 columns
    x = torch.zeros(rows, 2048, dtype=BF16, device="cuda")
    tail = torch.randn(200, 2048, device="cuda", generator=gen(9)).to(BF16)
    x[-200:] = tail
    gain = torch.ones(2048, device="cuda")
    small, large = g.gear_rmsnorm(tail, gain, 1e-6, q8=True), g.gear_rmsnorm(x, gain, 1e-6, q8=True)
    assert torch.equal(large.y[-200:], small.y) and (large.y[:5] == 0).all()
    w8 = g.gear_weights8(torch.randn(8, 2048, device="cuda", generator=gen(10)))
    assert torch.equal(g.gear_matmul8(large.rows8, w8)[-200:], g.gear_matmul8(small.rows8, w8))
    dx, _ = g.gear_rmsnorm_backward(x, gain, large.y, 1e-6)
    assert torch.equal(dx[-200:], g.gear_rmsnorm_backward(tail, gain, small.y, 1e-6)[0])
    w = g.ExpertWeights(torch.randn(2, 8, 2048, device="cuda", generator=gen(11)).to(BF16))
    off = torch.tensor([0, rows - 200, rows], dtype=torch.int32, device="cuda")
    dw = g.gear_expert_wgrad(x[:, :8].contiguous(), x, off)
    assert (dw[0] == 0).all() and torch.equal(dw[1], g.gear_expert_wgrad(tail[:, :8].contiguous(), tail)[0])
    wide = g.gear_expert_dgrad(x[:, :8].contiguous(), w, off)
    assert torch.equal(wide[-200:], g.gear_expert_dgrad(tail[:, :8].contiguous(), g.ExpertWeights(torch.randn(2, 8, 2048, device="cuda",
                       generator=gen(11))[1].to(BF16).contiguous())))


# ---- norm of gradients, clipping ----------------------------------------------------------------------------------------
def grad_list(lengths, kinds, seed, scale=1.0):
    r = gen(seed)
    flat = {k: (torch.randn(sum(lengths) + 8, device="cuda", generator=r) * scale).to(k) for k in (F32, BF16)}
    out, at = [], {F32: 1, BF16: 3}                          # no gradient begins where a vector does
    for n, k in zip(lengths, kinds):
        out.append(flat[k][at[k]:at[k] + n])
        at[k] += n
    return out


@pytest.mark.parametrize("lengths", [[1], [0, 5, 0], [6144, 64, 64, 1], [16384, 16383, 16385, 7, 40000], [3] * 500, [2_000_003, 17, 0, 999_999]])
@pytest.mark.parametrize("mix", [(F32,), (BF16,), (F32, BF16, BF16)])
def test_clipping(g, lengths, mix):
    kinds = [mix[i % len(mix)] for i in range(len(lengths))]
    grads = grad_list(lengths, kinds, sum(lengths))
    before = [t.clone() for t in grads]
    norm = math.sqrt(sum(t.double().square().sum().item() for t in grads))
    shifted = grad_list(lengths, kinds, 1)                  # other memory, which lies differently to 16 bytes
    shifted = [torch.cat([t.new_zeros(2), t])[2:] if t.numel() else t for t in shifted]
    for limit in (norm / 3, 0.9 * norm, 2 * norm + 1):
        c = min(1.0, limit / (norm + 1e-6))
        got = g.gear_clip_grads(g.GradList(grads, shifted), limit)
        assert abs(got.item() - norm) <= 2 * U * norm
        for t, o, k in zip(before, shifted, kinds):
            within(o, t.double() * c, (4 * U + HALF[k]) * c * t.double().abs())
            if limit > norm:
                assert torch.equal(o, t)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    assert g.gear_grad_norm(g.GradList(grads)).item() == got.item()
    inplace = g.GradList(grads)
    g.gear_clip_grads(inplace, 2 * norm + 1)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    g.gear_clip_grads(inplace, norm / 2)
    if norm > 1e-3:
        assert abs(g.gear_grad_norm(inplace).item() - norm / 2) <= 2.0 ** -8 * norm


def test_clipping_of_extreme_gradients(g):
    huge = [torch.full((1000,), 1e30, device="cuda"), torch.full((3,), 1e38, device="cuda", dtype=BF16)]
    norm = math.sqrt(sum(t.double().square().sum().item() for t in huge))
    assert abs(g.gear_clip_grads(g.GradList(huge), 1.0).item() / norm - 1) < 4 * U
    assert abs(math.sqrt(sum(t.double().square().sum().item() for t in huge)) - 1) < 2.0 ** -8
    tiny = [torch.full((1000,), 1e-30, device="cuda")]
    assert abs(g.gear_grad_norm(g.GradList(tiny)).item() / math.sqrt(1000 * 1e-60) - 1) < 1e-6
    a, b = torch.ones(20, device="cuda"), torch.ones(5, device="cuda", dtype=BF16)
    a[3] = math.inf
    assert g.gear_clip_grads(g.GradList([a, b]), 1.0).item() == math.inf
    assert (b == 0).all() and a[3].isnan() and (a[4:] == 0).all()
    b[2] = math.nan
    assert math.isnan(g.gear_clip_grads(g.GradList([b]), 1.0).item()) and b.isnan().all()


# ---- streams, graphs, refusals --------------------------------------------------------------------------------------------
def layer_step(g, x, res, gain, w, off, dy, grads):
    h, y, _ = g.gear_rmsnorm(x, gain, 1e-6, residual=res)
    weights = g.ExpertWeights(w)
    out = g.gear_expert_matmul(y, weights, off)
    dyy = g.gear_expert_dgrad(dy, weights, off)
    dw = g.gear_expert_wgrad(dy, y, off)
    dx, dgain = g.gear_rmsnorm_backward(h, gain, dyy, 1e-6, dsum=dyy)
    q = g.gear_rmsnorm(x, gain, 1e-6, residual=res, y=False, q8=True).rows8
    served = g.gear_matmul8(q, g.gear_weights8(w), off)
    norm = g.gear_clip_grads(grads, 0.5)
    return [h, out, dx, dgain, dw, served, norm, *grads.out]


def test_on_another_stream_and_in_a_graph(g):
    sizes = [100, 0, 157]
    x, dy, w = operands(BF16, sizes, 136, 136)
    res, gain, off = torch.randn_like(x), torch.ones(136, device="cuda"), offsets(sizes)
    src = [torch.randn(300, device="cuda"), torch.randn(77, device="cuda").to(BF16)]
    grads = g.GradList(src, [torch.empty_like(t) for t in src])
    want = [t.clone() for t in layer_step(g, x, res, gain, w, off, dy, grads)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer_step(g, x, res, gain, w, off, dy, grads)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer_step(g, x, res, gain, w, off, dy, grads)
    for _ in range(3):
        for t in out:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
        layer_step(g, x.flip(0).contiguous(), res, gain, w, off, dy, g.GradList(src, [torch.empty_like(t) for t in src]))


def test_refusals(g):
    x, gain = torch.randn(4, 72, device="cuda"), torch.ones(72, device="cuda")
    w = torch.randn(2, 64, 72, device="cuda")
    off = offsets([2, 2])
    weights, w8 = g.ExpertWeights(w), g.gear_weights8(w)
    q = g.gear_rows8(x)
    bad = [
        lambda: g.gear_rmsnorm(x.cpu(), gain, 1e-6),
        lambda: g.gear_rmsnorm(x.half(), gain, 1e-6),
        lambda: g.gear_rmsnorm(x[:, :70].contiguous(), gain[:70].contiguous(), 1e-6),                # 70 columns
        lambda: g.gear_rmsnorm(torch.randn(4, 77, device="cuda")[:, :72], gain, 1e-6),              # rows 77 apart
        lambda: g.gear_rmsnorm(torch.randn(4, 80, device="cuda")[:, 1:73], gain, 1e-6),             # begins on 4 bytes
        lambda: g.gear_rmsnorm(x, gain[:64].contiguous(), 1e-6),
        lambda: g.gear_rmsnorm(x, gain, -1.0),
        lambda: g.gear_rmsnorm(x, gain, math.nan),
        lambda: g.gear_rmsnorm(x, gain, 1e-6, residual=x.to(BF16)),
        lambda: g.gear_rmsnorm(x, gain, 1e-6, residual=x[:2]),
        lambda: g.gear_rmsnorm(x, gain, 1e-6, y=False),                                              # nothing asked for
        lambda: g.gear_rmsnorm(x, gain, 1e-6, residual=x, out=g.NormOutput(x, x, None)),             # two results in one place
        lambda: g.gear_rmsnorm(torch.randn(72, 4, device="cuda").t(), gain, 1e-6),                   # columns apart
        lambda: g.gear_rmsnorm_backward(x, gain, x[:3], 1e-6),
        lambda: g.gear_rmsnorm_backward(x, gain, x, math.inf),
        lambda: g.gear_weights8(w.transpose(1, 2)),
        lambda: g.gear_weights8(torch.randn(64, 70, device="cuda")),
        lambda: g.ExpertWeights(w, operand=torch.float16),
        lambda: g.gear_expert_matmul(x, weights),                                                    # two experts, no offsets
        lambda: g.gear_expert_matmul(x, weights, off.long()),
        lambda: g.gear_expert_matmul(x, weights, off[:2].contiguous()),
        lambda: g.gear_expert_matmul(x.to(BF16), weights, off),
        lambda: g.gear_expert_matmul(x, weights, off, out=torch.empty(4, 64, device="cuda", dtype=BF16)),   # fp32 products stay fp32
        lambda: g.gear_expert_matmul(x, weights, off, out=torch.empty(3, 64, device="cuda")),
        lambda: g.gear_expert_matmul(x[:, :64].contiguous(), weights, off),
        lambda: g.gear_expert_dgrad(x[:, :64].contiguous(), g.ExpertWeights(w, backward=False), off),
        lambda: g.gear_expert_wgrad(x[:3], x, off),
        lambda: g.gear_matmul8(g.Rows8(q.q, q.scale, 136), w8, off),
        lambda: g.gear_matmul8(g.Rows8(q.q[:, :64], q.scale, 72), w8, off),
        lambda: g.gear_matmul8(g.gear_rows8(torch.randn(4, 64, device="cuda")), w8, off),
        lambda: weights.update(w[:1].contiguous()),
        lambda: g.GradList([]),
        lambda: g.GradList([x.cpu()]),
        lambda: g.GradList([x], [x.to(BF16)]),
        lambda: g.GradList([x[:, :8]]),
        lambda: g.gear_clip_grads(g.GradList([x.clone()]), 0.0),
        lambda: g.gear_clip_grads(g.GradList([x.clone()]), math.inf),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(g.GearError) as e:
            call()
        assert e.value.code == g.GEAR_ERR_INVALID, i


def test_more_rows_than_threads_of_a_launch(g):
    """2^21 workgroups of a row each and some more: the first ones take a second row."""
    rows = (1 << 21) + 5
    x = torch.zeros(rows, 2056, dtype=BF16, device="cuda")
    tail = torch.randn(6, 2056, device="cuda", generator=gen(12)).to(BF16)
    x[-6:] = tail
    gain = torch.ones(2056, device="cuda")
    g.gear_rmsnorm(x, gain, 1e-6, out=g.NormOutput(None, x, None))
    assert torch.equal(x[-6:], g.gear_rmsnorm(tail, gain, 1e-6).y) and not x[:-6].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(700, 1152), (300, 72), (40, 5000), (9, 12000)])
def test_norm_in_8_bits_is_rounded_once(g, dtype, rows, dim):
    """The 8 bits are those nearest to the norm in 64 bits, scales too: 64-bit sums differ in the last bits only, and no value of
    these lies that near to a border."""
    r = gen(rows + 2 * dim)
    x = (torch.randn(rows, dim, device="cuda", generator=r) * torch.exp(torch.randn(rows, 1, device="cuda", generator=r))).to(dtype)
    res = torch.randn(rows, dim, device="cuda", generator=r).to(dtype)
    gain = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r)
    _, y = norm_ref(x, res, gain, float(torch.tensor(1e-6)))
    out = g.gear_rmsnorm(x, gain, 1e-6, residual=res, q8=True)
    e = exponents(y)
    assert torch.equal(out.rows8.scale[:, :e.shape[1]].long() - 127, e)
    unit = torch.exp2(e.double()).repeat_interleave(128, 1)
    want = nearest8(torch.nn.functional.pad(y, (0, -dim % 128)) / unit)
    within(out.rows8.q.view(torch.float8_e4m3fn).double(), want, 0.0)
    within(out.y, (want * unit)[:, :dim], 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(5, 2056), (300, 2176), (7, 3584), (33, 4096), (3, 4104)])
def test_norm_in_8_bits_of_rows_wider_than_a_wavefront(g, dtype, rows, dim):
    """Rows of several wavefronts, whole and ragged, with and without a residual: 8 bits and scales are those of the norm in 64 bits."""
    r = gen(7 * rows + dim)
    x = torch.randn(rows, dim, device="cuda", generator=r).to(dtype)
    gain = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r)
    for res in (None, torch.randn(rows, dim, device="cuda", generator=r).to(dtype)):
        _, y = norm_ref(x, res, gain, float(torch.tensor(1e-6)))
        out = g.gear_rmsnorm(x, gain, 1e-6, residual=res, y=False, q8=True)
        e = exponents(y)
        assert torch.equal(out.rows8.scale[:, :e.shape[1]].long() - 127, e)
        want = nearest8(torch.nn.functional.pad(y, (0, -dim % 128)) / torch.exp2(e.double()).repeat_interleave(128, 1))
        within(out.rows8.q.view(torch.float8_e4m3fn).double(), want, 0.0)


def test_products_refuse_results_of_other_types(g):
    x = torch.zeros(4, 64, device="cuda", dtype=BF16)
    w = torch.zeros(64, 64, device="cuda", dtype=BF16)
    for call in (lambda d: g.gear_expert_matmul(x, g.ExpertWeights(w), out_dtype=d), lambda d: g.gear_expert_dgrad(x, g.ExpertWeights(w), out_dtype=d),
                 lambda d: g.gear_matmul8(g.gear_rows8(x), g.gear_weights8(w), out_dtype=d)):
        for other in (torch.float16, torch.float64, torch.int32):
            with pytest.raises(g.GearError):
                call(other)
        for right in (F32, BF16):
            assert not call(right).any()


@pytest.mark.parametrize("sizes,n,k", [([1, 1300, 230], 776, 200), ([1500, 0, 30], 1160, 72), ([2200, 0, 7000, 41], 264, 136), ([5300, 301], 376, 64),
                                       ([4000, 90, 33], 584, 136), ([9000, 129, 0, 7200], 1160, 72)])
def test_products_between_few_tiles_and_many(g, sizes, n, k):
    """Ragged rows of as many as each shape of tile is meant for, one at a time: 64 x 128 (twice), 128 x 128 (twice), 64 x 256 and 128 x 256."""
    for dtype in (F32, BF16):
        test_expert_products(g, dtype, sizes, n, k)
    test_products_in_8_bits(g, sizes, n, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n,k", [(20011, 72, 128), (9000, 8, 8), (40000, 72, 320), (33000, 264, 320)])
def test_weight_gradient_of_long_lists_and_few_columns(g, dtype, rows, n, k):
    """Many pieces of a small gradient, added up in shares; the same again, bit for bit."""
    r = gen(rows + n)
    dy, x = (torch.randn(rows, w, device="cuda", generator=r).to(dtype) for w in (n, k))
    a, b = dy.double(), x.double()
    dw = g.gear_expert_wgrad(dy, x)
    within(dw[0], a.t().contiguous() @ b, (rows + 8) * 2 * U * (a.abs().t().contiguous() @ b.abs()))
    assert torch.equal(dw, g.gear_expert_wgrad(dy, x))


@pytest.mark.parametrize("sizes,n,k", [([16384 + 40], 1024, 64), ([8000, 0, 8500, 130], 1024, 72), ([9000, 7400, 1], 1032, 136), ([33000], 1000, 64)])
def test_products_whose_last_round_is_halved(g, sizes, n, k):
    """A little more than one round (or two) of the largest tiles, the last of them with few rows and with many."""
    test_expert_products(g, BF16, sizes, n, k)
    test_products_in_8_bits(g, sizes, n, k)


@pytest.mark.parametrize("sizes,n,k", [([300, 41], 520, 3104), ([70, 0, 200], 776, 6152), ([129], 1160, 6200)])
def test_products_of_few_tiles_and_long_rows(g, sizes, n, k):
    """Tiles that are split over k: rows of 48 k-blocks of 128 bytes and more, whole and not."""
    test_expert_products(g, BF16, sizes, n, k)
    test_products_in_8_bits(g, sizes, n, k)
