"""The operators of a Dense Part made of experts where numbers, lists and reports reach their limits.

Tolerances are those of test_gpu_experts.py.  Of the norm's backward pass: rows of up to 128 columns are added up by 16 threads and up
to 256 by 32, at most eight values each and then a tree, which (dim / 64 + 16) u covers as well."""
import ctypes as C
import math

import pytest
import torch

from test_gpu_experts import BF16, F32, HALF, U, g, gen, norm_back_ref, norm_bound, within  # noqa: F401 (g: the fixture)

pytestmark = pytest.mark.gpu


# ---- the norm's backward pass ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(3, 72), (40, 264), (7, 1024), (5, 2056), (2, 12000)])
@pytest.mark.parametrize("size,eps", [(1e13, 1e-6), (1e14, 1e-6), (1e15, 1e-6), (1e16, 1e-6), (1e-13, 0.0), (1e-16, 1e-38), (1e-16, 1e-30)])
def test_norm_backward_of_rows_of_any_size(g, dtype, rows, dim, size, eps):
    """dx and dgain are ordinary numbers as long as the norm is: nothing on the way may leave fp32's range.  Rows lie along dy in part,
    so that what is taken off dx is as large as dx.  eps is fp32, as the call takes it."""
    eps = float(torch.tensor(eps))
    r = gen(rows + dim)
    dy = torch.randn(rows, dim, device="cuda", generator=r)
    h = ((torch.randn(rows, dim, device="cuda", generator=r) + dy) * size).to(dtype)
    dy = dy.to(dtype)
    gain = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r)
    dx, dgain, scale, total = norm_back_ref(h, gain, dy, eps)
    got, got_gain = g.gear_rmsnorm_backward(h, gain, dy, eps)
    within(got, dx, 4 * norm_bound(dim, F32) * scale + HALF[dtype] * dx.abs())
    within(got_gain, dgain, (norm_bound(dim, F32) + (rows + 8) * U) * total)


@pytest.mark.parametrize("eps", [1e-26, 1e-30, 1e-36])
def test_norm_backward_of_rows_of_zeros_and_next_to_no_eps(g, eps):
    """The definition: dx = dy gain eps^-1/2 and nothing for dgain."""
    eps = float(torch.tensor(eps))
    h, dy = torch.zeros(6, 520, device="cuda"), torch.randn(6, 520, device="cuda", generator=gen(2))
    h[3] = torch.randn(520, device="cuda", generator=gen(3))
    gain = 1 + 0.3 * torch.randn(520, device="cuda", generator=gen(4))
    dx, dgain, scale, total = norm_back_ref(h, gain, dy, eps)
    got, got_gain = g.gear_rmsnorm_backward(h, gain, dy, eps)
    within(got, dx, 4 * norm_bound(520, F32) * scale)
    within(got_gain, dgain, (norm_bound(520, F32) + 14 * U) * total)


# ---- reports of offsets that are no list ------------------------------------------------------------------------------
def operands(sizes, n, k):
    r = gen(n + k)
    rows = sum(sizes)
    off = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).cuda()
    draw = lambda *s: torch.randn(s, device="cuda", generator=r).to(BF16)
    return draw(rows, k), draw(rows, n), draw(len(sizes), n, k), off


def dirty_memory():
    """Blocks of all sizes that weights are laid out in, left full of ones to whoever is given them next."""
    torch.cuda.synchronize()
    blocks = [torch.full((1 << p,), 255, dtype=torch.uint8, device="cuda") for p in range(9, 22) for _ in range(8)]
    torch.cuda.synchronize()
    del blocks


def test_weights_report_nothing_before_the_first_product(g):
    _, _, w, _ = operands([3, 4], 72, 64)
    for _ in range(3):
        dirty_memory()
        assert g.ExpertWeights(w).status.item() == 0 and g.gear_weights8(w).status.item() == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_product_that_works_does_not_erase_the_report_of_one_that_did_not(g, kind):
    x, dy, w, good = operands([50, 50], 72, 64)
    bad = torch.tensor([0, 60, 50], dtype=torch.int32, device="cuda")
    weights = g.ExpertWeights(w) if kind == "bf16" else g.gear_weights8(w)
    call = (lambda off: g.gear_expert_matmul(x, weights, off)) if kind == "bf16" else (lambda off: g.gear_matmul8(g.gear_rows8(x), weights, off))
    try:
        call(good)
        assert weights.status.item() == 0
        call(bad)
        call(good)
        if kind == "bf16":
            g.gear_expert_dgrad(dy, weights, good)
        assert weights.status.item() == g.GEAR_ERR_RANGE
    finally:
        weights.status.zero_()
    call(good)
    assert weights.status.item() == 0                       # cleared by the caller, and only by the caller


def test_a_status_of_ones_own_is_written_by_every_product(g):
    x, _, w, good = operands([50, 50], 72, 64)
    weights, status = g.ExpertWeights(w), torch.full((1,), 7, dtype=torch.int32, device="cuda")
    g.gear_expert_matmul(x, weights, good, status=status)
    assert status.item() == 0
    g.gear_expert_matmul(x, weights, good + 1, status=status)
    assert status.item() == g.GEAR_ERR_RANGE and weights.status.item() == 0


def test_a_weight_gradient_reports_without_a_status_of_its_own(g):
    x, dy, w, good = operands([50, 50], 72, 64)
    word = g.gear_expert_status()
    want = g.gear_expert_wgrad(dy, x, good)
    assert word.item() == 0 and g.gear_expert_status(x.device) is word
    try:
        dw = torch.full((2, 72, 64), 7.0, device="cuda")
        g.gear_expert_wgrad(dy, x, torch.tensor([0, 60, 50], dtype=torch.int32, device="cuda"), dw=dw)
        assert torch.equal(g.gear_expert_wgrad(dy, x, good), want)
        g.gear_expert_matmul(x, g.ExpertWeights(w), good)
        assert word.item() == g.GEAR_ERR_RANGE and (dw == 7).all()
    finally:
        word.zero_()
    g.gear_expert_wgrad(dy, x, good)
    assert word.item() == 0


def test_reports_from_a_graph_and_from_two_streams(g):
    """Every replay reports; calls that work, on whatever stream, leave the report alone."""
    x, dy, w, good = operands([50, 50], 72, 64)
    weights, word, off = g.ExpertWeights(w), g.gear_expert_status(), good.clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        g.gear_expert_matmul(x, weights, off)
        g.gear_expert_wgrad(dy, x, off)
    try:
        for wrong in (False, True, False, True):
            off.copy_(good + 1 if wrong else good)
            graph.replay()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for _ in range(3):
                    g.gear_expert_matmul(x, weights, good)
            torch.cuda.synchronize()
            assert word.item() == (g.GEAR_ERR_RANGE if wrong else 0)
            word.zero_()
    finally:
        word.zero_()


# ---- clipping -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [40, 20_000, 200_000])
def test_clipping_of_gradients_whose_norm_fp32_does_not_hold(g, n):
    """Each gradient is finite and so is the norm in 64 bits; the reported fp32 norm is infinite, what is clipped is not lost.  One
    rounding of c and one of the result, either of which may be below the normal numbers: 2^-149."""
    a, b = torch.full((n,), 3.0e38, device="cuda"), torch.full((7,), -1.0e38, device="cuda", dtype=BF16)
    norm = math.sqrt(sum(t.double().square().sum().item() for t in (a, b)))
    out = [torch.empty_like(a), torch.empty_like(b)]
    limit = 100.0
    c = limit / norm
    assert norm > 3.5e38 and c < 1
    got = g.gear_clip_grads(g.GradList([a, b], out), limit)
    assert got.item() == math.inf
    for t, o in zip((a, b), out):
        within(o, t.double() * c, torch.full_like(t.double(), 2.0 ** -149) + (4 * U + HALF[t.dtype] + 2.0 ** -149 / c) * c * t.double().abs())


def test_lists_whose_tensors_share_memory(g):
    a, b = torch.randn(1000, device="cuda", generator=gen(1)), torch.randn(1000, device="cuda", generator=gen(2))
    before, room = a.clone(), torch.empty(2000, device="cuda")
    norm = a.double().norm().item()
    twice = g.GradList([a, a])
    assert abs(g.gear_grad_norm(twice).item() - math.sqrt(2) * norm) <= 2 * U * 2 * norm
    for refused in (lambda: g.gear_clip_grads(twice, norm / 2), lambda: g.gear_clip_grads(g.GradList([a, a[500:]]), 1.0),
                    lambda: g.GradList([a, b], [room[:1000], room[999:1999]]), lambda: g.GradList([a, b], [b, a]),
                    lambda: g.GradList([room[:1000]], [room[1:1001]])):
        with pytest.raises(g.GearError) as e:
            refused()
        assert e.value.code == g.GEAR_ERR_INVALID
    assert torch.equal(a, before)
    g.gear_clip_grads(g.GradList([a, a], [room[:1000], room[1000:]]), norm / 2)       # twice into two places
    c = norm / 2 / (math.sqrt(2) * norm + 1e-6)
    for part in (room[:1000], room[1000:]):
        within(part, a.double() * c, 4 * U * c * a.double().abs())
    g.gear_clip_grads(g.GradList([room[:1000], room[1000:]]), norm / 4)               # neighbours in place
    assert abs(room.double().norm().item() - norm / 4) <= 1e-5 * norm


# ---- many experts, some of whose rows are cut into pieces ---------------------------------------------------------------
MANY = [[i % 3 for i in range(70)], [1] * 131]
MANY[0][3], MANY[0][64], MANY[0][69] = 3000, 2500, 4100
MANY[1][0], MANY[1][66], MANY[1][130] = 5000, 1800, 2600


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k", [(8, 8), (40, 136), (72, 128), (136, 320)])
@pytest.mark.parametrize("sizes", MANY)
def test_weight_gradients_of_more_than_64_experts_some_of_them_long(g, dtype, n, k, sizes):
    """More experts than one look at the offsets finds: pieces, and the partial results before them, behind the 64th too."""
    r = gen(n + k)
    rows = sum(sizes)
    dy, x = (torch.randn(rows, w, device="cuda", generator=r).to(dtype) for w in (n, k))
    off = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).cuda()
    dw = g.gear_expert_wgrad(dy, x, off)
    at = 0
    for e, m in enumerate(sizes):
        a, b = dy[at:at + m].double(), x[at:at + m].double()
        within(dw[e], a.t().contiguous() @ b, (m + 8) * 2 * U * (a.abs().t().contiguous() @ b.abs()))
        at += m
    assert torch.equal(dw, g.gear_expert_wgrad(dy, x, off))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(1, 72), (9, 1152), (5000, 264), (700, 2056)])
def test_norm_backward_without_the_gradient_of_the_gain(g, dtype, rows, dim):
    """dgain = NULL needs no workspace and leaves dx as it is with one."""
    r = gen(rows + dim)
    h, dy = (torch.randn(rows, dim, device="cuda", generator=r).to(dtype) for _ in range(2))
    gain, dx = 1 + 0.3 * torch.randn(dim, device="cuda", generator=r), torch.empty_like(h)
    a = g.binding.gear_norm_backward_args(rows, dim, g.GEAR_F32 if dtype is F32 else g.GEAR_BF16, 1e-5, h.data_ptr(), dy.data_ptr(), None,
                                          gain.data_ptr(), dx.data_ptr(), None, dim, dim, 0, dim)
    assert g.lib.gear_rmsnorm_backward(C.byref(a), None, 0, torch.cuda.current_stream().cuda_stream) == g.GEAR_OK
    assert torch.equal(dx, g.gear_rmsnorm_backward(h, gain, dy, 1e-5)[0])


def test_a_weight_gradient_of_as_many_tiles_as_there_may_be(g):
    """2^23 tiles of 64 x 64, 137 GB of them: 2^31 threads, and as many again would be more than a launch takes."""
    torch.cuda.empty_cache()
    n, k = (1 << 20) - 8, 1 << 15
    if torch.cuda.mem_get_info()[0] < 4 * n * k + (8 << 30):
        pytest.skip("needs 146 GB of the GPU's memory")
    dy, x = torch.randn(1, n, device="cuda", generator=gen(1)), torch.randn(1, k, device="cuda", generator=gen(2))
    dw = g.gear_expert_wgrad(dy, x, torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    for at in (0, 12_345, n - 1):
        assert torch.equal(dw[0, at], dy[0, at] * x[0])     # one product each: nothing is added
    for at in (0, 777, k - 1):
        assert torch.equal(dw[0, :, at], dy[0] * x[0, at])
    assert g.gear_expert_status().item() == 0
    del dw
    torch.cuda.empty_cache()
