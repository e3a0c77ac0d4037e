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
