"""What the operators of a Dense Part made of experts check on the host: no GPU is needed to be refused."""
import ctypes as C

import pytest

from paper_1806_03925_amd import binding as b

INVALID, CAPACITY, OK = b.GEAR_ERR_INVALID, b.GEAR_ERR_CAPACITY, b.GEAR_OK
P = 1 << 20        # an address that is aligned and never used: every call below is refused before it could be


def norm(**kw):
    a = dict(rows=4, dim=64, dtype=b.GEAR_BF16, eps=1e-6, x=P, residual=None, gain=P, sum=None, y=P, ld_x=64, ld_residual=0, ld_sum=0,
             ld_y=64, q8=None, scale=None)
    a.update(kw)
    return b.lib.gear_rmsnorm(C.byref(b.gear_norm_args(**a)), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 31), dict(dim=0), dict(dim=12), dict(dim=65544), dict(dtype=2), dict(dtype=-1), dict(eps=-1e-6),
    dict(eps=float("nan")), dict(x=None), dict(gain=None), dict(gain=P + 4), dict(y=None), dict(x=P + 8), dict(ld_x=56), dict(ld_x=68),
    dict(ld_x=1 << 20), dict(residual=P), dict(sum=P, ld_sum=64), dict(q8=P), dict(scale=P), dict(q8=P + 4, scale=P), dict(q8=P, scale=P + 2)])
def test_norm_refuses(kw):
    assert norm(**kw) == INVALID


def test_norm_of_no_rows_needs_no_memory():
    assert norm(rows=0, x=None, gain=None) == OK


def test_sizes():
    assert b.lib.gear_rows8_ld(1) == 128 and b.lib.gear_rows8_ld(128) == 128 and b.lib.gear_rows8_ld(136) == 256
    assert b.lib.gear_scales8_ld(512) == 4 and b.lib.gear_scales8_ld(520) == 8 and b.lib.gear_rows8_ld(0) == 0
    # 3 experts x 3 strips of 32 outputs x 2 blocks of 64 bf16 values x 4 KB
    assert b.lib.gear_packed_weights_bytes(b.GEAR_BF16, 3, 72, 104, 0) == 3 * 3 * 2 * 4096
    assert b.lib.gear_packed_weights_bytes(b.GEAR_BF16, 3, 72, 104, 1) == 3 * 4 * 2 * 4096
    assert b.lib.gear_packed_weights_bytes(b.GEAR_F32, 1, 8, 8, 0) == 4096
    assert b.lib.gear_packed_weights_bytes(b.GEAR_E4M3, 1, 40, 136, 0) == 2 * 2 * 4096
    assert b.lib.gear_weight_scales_bytes(2, 136, 136) == 2 * 2 * 4
    for bad in [(b.GEAR_E4M3, 1, 8, 8, 1), (3, 1, 8, 8, 0), (0, 0, 8, 8, 0), (0, 1, 12, 8, 0), (0, 1, 8, 4, 0), (0, 1025, 8, 8, 0)]:
        assert b.lib.gear_packed_weights_bytes(*bad) == 0


def product(**kw):
    a = dict(dtype=b.GEAR_BF16, out_dtype=b.GEAR_BF16, rows=4, K=64, N=72, experts=2, x=P, x_scale=None, packed=P, w_scale=None, off=P,
             out=P, ld_x=64, ld_out=72, status=P)
    a.update(kw)
    return b.lib.gear_expert_product(C.byref(b.gear_expert_args(**a)), None)


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(out_dtype=2), dict(dtype=b.GEAR_F32), dict(rows=-1), dict(rows=2 ** 30 + 1), dict(K=0), dict(K=60), dict(N=70),
    dict(experts=0), dict(experts=1025), dict(x=None), dict(x=P + 8), dict(packed=None), dict(packed=P + 8), dict(off=None), dict(out=None),
    dict(out=P + 8), dict(status=None), dict(ld_x=56), dict(ld_x=66), dict(ld_out=64), dict(ld_out=1 << 20), dict(dtype=b.GEAR_E4M3),
    dict(dtype=b.GEAR_E4M3, x_scale=P, w_scale=P, ld_x=64), dict(dtype=b.GEAR_E4M3, x_scale=P, ld_x=128),
    dict(dtype=b.GEAR_E4M3, w_scale=P, ld_x=128), dict(dtype=b.GEAR_E4M3, x_scale=P + 1, w_scale=P, ld_x=128),
    dict(rows=2 ** 30, N=(1 << 20) - 8, ld_out=(1 << 20) - 8)])
def test_product_refuses(kw):
    assert product(**kw) == INVALID


def wgrad(ws=P, bytes_=1 << 40, **kw):
    a = dict(dtype=b.GEAR_BF16, rows=4, K=64, N=72, experts=2, dy=P, x=P, off=P, dw=P, ld_dy=72, ld_x=64, status=P)
    a.update(kw)
    return b.lib.gear_expert_wgrad(C.byref(b.gear_expert_wgrad_args(**a)), ws, bytes_, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(rows=-1), dict(K=12), dict(N=4), dict(experts=0), dict(dy=None), dict(x=P + 2), dict(off=None), dict(dw=None),
    dict(dw=P + 4), dict(ld_dy=64), dict(ld_x=65), dict(status=None), dict(ws=None), dict(ws=P + 16)])
def test_wgrad_refuses(kw):
    assert wgrad(**kw) == INVALID


def test_workspaces_that_are_too_small():
    assert wgrad(bytes_=0) == CAPACITY
    a = b.gear_norm_backward_args(rows=4, dim=64, dtype=1, eps=1e-6, h=P, dy=P, dsum=None, gain=P, dx=P, dgain=P, ld_h=64, ld_dy=64, ld_dsum=0,
                                  ld_dx=64)
    size = b.lib.gear_norm_backward_workspace_bytes(4, 64)
    assert size >= 256 and b.lib.gear_rmsnorm_backward(C.byref(a), P, size - 1, None) == CAPACITY
    assert b.lib.gear_rmsnorm_backward(C.byref(a), None, size, None) == INVALID
    assert b.lib.gear_clip_grads(P, 1, 1, 1.0, P, b.lib.gear_grad_workspace_bytes(1) - 1, P, None) == CAPACITY


def test_gradient_lists():
    lengths = [0, 1, 100_000, 0, 7]
    t = (b.gear_grad_tensor * 5)(*[b.gear_grad_tensor(P, P, n, i % 2) for i, n in enumerate(lengths)])
    room = (C.c_uint8 * b.lib.gear_grad_list_bytes(5))()
    chunks = C.c_int64(-1)
    assert b.lib.gear_grad_list_pack(t, 5, room, C.byref(chunks)) == OK
    assert chunks.value >= 3            # every tensor that has elements is a piece of work of its own
    t[2].src = None
    assert b.lib.gear_grad_list_pack(t, 5, room, C.byref(chunks)) == INVALID
    t[2].src = P + 2                    # fp32 on two bytes
    assert b.lib.gear_grad_list_pack(t, 5, room, C.byref(chunks)) == INVALID
    t[2].src, t[2].n = P, -1
    assert b.lib.gear_grad_list_pack(t, 5, room, C.byref(chunks)) == INVALID
    t[2].n, t[2].dtype = 1, 2
    assert b.lib.gear_grad_list_pack(t, 5, room, C.byref(chunks)) == INVALID
    assert b.lib.gear_grad_list_bytes(0) == 0
    for limit in (0.0, -1.0, float("inf"), float("nan")):
        assert b.lib.gear_clip_grads(P, 1, 1, limit, P, 1 << 30, P, None) == INVALID
