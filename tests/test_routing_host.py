"""What rows that choose their experts, and products in 8-bit integers, check on the host: no GPU is needed to be refused."""
import ctypes as C
import itertools

import pytest

from paper_1806_03925_amd import binding as b
from paper_1806_03925_amd import routing

INVALID, CAPACITY, OK = b.GEAR_ERR_INVALID, b.GEAR_ERR_CAPACITY, b.GEAR_OK
P = 1 << 20        # an address that is aligned and never used: every call below is refused before it could be
NAN, INF = float("nan"), float("inf")


def route(ws=P, bytes_=1 << 40, **kw):
    a = dict(rows=4, experts=12, k=2, dtype=b.GEAR_F32, score=0, groups=1, groups_kept=1, group_best=1, renormalise=1, scale=1.0, logits=P,
             ld_logits=12, bias=None, n=None, expert=P, weight=P, off=P, place=P)
    a.update(kw)
    return b.lib.gear_route(C.byref(b.gear_route_args(**a)), ws, bytes_, None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 30 + 1), dict(rows=2 ** 30, k=2), dict(experts=0), dict(experts=1025, ld_logits=1025), dict(k=0), dict(k=13),
    dict(experts=64, ld_logits=64, k=33), dict(dtype=2), dict(dtype=-1), dict(score=2), dict(score=-1), dict(groups=0), dict(groups=5),
    dict(groups=65, experts=130, ld_logits=130), dict(groups=3, groups_kept=0), dict(groups=3, groups_kept=4), dict(groups=6, groups_kept=1, k=3),
    dict(groups=3, group_best=0), dict(groups=3, group_best=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
    dict(logits=None), dict(logits=P + 2), dict(dtype=b.GEAR_BF16, logits=P + 1), dict(ld_logits=11), dict(ld_logits=1 << 20), dict(bias=P + 1),
    dict(n=P + 2), dict(expert=None), dict(weight=None), dict(expert=P + 1), dict(weight=P + 2), dict(off=None), dict(place=None),
    dict(off=P + 1), dict(place=P + 2), dict(ws=None), dict(ws=P + 16)])
def test_route_refuses(kw):
    assert route(**kw) == INVALID


def test_route_needs_its_workspace():
    size = b.lib.gear_route_workspace_bytes(4, 12, 2, 1)
    assert size >= 48 and size % 256 == 0
    assert route(bytes_=size - 1) == CAPACITY
    assert b.lib.gear_route_workspace_bytes(1 << 20, 1024, 8, 1) <= 1 << 20         # counts of 256 runs at most
    for bad in [(-1, 12, 2, 1), (4, 0, 1, 1), (4, 12, 0, 1), (4, 12, 13, 1), (1 << 30, 12, 2, 1), (4, 12, 2, 0), (4, 1025, 2, 1)]:
        assert b.lib.gear_route_workspace_bytes(*bad) == 0


def test_route_of_no_rows_without_an_order_needs_no_memory():
    assert route(rows=0, logits=None, expert=None, weight=None, off=None, place=None, ws=None) == OK


def back(**kw):
    a = dict(rows=4, experts=12, k=2, dtype=b.GEAR_F32, score=0, renormalise=1, scale=1.0, logits=P, ld_logits=12, expert=P, weight=P, dweight=P,
             dlogits=P, ld_dlogits=12)
    a.update(kw)
    return b.lib.gear_route_backward(C.byref(b.gear_route_backward_args(**a)), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(experts=0), dict(k=0), dict(k=13), dict(dtype=2), dict(score=2), dict(scale=0.0), dict(scale=NAN), dict(logits=None),
    dict(logits=P + 2), dict(expert=None), dict(weight=None), dict(dweight=None), dict(dlogits=None), dict(dlogits=P + 1), dict(dweight=P + 2),
    dict(ld_logits=11), dict(ld_dlogits=11), dict(ld_dlogits=1 << 20)])
def test_route_backward_refuses(kw):
    assert back(**kw) == INVALID


def gather(x=P, dtype=b.GEAR_BF16, ld_x=64, rows=4, dim=64, place=P, k=2, xs=P, ld_xs=64):
    return b.lib.gear_expert_gather(x, dtype, ld_x, rows, dim, place, k, xs, ld_xs, None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(x=P + 8), dict(dtype=2), dict(ld_x=56), dict(ld_x=68), dict(ld_x=1 << 20), dict(rows=-1), dict(rows=2 ** 30), dict(dim=0),
    dict(dim=60), dict(dim=65544, ld_x=65544, ld_xs=65544), dict(place=None), dict(place=P + 2), dict(k=0), dict(k=33), dict(xs=None),
    dict(xs=P + 4), dict(ld_xs=32)])
def test_gather_refuses(kw):
    assert gather(**kw) == INVALID


def combine(**kw):
    a = dict(rows=4, dim=64, k=2, dtype=b.GEAR_BF16, y=P, residual=None, place=P, weight=P, out=P, ld_y=64, ld_residual=0, ld_out=64)
    a.update(kw)
    return b.lib.gear_expert_combine(C.byref(b.gear_expert_combine_args(**a)), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(dim=4), dict(dim=65544), dict(k=0), dict(k=33), dict(dtype=2), dict(y=None), dict(y=P + 8), dict(ld_y=60), dict(residual=P),
    dict(residual=P + 8, ld_residual=64), dict(place=None), dict(place=P + 1), dict(weight=P + 2), dict(out=None), dict(ld_out=72 - 4),
    dict(ld_out=1 << 20)])
def test_combine_refuses(kw):
    assert combine(**kw) == INVALID


def combine_back(**kw):
    a = dict(rows=4, dim=64, k=2, dtype=b.GEAR_BF16, dout=P, y=P, place=P, weight=P, dy=P, dweight=P, ld_dout=64, ld_y=64, ld_dy=64)
    a.update(kw)
    return b.lib.gear_expert_combine_backward(C.byref(b.gear_expert_combine_backward_args(**a)), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(dim=12), dict(k=0), dict(dtype=2), dict(dout=None), dict(dout=P + 8), dict(y=None), dict(place=None), dict(weight=None),
    dict(dy=None, dweight=None), dict(dy=P + 8), dict(dweight=P + 2), dict(ld_dout=56), dict(ld_y=56), dict(ld_dy=56)])
def test_combine_backward_refuses(kw):
    assert combine_back(**kw) == INVALID


def test_calls_on_no_rows_need_no_memory():
    assert gather(rows=0, x=None, place=None, xs=None) == OK
    assert combine(rows=0, y=None, place=None, out=None) == OK
    assert combine_back(rows=0, dout=None, y=None, place=None, weight=None) == OK
    assert back(rows=0, logits=None, expert=None, weight=None, dweight=None, dlogits=None) == OK
    assert b.lib.gear_rows_i8(None, 0, 0, 0, 64, None, 1, None, None, None) == OK


def rows_i8(x=P, dtype=b.GEAR_BF16, ld_x=64, rows=4, dim=64, place=None, k=1, q=P, scale=P):
    return b.lib.gear_rows_i8(x, dtype, ld_x, rows, dim, place, k, q, scale, None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(x=P + 8), dict(dtype=2), dict(dtype=3), dict(ld_x=56), dict(rows=-1), dict(dim=4), dict(dim=65544), dict(k=2),
    dict(place=P + 2), dict(place=P, k=33), dict(q=None), dict(q=P + 8), dict(scale=None), dict(scale=P + 2)])
def test_rows_i8_refuses(kw):
    assert rows_i8(**kw) == INVALID


def test_sizes_of_weights():
    assert b.lib.gear_packed_i8_bytes(3, 72, 136) == 3 * 3 * 2 * 4096
    for bad in [(0, 8, 8), (1025, 8, 8), (1, 12, 8), (1, 8, 12), (1, 0, 8), (1, 8, 65544), (1, 1 << 20, 8)]:
        assert b.lib.gear_packed_i8_bytes(*bad) == 0


@pytest.mark.parametrize("kw", [
    dict(w=None), dict(w=P + 8), dict(code=2), dict(experts=0), dict(n=12), dict(k=4), dict(packed=None), dict(packed=P + 8), dict(scale=None),
    dict(scale=P + 4), dict(experts=1024, n=(1 << 20) - 8)])
def test_pack_i8_refuses(kw):
    a = dict(w=P, code=0, experts=2, n=72, k=64, packed=P, scale=P)
    a.update(kw)
    assert b.lib.gear_pack_weights_i8(a["w"], a["code"], a["experts"], a["n"], a["k"], a["packed"], a["scale"], None) == INVALID


def product(**kw):
    a = dict(out_dtype=b.GEAR_BF16, rows=4, K=64, N=72, experts=2, x=P, x_scale=P, packed=P, w_scale=P, off=P, out=P, ld_x=128, ld_out=72, status=P)
    a.update(kw)
    return b.lib.gear_product_i8(C.byref(b.gear_i8_args(**a)), None)


@pytest.mark.parametrize("kw", [
    dict(out_dtype=2), dict(out_dtype=3), dict(rows=-1), dict(rows=2 ** 30 + 1), dict(K=0), dict(K=60), dict(K=65544, ld_x=65664), dict(N=70),
    dict(experts=0), dict(experts=1025), dict(x=None), dict(x=P + 8), dict(x_scale=None), dict(x_scale=P + 2), dict(packed=None), dict(packed=P + 8),
    dict(w_scale=None), dict(w_scale=P + 8), dict(off=None), dict(out=None), dict(out=P + 8), dict(status=None), dict(ld_x=64), dict(ld_x=136),
    dict(ld_out=64), dict(ld_out=1 << 20), dict(rows=2 ** 30, N=(1 << 20) - 8, ld_out=(1 << 20) - 8)])
def test_product_i8_refuses(kw):
    assert product(**kw) == INVALID


def test_the_other_products_do_not_take_integers():
    """GEAR_I8 stands for the type of these weights alone."""
    assert b.lib.gear_packed_weights_bytes(b.GEAR_I8, 1, 8, 8, 0) == 0
    a = b.gear_expert_args(dtype=b.GEAR_I8, out_dtype=1, rows=4, K=64, N=72, experts=1, x=P, packed=P, out=P, ld_x=128, ld_out=72)
    assert b.lib.gear_expert_product(C.byref(a), None) == INVALID


def test_memory_of_results_is_apart_from_what_is_read():
    """Every byte listed: nothing that shares one is let through, and of one distance between rows nothing that shares none is refused."""
    def lines(at, rows, apart, width):
        return routing._Lines(at, rows, apart, width), {at + r * apart + i for r in range(rows) for i in range(width)}

    def refused(*a):
        try:
            routing._apart(*a)
            return False
        except b.GearError:
            return True
    some = [lines(at, rows, apart, width) for at, rows, (apart, width) in itertools.product(range(100, 131, 3), (0, 1, 3), ((0, 4), (4, 4), (9, 3), (9, 6)))]
    for (out, mine), (other, its) in itertools.product(some, some):
        shared = bool(mine & its)
        assert refused(out, other, "", "") >= shared
        if out.apart == other.apart > 0 and not shared:
            # a row that wraps round the distance is refused though it may lie beyond the other's last one
            between = (other.at - out.at) % out.apart
            assert not refused(out, other, "", "") or between < out.width or between + other.width > out.apart
        assert refused(out, other, "", "", True) == (refused(out, other, "", "") and out != other)
